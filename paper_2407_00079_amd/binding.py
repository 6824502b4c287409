"""Binding of ``libmooncake_hip.so`` (ctypes, and ``_mccall`` for the calls that enqueue work): argument marshalling only.

Function names and argument order are those of ``include/mc.h``.  torch is used
for device memory and streams; every step of the path runs in the library's
kernels.  There is no fallback: if the library has not been built, loading
raises.
"""
from __future__ import annotations

import array
import ctypes
import os
from typing import Optional

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libmooncake_hip.so")

MC_OK = 0
MC_ERR_NULL, MC_ERR_SHAPE, MC_ERR_UNSUPPORTED, MC_ERR_ALIGN, MC_ERR_RANGE, MC_ERR_WORKSPACE, MC_ERR_HIP = range(1, 8)
MC_DTYPE_BF16, MC_DTYPE_F32 = 0, 1

EXPORTS = ("mc_status_string", "mc_prefill_attn_workspace_bytes", "mc_prefill_attn_paged",
           "mc_kv_pack_layer", "mc_kv_unpack_layer", "mc_kv_append_workspace_bytes", "mc_kv_append_paged",
           "mc_prefill_attn_split_workspace_bytes", "mc_prefill_attn_paged_split", "mc_attn_merge_lse",
           "mc_kv_load_layer", "mc_kv_store_layer", "mc_prefix_hash_workspace_bytes", "mc_prefix_hash",
           "mc_prefix_match_workspace_bytes", "mc_prefix_match", "mc_kv_page_order", "mc_kv_pack_layer_ordered",
           "mc_kv_unpack_layer_ordered", "mc_prefill_attn_suggest_kv_splits", "mc_kv_check_page_ids",
           "mc_prefill_attn_plan", "mc_prefill_attn_prepare", "mc_prefill_attn_run", "mc_prefill_attn_run_split",
           "mc_kv_append_run", "mc_prefill_attn_auto_workspace_bytes", "mc_prefill_attn_auto",
           "mc_prefill_attn_paged_noalloc", "mc_rope_init", "mc_kv_rope_append_paged", "mc_kv_rope_append_run",
           "mc_kv_rope_append_decode", "mc_decode_attn_workspace_bytes", "mc_decode_attn_paged",
           "mc_kv_pages_workspace_bytes", "mc_kv_pages_fork", "mc_kv_pages_grow", "mc_kv_pages_free", "mc_kv_pages_compact",
           "mc_kv_pages_remap", "mc_kv_copy_pages")
MC_PAGES_SHORT, MC_PAGES_BAD_ROW, MC_PAGES_BAD_ID = 1, 2, 4
MC_MAX_COPY_LAYERS = 128
MC_ROPE_HALF, MC_ROPE_PAIRS = 0, 1
MC_ROPE_PLAIN, MC_ROPE_LINEAR, MC_ROPE_BASE, MC_ROPE_BY_PARTS = 0, 1, 2, 3
MC_MAX_KV_SPLITS = 256


class McAttnParams(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_pages", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float)]


class McAttnPlan(ctypes.Structure):
    _fields_ = [("n_items", ctypes.c_int32), ("batch", ctypes.c_int32), ("kv_splits", ctypes.c_int32),
                ("need_pages", ctypes.c_int32), ("total_new_tokens", ctypes.c_int64), ("reqs_offset", ctypes.c_int64),
                ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class McRopeParams(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("layout", ctypes.c_int32), ("norm_eps", ctypes.c_float), ("gain", ctypes.c_float),
                ("inv_freq", ctypes.c_double * 64)]


class McError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: mc_status {status} ({status_string(status)})")
        self.status = status


_lib = None


def lib():
    """The loaded library; raises if it was never built (run ``__graft_entry__.build()``)."""
    global _lib, _call, _misfit, _row_stride
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2407_00079_amd.build` "
                               "(there is no CPU fallback)")
        # torch first: its bundled HIP runtime must be the one in the process, so that the
        # streams and device pointers it hands out belong to the runtime this library calls
        import torch  # noqa: F401
        l = ctypes.CDLL(LIB_PATH)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        l.mc_status_string.restype = ctypes.c_char_p
        l.mc_status_string.argtypes = [ctypes.c_int]
        l.mc_prefill_attn_workspace_bytes.restype = ctypes.c_size_t
        l.mc_prefill_attn_workspace_bytes.argtypes = [ctypes.POINTER(McAttnParams), i32, i64]
        l.mc_prefill_attn_paged.restype = ctypes.c_int
        l.mc_prefill_attn_paged.argtypes = [ctypes.POINTER(McAttnParams), vp, vp, vp, vp, i32, vp, vp, i32,
                                            vp, vp, vp, ctypes.c_size_t, vp]
        for f in (l.mc_kv_pack_layer, l.mc_kv_unpack_layer):
            f.restype = ctypes.c_int
            f.argtypes = [vp, vp, i64, i64, vp, i64, vp, vp, vp]
        l.mc_kv_page_order.restype = ctypes.c_int
        l.mc_kv_page_order.argtypes = [vp, i64, vp, vp]
        l.mc_kv_check_page_ids.restype = ctypes.c_int
        l.mc_kv_check_page_ids.argtypes = [vp, i64, i64, vp, vp]
        for f in (l.mc_kv_pack_layer_ordered, l.mc_kv_unpack_layer_ordered):
            f.restype = ctypes.c_int
            f.argtypes = [vp, vp, i64, i64, vp, vp, i64, vp, vp, vp]
        l.mc_kv_append_workspace_bytes.restype = ctypes.c_size_t
        l.mc_kv_append_workspace_bytes.argtypes = [i32]
        l.mc_kv_append_paged.restype = ctypes.c_int
        l.mc_kv_append_paged.argtypes = [ctypes.POINTER(McAttnParams), vp, vp, vp, vp, vp, i32, vp, vp, i32, vp,
                                         ctypes.c_size_t, vp]
        l.mc_prefill_attn_split_workspace_bytes.restype = ctypes.c_size_t
        l.mc_prefill_attn_split_workspace_bytes.argtypes = [ctypes.POINTER(McAttnParams), i32, i64, i32]
        pp, pl_ = ctypes.POINTER(McAttnParams), ctypes.POINTER(McAttnPlan)
        l.mc_prefill_attn_auto_workspace_bytes.restype = ctypes.c_size_t
        l.mc_prefill_attn_auto_workspace_bytes.argtypes = [pp, vp, vp, i32]
        l.mc_prefill_attn_auto.restype = ctypes.c_int
        l.mc_prefill_attn_auto.argtypes = [pp, vp, vp, vp, vp, i32, vp, vp, i32, vp, vp, vp, ctypes.c_size_t, vp]
        l.mc_prefill_attn_paged_noalloc.restype = ctypes.c_int
        l.mc_prefill_attn_paged_noalloc.argtypes = [pp, vp, vp, vp, vp, i32, vp, vp, i32, vp, vp, vp]
        l.mc_prefill_attn_prepare.restype = ctypes.c_int
        l.mc_prefill_attn_prepare.argtypes = [pp, vp, vp, i32, i32, vp, ctypes.c_size_t, vp, pl_]
        l.mc_prefill_attn_run.restype = ctypes.c_int
        l.mc_prefill_attn_run.argtypes = [pp, pl_, vp, vp, vp, vp, i32, vp, vp, vp, vp]
        l.mc_prefill_attn_run_split.restype = ctypes.c_int
        l.mc_prefill_attn_run_split.argtypes = [pp, pl_, vp, vp, vp, vp, i32, vp, vp, vp, vp]
        l.mc_kv_append_run.restype = ctypes.c_int
        l.mc_kv_append_run.argtypes = [pp, pl_, vp, vp, vp, vp, vp, i32, vp, vp]
        l.mc_prefill_attn_plan.restype = ctypes.c_int
        l.mc_prefill_attn_plan.argtypes = [ctypes.POINTER(McAttnParams), vp, vp, i32, i32, vp, i64, vp]
        l.mc_prefill_attn_suggest_kv_splits.restype = ctypes.c_int32
        l.mc_prefill_attn_suggest_kv_splits.argtypes = [ctypes.POINTER(McAttnParams), vp, vp, i32]
        l.mc_prefill_attn_paged_split.restype = ctypes.c_int
        l.mc_prefill_attn_paged_split.argtypes = [ctypes.POINTER(McAttnParams), vp, vp, vp, vp, i32, vp, vp, i32, i32,
                                                  vp, vp, vp, ctypes.c_size_t, vp]
        l.mc_kv_load_layer.restype = ctypes.c_int
        l.mc_kv_load_layer.argtypes = [vp, vp, vp, vp, i64, i64, vp, i64, vp, vp, vp]
        l.mc_kv_store_layer.restype = ctypes.c_int
        l.mc_kv_store_layer.argtypes = [vp, vp, i64, i64, vp, i64, vp, vp, vp, vp, vp]
        l.mc_prefix_hash_workspace_bytes.restype = ctypes.c_size_t
        l.mc_prefix_hash_workspace_bytes.argtypes = [i32]
        l.mc_prefix_hash.restype = ctypes.c_int
        l.mc_prefix_hash.argtypes = [vp, vp, i32, i32, vp, vp, ctypes.c_size_t, vp]
        l.mc_prefix_match_workspace_bytes.restype = ctypes.c_size_t
        l.mc_prefix_match_workspace_bytes.argtypes = [i32, i32]
        l.mc_prefix_match.restype = ctypes.c_int
        l.mc_prefix_match.argtypes = [vp, vp, i32, vp, vp, i32, vp, vp, vp, vp, ctypes.c_size_t, vp]
        l.mc_attn_merge_lse.restype = ctypes.c_int
        l.mc_attn_merge_lse.argtypes = [vp, vp, i32, i64, i32, i32, vp, vp, vp]
        f64, rp = ctypes.c_double, ctypes.POINTER(McRopeParams)
        l.mc_rope_init.restype = ctypes.c_int
        l.mc_rope_init.argtypes = [rp, i32, f64, i32, f64, f64, f64, f64]
        l.mc_kv_rope_append_paged.restype = ctypes.c_int
        l.mc_kv_rope_append_paged.argtypes = [pp, rp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, i32, vp, ctypes.c_size_t, vp]
        l.mc_kv_rope_append_run.restype = ctypes.c_int
        l.mc_kv_rope_append_run.argtypes = [pp, pl_, rp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp]
        l.mc_kv_rope_append_decode.restype = ctypes.c_int
        l.mc_kv_rope_append_decode.argtypes = [pp, rp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, i32, vp]
        l.mc_decode_attn_workspace_bytes.restype = ctypes.c_size_t
        l.mc_decode_attn_workspace_bytes.argtypes = [pp, i32]
        l.mc_decode_attn_paged.restype = ctypes.c_int
        l.mc_decode_attn_paged.argtypes = [pp, vp, vp, vp, vp, i32, vp, i32, vp, vp, vp, ctypes.c_size_t, vp]
        sz = ctypes.c_size_t
        l.mc_kv_pages_workspace_bytes.restype = sz
        l.mc_kv_pages_workspace_bytes.argtypes = [i64, i32]
        state = [vp, i64, vp, i32, i32, vp, i32]           # counts, pages, tables, their columns, page size, lengths, rows
        for f, more in ((l.mc_kv_pages_fork, [vp, vp, i32, vp, vp, vp, sz]), (l.mc_kv_pages_grow, [vp, vp, vp, sz]),
                        (l.mc_kv_pages_free, [vp, i32, vp]), (l.mc_kv_pages_remap, [vp, vp, i32])):
            f.restype = ctypes.c_int
            f.argtypes = [*state, *more, vp]
        l.mc_kv_pages_compact.restype = ctypes.c_int
        l.mc_kv_pages_compact.argtypes = [vp, i64, i32, vp, vp, vp, sz, vp]
        l.mc_kv_copy_pages.restype = ctypes.c_int
        l.mc_kv_copy_pages.argtypes = [vp, vp, i32, i64, i64, vp, vp, i32, vp]
        try:
            from . import _mccall
        except ModuleNotFoundError:                        # none was built for this Python
            _function.update((name, getattr(l, name)) for name in EXPORTS)
            _call = _call_by_ctypes
        else:
            _function.update((name, ctypes.cast(getattr(l, name), ctypes.c_void_p).value) for name in EXPORTS)
            _call, _misfit, _row_stride = _mccall.call, _mccall.misfit, _mccall.row_stride
        _lib = l
    return _lib


_function: dict = {}           # the library's functions, as `_call` takes them
_call = None                   # csrc/pycall.cpp, or _call_by_ctypes


def _call_by_ctypes(function, kinds: str, *args) -> int:
    """What csrc/pycall.cpp does, for an interpreter it was not built for."""
    keep, given = [], []
    for kind, a in zip(kinds, args):
        if kind == "p":
            a = _dev_ptr(a)
        elif kind == "s" and a is not None:
            a = ctypes.byref(a)
        elif kind in "IQ":
            keep.append(a if isinstance(a, _Ints) else _Ints("i" if kind == "I" else "q", a, len(a)))
            a = keep[-1].at
        given.append(a)
    return function(*given)


# How each argument of the calls that enqueue work is handed over, one letter an argument (csrc/pycall.cpp says what they mean).
_KINDS = {
    "mc_prefill_attn_paged": "sppppiIIipppii",
    "mc_prefill_attn_auto": "sppppiIIipppii",
    "mc_prefill_attn_paged_noalloc": "sppppiIIippi",
    "mc_prefill_attn_run": "ssppppipppi",
    "mc_kv_append_run": "sspppppipi",
    "mc_kv_pack_layer": "ppiipippi",
    "mc_kv_unpack_layer": "ppiipippi",
    "mc_kv_page_order": "pipi",
    "mc_kv_pack_layer_ordered": "ppiippippi",
    "mc_kv_unpack_layer_ordered": "ppiippippi",
    "mc_prefix_hash": "pQiippii",
    "mc_prefix_match": "pQipQippppii",
    "mc_kv_append_paged": "spppppiIIipii",
}
# ... and of those that keep the cache beside the prefill's attention (strides: three integers in a ctypes array).
_CACHE_KINDS = {
    "mc_kv_rope_append_paged": "sspppsppppppiIIipii",
    "mc_kv_rope_append_run": "ssspppsppppppipi",
    "mc_kv_rope_append_decode": "sspppsppppppipii",
    "mc_decode_attn_paged": "sppppipipppii",
    "mc_kv_pages_fork": "pipiipippipppii",
    "mc_kv_pages_grow": "pipiipipppii",
    "mc_kv_pages_free": "pipiipipipi",
    "mc_kv_pages_compact": "piipppii",
    "mc_kv_pages_remap": "pipiipippii",
    "mc_kv_copy_pages": "QQiiippii",
}
_ALL_KINDS = {**_KINDS, **_CACHE_KINDS}


def _enqueue(name: str, *args) -> None:
    """The library's function ``name`` with arguments as _KINDS and _CACHE_KINDS have them."""
    if _call is None:
        lib()
    st = _call(_function[name], _ALL_KINDS[name], *args)
    if st != MC_OK:
        raise McError(st, name)


def _params(params):
    if params is not None and not isinstance(params, McAttnParams):
        raise TypeError(f"McAttnParams wanted, not {type(params).__name__}")
    return params


def _plan(plan):
    if not isinstance(plan, McAttnPlan):
        raise TypeError(f"McAttnPlan wanted, not {type(plan).__name__}")
    return plan


def status_string(status: int) -> str:
    return lib().mc_status_string(int(status)).decode()


def _dev_ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _nbytes(t) -> int:
    return 0 if t is None else t.nbytes


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        return _current_stream() or None
    return stream.cuda_stream or None


_raw_stream = _device = None


def _current_stream() -> int:
    """Handle of torch's current stream of the current device.  torch.cuda.current_stream() builds a Stream object
    through several Python layers; small calls are bound by the host, so the handle is asked for directly where this torch
    can (0.15 us)."""
    global _raw_stream, _device
    if _raw_stream is not None:
        return _raw_stream(_device())
    import torch
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw is None or device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    _device, _raw_stream = device, raw                     # in this order: a thread that sees the second uses both
    return raw(device())


def _ask_torch_again() -> None:
    """In a forked child: torch, not the parent's runtime, says whether the GPU can be used there."""
    global _raw_stream, _device
    _raw_stream = _device = None


os.register_at_fork(after_in_child=_ask_torch_again)


def _on(stream) -> int:
    return _current_stream() if stream is None else stream.cuda_stream or 0


class _Ints:
    """Host ints in C memory (int32 "i" or int64 "q").  array.array converts a list several times faster than a ctypes array
    does (65 offsets: 2.6 us against 12.3); what it refuses (floats, values that do not fit, a list that does not have the
    `n` entries asked for, an empty list's missing address) is converted the general way."""
    __slots__ = ("keep", "at")

    def __init__(self, code: str, values, n: int):
        try:
            if n == 0 or len(values) != n or isinstance(values, (bytes, bytearray)):
                raise TypeError
            self.keep = array.array(code, values)
            self.at = self.keep.buffer_info()[0]
        except (TypeError, OverflowError):
            kind = ctypes.c_int32 if code == "i" else ctypes.c_int64
            self.keep = (kind * max(n, 1))(*[int(x) for x in values])
            self.at = ctypes.addressof(self.keep)

    def __index__(self):
        return self.at


def _ints(code: str, values, n: int):
    """What stands for ``n`` host ints in a call: the list itself, which the call lays out, or its C copy."""
    return values if type(values) is list and len(values) == n and n > 0 else _Ints(code, values, n)


def _lens(prefix_lens, new_lens):
    batch = len(prefix_lens)
    return batch, _Ints("i", prefix_lens, batch), _Ints("i", new_lens, batch)


def mc_prefill_attn_workspace_bytes(params: McAttnParams, batch: int, total_new_tokens: int) -> int:
    return int(lib().mc_prefill_attn_workspace_bytes(ctypes.byref(params), batch, total_new_tokens))


def mc_prefill_attn_paged_raw(params, q, k_pool, v_pool, block_tables, max_pages_per_req, prefix_lens, new_lens,
                              batch, out, lse, workspace, workspace_bytes, hip_stream) -> int:
    """Plain-pointer call: every argument is an int address / ctypes object; returns the status."""
    return int(lib().mc_prefill_attn_paged(ctypes.byref(params) if params is not None else None, q, k_pool, v_pool,
                                           block_tables, max_pages_per_req, prefix_lens, new_lens, batch, out, lse,
                                           workspace, workspace_bytes, hip_stream))


def mc_prefill_attn_paged(params: McAttnParams, q, k_pool, v_pool, block_tables, prefix_lens, new_lens,
                          out, lse=None, workspace=None, stream=None) -> None:
    """Enqueue attention on ``stream`` (torch stream; default: current).

    q, k_pool, v_pool, out: torch device tensors; block_tables: int32 device
    tensor [batch, max_pages]; prefix_lens / new_lens: host sequences of ints;
    workspace: uint8 device tensor of at least the size the library asks for.
    """
    n = len(prefix_lens)
    _enqueue("mc_prefill_attn_paged", _params(params), q, k_pool, v_pool, block_tables,
             _max_pages(block_tables), _ints("i", prefix_lens, n), _ints("i", new_lens, n), n, out, lse, workspace,
             _nbytes(workspace), _on(stream))


def mc_prefill_attn_split_workspace_bytes(params: McAttnParams, batch: int, total_new_tokens: int,
                                          kv_splits: int) -> int:
    return int(lib().mc_prefill_attn_split_workspace_bytes(ctypes.byref(params), batch, total_new_tokens, kv_splits))


def mc_prefill_attn_auto_workspace_bytes(params: McAttnParams, prefix_lens, new_lens) -> int:
    batch, pl, nl = _lens(prefix_lens, new_lens)
    return int(lib().mc_prefill_attn_auto_workspace_bytes(ctypes.byref(params), pl.at, nl.at, batch))


def mc_prefill_attn_auto(params: McAttnParams, q, k_pool, v_pool, block_tables, prefix_lens, new_lens, out, lse,
                         workspace, stream=None) -> None:
    """mc_prefill_attn_paged with the whole-row / key-slices choice made by the library (larger workspace)."""
    n = len(prefix_lens)
    _enqueue("mc_prefill_attn_auto", _params(params), q, k_pool, v_pool, block_tables,
             _max_pages(block_tables), _ints("i", prefix_lens, n), _ints("i", new_lens, n), n, out, lse, workspace,
             _nbytes(workspace), _on(stream))


def mc_prefill_attn_paged_noalloc_raw(params, q, k_pool, v_pool, block_tables, max_pages_per_req, prefix_lens,
                                      new_lens, batch, out, lse, hip_stream) -> int:
    return int(lib().mc_prefill_attn_paged_noalloc(ctypes.byref(params) if params is not None else None, q, k_pool,
                                                   v_pool, block_tables, max_pages_per_req, prefix_lens, new_lens,
                                                   batch, out, lse, hip_stream))


def mc_prefill_attn_paged_noalloc(params: McAttnParams, q, k_pool, v_pool, block_tables, prefix_lens, new_lens, out,
                                  lse=None, stream=None) -> None:
    """mc_prefill_attn_paged without a workspace: the work list is built on the device in the library's own
    fixed array (no allocation, no upload)."""
    n = len(prefix_lens)
    _enqueue("mc_prefill_attn_paged_noalloc", _params(params), q, k_pool, v_pool, block_tables,
             _max_pages(block_tables), _ints("i", prefix_lens, n), _ints("i", new_lens, n), n, out, lse, _on(stream))


def _max_pages(block_tables) -> int:
    return block_tables.size(1) if block_tables is not None and block_tables.dim() == 2 else 0


def mc_prefill_attn_prepare(params: McAttnParams, prefix_lens, new_lens, kv_splits: int, workspace,
                            stream=None) -> McAttnPlan:
    """Build and upload the work list and request table of a batch ONCE; the returned plan drives any number of
    mc_prefill_attn_run / mc_prefill_attn_run_split / mc_kv_append_run calls (one per layer) on the same workspace."""
    batch, pl, nl = _lens(prefix_lens, new_lens)
    ws_bytes = _nbytes(workspace)
    plan = McAttnPlan()
    st = int(lib().mc_prefill_attn_prepare(ctypes.byref(params), pl.at, nl.at, batch, kv_splits, _dev_ptr(workspace), ws_bytes,
                                           _stream_handle(stream), ctypes.byref(plan)))
    if st != MC_OK:
        raise McError(st, "mc_prefill_attn_prepare")
    return plan


def mc_prefill_attn_run(params: McAttnParams, plan: McAttnPlan, q, k_pool, v_pool, block_tables, out, lse, workspace,
                        stream=None) -> None:
    _enqueue("mc_prefill_attn_run", _params(params), _plan(plan), q, k_pool, v_pool, block_tables,
             _max_pages(block_tables), out, lse, workspace, _on(stream))


def mc_prefill_attn_run_split(params: McAttnParams, plan: McAttnPlan, q, k_pool, v_pool, block_tables, o_parts,
                              lse_parts, workspace, stream=None) -> None:
    st = int(lib().mc_prefill_attn_run_split(ctypes.byref(params), ctypes.byref(plan), _dev_ptr(q), _dev_ptr(k_pool),
                                             _dev_ptr(v_pool), _dev_ptr(block_tables), _max_pages(block_tables),
                                             _dev_ptr(o_parts), _dev_ptr(lse_parts), _dev_ptr(workspace),
                                             _stream_handle(stream)))
    if st != MC_OK:
        raise McError(st, "mc_prefill_attn_run_split")


def mc_kv_append_run(params: McAttnParams, plan: McAttnPlan, k_new, v_new, k_pool, v_pool, block_tables, workspace,
                     stream=None) -> None:
    _enqueue("mc_kv_append_run", _params(params), _plan(plan), k_new, v_new, k_pool, v_pool, block_tables,
             _max_pages(block_tables), workspace, _on(stream))


def mc_prefill_attn_plan(params: McAttnParams, prefix_lens, new_lens, kv_splits: int = 0):
    """The work list of an attention launch, in launch order: a list of (request, kv_head, row0, slice) tuples.
    Host arithmetic only (no GPU)."""
    batch, pl, nl = _lens(prefix_lens, new_lens)
    n = ctypes.c_int64(-1)
    st = int(lib().mc_prefill_attn_plan(ctypes.byref(params), pl.at, nl.at, batch, kv_splits, None, 0, ctypes.byref(n)))
    if st != MC_OK:
        raise McError(st, "mc_prefill_attn_plan")
    buf = (ctypes.c_int32 * (4 * max(n.value, 1)))()
    st = int(lib().mc_prefill_attn_plan(ctypes.byref(params), pl.at, nl.at, batch, kv_splits, buf, n.value, ctypes.byref(n)))
    if st != MC_OK:
        raise McError(st, "mc_prefill_attn_plan")
    return [tuple(buf[4 * i:4 * i + 4]) for i in range(n.value)]


def mc_prefill_attn_suggest_kv_splits(params: McAttnParams, prefix_lens, new_lens) -> int:
    """Key slices that fill the GPU for this batch (1: use the whole-row call); 0 for arguments the library rejects."""
    batch, pl, nl = _lens(prefix_lens, new_lens)
    return int(lib().mc_prefill_attn_suggest_kv_splits(ctypes.byref(params), pl.at, nl.at, batch))


def mc_prefill_attn_paged_split_raw(params, q, k_pool, v_pool, block_tables, max_pages_per_req, prefix_lens, new_lens,
                                    batch, kv_splits, o_parts, lse_parts, workspace, workspace_bytes, hip_stream) -> int:
    return int(lib().mc_prefill_attn_paged_split(ctypes.byref(params) if params is not None else None, q, k_pool,
                                                 v_pool, block_tables, max_pages_per_req, prefix_lens, new_lens, batch,
                                                 kv_splits, o_parts, lse_parts, workspace, workspace_bytes, hip_stream))


def mc_prefill_attn_paged_split(params: McAttnParams, q, k_pool, v_pool, block_tables, prefix_lens, new_lens,
                                kv_splits: int, o_parts, lse_parts, workspace, stream=None) -> None:
    """Enqueue attention over ``kv_splits`` key slices; partial results go to the fp32 device tensors
    ``o_parts`` [kv_splits, total_new, Hq, D] and ``lse_parts`` [kv_splits, total_new, Hq]."""
    batch, pl, nl = _lens(prefix_lens, new_lens)
    max_pages = _max_pages(block_tables)
    ws_bytes = _nbytes(workspace)
    st = mc_prefill_attn_paged_split_raw(params, _dev_ptr(q), _dev_ptr(k_pool), _dev_ptr(v_pool),
                                         _dev_ptr(block_tables), max_pages, pl.at, nl.at, batch, kv_splits, _dev_ptr(o_parts),
                                         _dev_ptr(lse_parts), _dev_ptr(workspace), ws_bytes, _stream_handle(stream))
    if st != MC_OK:
        raise McError(st, "mc_prefill_attn_paged_split")


def mc_attn_merge_lse_raw(o_parts, lse_parts, kv_splits, rows, head_dim, dtype, out, lse, hip_stream) -> int:
    return int(lib().mc_attn_merge_lse(o_parts, lse_parts, kv_splits, rows, head_dim, dtype, out, lse, hip_stream))


def mc_attn_merge_lse(o_parts, lse_parts, kv_splits: int, rows: int, head_dim: int, dtype: int, out, lse=None,
                      stream=None) -> None:
    """Enqueue the merge of ``kv_splits`` partial results (fp32 device tensors) into ``out`` / ``lse``."""
    st = mc_attn_merge_lse_raw(_dev_ptr(o_parts), _dev_ptr(lse_parts), kv_splits, rows, head_dim, dtype,
                               _dev_ptr(out), _dev_ptr(lse), _stream_handle(stream))
    if st != MC_OK:
        raise McError(st, "mc_attn_merge_lse")


def mc_kv_pack_layer_raw(k_pool, v_pool, num_pages, page_bytes, page_ids, n, k_out, v_out, hip_stream) -> int:
    return int(lib().mc_kv_pack_layer(k_pool, v_pool, num_pages, page_bytes, page_ids, n, k_out, v_out, hip_stream))


def mc_kv_unpack_layer_raw(k_in, v_in, num_pages, page_bytes, page_ids, n, k_pool, v_pool, hip_stream) -> int:
    return int(lib().mc_kv_unpack_layer(k_in, v_in, num_pages, page_bytes, page_ids, n, k_pool, v_pool, hip_stream))


def mc_kv_pack_layer(k_pool_layer, v_pool_layer, num_pages: int, page_bytes: int, page_ids, n: int,
                     k_out, v_out, stream=None) -> None:
    _enqueue("mc_kv_pack_layer", k_pool_layer, v_pool_layer, num_pages, page_bytes, page_ids, n, k_out, v_out, _on(stream))


def mc_kv_unpack_layer(k_in, v_in, num_pages: int, page_bytes: int, page_ids, n: int,
                       k_pool_layer, v_pool_layer, stream=None) -> None:
    _enqueue("mc_kv_unpack_layer", k_in, v_in, num_pages, page_bytes, page_ids, n, k_pool_layer, v_pool_layer, _on(stream))


def mc_kv_page_order(page_ids, n: int, order, stream=None) -> None:
    """Enqueue order[r] = position of the r-th smallest page id (int32 device tensors)."""
    _enqueue("mc_kv_page_order", page_ids, n, order, _on(stream))


def mc_kv_check_page_ids(page_ids, n: int, num_pages: int, report, stream=None) -> None:
    """Enqueue the range check of an int32 device id list: report[0] = ids outside [0, num_pages), report[1] =
    position of the first of them (n if none); ``report`` is an int32 device tensor of 2."""
    st = int(lib().mc_kv_check_page_ids(_dev_ptr(page_ids), n, num_pages, _dev_ptr(report), _stream_handle(stream)))
    if st != MC_OK:
        raise McError(st, "mc_kv_check_page_ids")


def mc_kv_pack_layer_ordered(k_pool_layer, v_pool_layer, num_pages: int, page_bytes: int, page_ids, order, n: int,
                             k_out, v_out, stream=None) -> None:
    _enqueue("mc_kv_pack_layer_ordered", k_pool_layer, v_pool_layer, num_pages, page_bytes, page_ids, order, n, k_out, v_out,
             _on(stream))


def mc_kv_unpack_layer_ordered(k_in, v_in, num_pages: int, page_bytes: int, page_ids, order, n: int, k_pool_layer,
                               v_pool_layer, stream=None) -> None:
    _enqueue("mc_kv_unpack_layer_ordered", k_in, v_in, num_pages, page_bytes, page_ids, order, n, k_pool_layer, v_pool_layer,
             _on(stream))


def mc_kv_load_layer_raw(k_host, v_host, k_stage, v_stage, num_pages, page_bytes, page_ids, n, k_pool, v_pool,
                         hip_stream) -> int:
    return int(lib().mc_kv_load_layer(k_host, v_host, k_stage, v_stage, num_pages, page_bytes, page_ids, n, k_pool,
                                      v_pool, hip_stream))


def mc_kv_store_layer_raw(k_pool, v_pool, num_pages, page_bytes, page_ids, n, k_stage, v_stage, k_host, v_host,
                          hip_stream) -> int:
    return int(lib().mc_kv_store_layer(k_pool, v_pool, num_pages, page_bytes, page_ids, n, k_stage, v_stage, k_host,
                                       v_host, hip_stream))


def mc_kv_load_layer(k_host, v_host, k_stage, v_stage, num_pages: int, page_bytes: int, page_ids, n: int,
                     k_pool_layer, v_pool_layer, stream=None) -> None:
    """Host (pinned torch tensors) -> staging -> the listed pool pages, enqueued on ``stream``."""
    st = mc_kv_load_layer_raw(_dev_ptr(k_host), _dev_ptr(v_host), _dev_ptr(k_stage), _dev_ptr(v_stage), num_pages,
                              page_bytes, _dev_ptr(page_ids), n, _dev_ptr(k_pool_layer), _dev_ptr(v_pool_layer),
                              _stream_handle(stream))
    if st != MC_OK:
        raise McError(st, "mc_kv_load_layer")


def mc_kv_store_layer(k_pool_layer, v_pool_layer, num_pages: int, page_bytes: int, page_ids, n: int, k_stage,
                      v_stage, k_host, v_host, stream=None) -> None:
    """The listed pool pages -> staging -> host (pinned torch tensors), enqueued on ``stream``."""
    st = mc_kv_store_layer_raw(_dev_ptr(k_pool_layer), _dev_ptr(v_pool_layer), num_pages, page_bytes,
                               _dev_ptr(page_ids), n, _dev_ptr(k_stage), _dev_ptr(v_stage), _dev_ptr(k_host),
                               _dev_ptr(v_host), _stream_handle(stream))
    if st != MC_OK:
        raise McError(st, "mc_kv_store_layer")


def mc_prefix_hash_workspace_bytes(batch: int) -> int:
    return int(lib().mc_prefix_hash_workspace_bytes(batch))


def mc_prefix_match_workspace_bytes(batch: int, n_inst: int) -> int:
    return int(lib().mc_prefix_match_workspace_bytes(batch, n_inst))


def mc_prefix_hash_raw(tokens, tok_offsets, batch, block_tokens, keys, workspace, workspace_bytes, hip_stream) -> int:
    return int(lib().mc_prefix_hash(tokens, tok_offsets, batch, block_tokens, keys, workspace, workspace_bytes,
                                    hip_stream))


def mc_prefix_hash(tokens, tok_offsets, block_tokens: int, keys, workspace, stream=None) -> None:
    """Enqueue the block keys of every request: ``tokens`` int32 device tensor, ``tok_offsets`` host sequence of
    batch + 1 ints, ``keys`` int64 device tensor (the uint64 bit patterns) with one entry per block."""
    n = len(tok_offsets)
    _enqueue("mc_prefix_hash", tokens, _ints("q", tok_offsets, n), n - 1, block_tokens, keys, workspace,
             _nbytes(workspace), _on(stream))


def mc_prefix_match_raw(keys, key_offsets, batch, cache_keys, cache_offsets, n_inst, prefix_len, best_len, best_inst,
                        workspace, workspace_bytes, hip_stream) -> int:
    return int(lib().mc_prefix_match(keys, key_offsets, batch, cache_keys, cache_offsets, n_inst, prefix_len, best_len,
                                     best_inst, workspace, workspace_bytes, hip_stream))


def mc_prefix_match(keys, key_offsets, cache_keys, cache_offsets, prefix_len, best_len, best_inst, workspace,
                    stream=None) -> None:
    """Enqueue the longest-prefix match of every request against every instance (device tensors; offsets on the host)."""
    n, m = len(key_offsets), len(cache_offsets)
    _enqueue("mc_prefix_match", keys, _ints("q", key_offsets, n), n - 1, cache_keys,
             _ints("q", cache_offsets, m), m - 1, prefix_len, best_len, best_inst, workspace, _nbytes(workspace), _on(stream))


def mc_kv_append_workspace_bytes(batch: int) -> int:
    return int(lib().mc_kv_append_workspace_bytes(batch))


def mc_kv_append_paged_raw(params, k_new, v_new, k_pool, v_pool, block_tables, max_pages_per_req, prefix_lens,
                           new_lens, batch, workspace, workspace_bytes, hip_stream) -> int:
    return int(lib().mc_kv_append_paged(ctypes.byref(params) if params is not None else None, k_new, v_new, k_pool,
                                        v_pool, block_tables, max_pages_per_req, prefix_lens, new_lens, batch,
                                        workspace, workspace_bytes, hip_stream))


def mc_kv_append_paged(params: McAttnParams, k_new, v_new, k_pool, v_pool, block_tables, prefix_lens, new_lens,
                       workspace, stream=None) -> None:
    """Enqueue the scatter of the new tokens' K/V rows into their page slots (torch device tensors)."""
    n = len(prefix_lens)
    _enqueue("mc_kv_append_paged", _params(params), k_new, v_new, k_pool, v_pool, block_tables,
             _max_pages(block_tables), _ints("i", prefix_lens, n), _ints("i", new_lens, n), n, workspace,
             _nbytes(workspace), _on(stream))


def attn_params(num_q_heads: int, num_kv_heads: int, head_dim: int, page_size: int, num_pages: int,
                dtype: str, softmax_scale: float = 0.0) -> McAttnParams:
    return McAttnParams(num_q_heads, num_kv_heads, head_dim, page_size, num_pages,
                        MC_DTYPE_BF16 if dtype == "bf16" else MC_DTYPE_F32, softmax_scale)


def rope_params(rotary_dim: int, layout: int, base: float = 10000.0, scaling: int = MC_ROPE_PLAIN, factor: float = 1.0, low: float = 1.0,
                high: float = 4.0, original_len: float = 8192.0, gain: float = 1.0, norm_eps: float = 1e-6) -> McRopeParams:
    """The rotation of mc_kv_rope_append_*; frequencies by mc_rope_init (or set ``inv_freq`` afterwards)."""
    r = McRopeParams(0, layout, norm_eps, gain)
    st = int(lib().mc_rope_init(ctypes.byref(r), rotary_dim, base, scaling, factor, low, high, original_len))
    if st != MC_OK:
        raise McError(st, "mc_rope_init")
    return r


_torch = None
_DTYPES: dict = {}             # mc_dtype -> torch dtype


def _dtypes() -> dict:
    global _torch
    if _torch is None:
        import torch
        lib()
        _DTYPES.update({MC_DTYPE_BF16: torch.bfloat16, MC_DTYPE_F32: torch.float32})
        _torch = torch
    return _DTYPES


def _type(params):
    """torch's type of a call's tensors; parameters that have none are refused as the library does."""
    if _params(params) is None:
        raise McError(MC_ERR_NULL, "params")
    dtype = (_DTYPES or _dtypes()).get(params.dtype)
    if dtype is None:
        raise McError(MC_ERR_UNSUPPORTED, f"dtype {params.dtype}")
    return dtype


def _misfit_by_python(device: int, dtype, *tensors) -> int:
    """What csrc/pycall.cpp does, for an interpreter it was not built for."""
    for i, (t, least) in enumerate(zip(tensors[::2], tensors[1::2])):
        if t.dtype is not dtype or t.get_device() != device or not t.is_contiguous() or t.numel() < least:
            return i
    return -1


def _row_stride_by_python(device: int, dtype, t, tokens: int, heads: int, dim: int) -> int:
    shape, stride = tuple(t.shape), t.stride()
    fits = (len(shape) == 2 and shape[1] == heads * dim and stride[1] == 1) or (
        len(shape) == 3 and shape[1] == heads and shape[2] == dim and stride[2] == 1 and (stride[1] == dim or heads == 1))
    if not fits or shape[0] != tokens or t.dtype is not dtype or t.get_device() != device:
        return -1
    return stride[0] if tokens > 1 else heads * dim


_misfit, _row_stride = _misfit_by_python, _row_stride_by_python


def _is(t) -> str:
    return f"{t.dtype} {tuple(t.shape)} strides {t.stride()} on {t.device}"


def _dense(names: str, device: int, dtype, *tensors) -> None:
    """Tensors of a call, each followed by the number of elements the call will use: dense, of this type, on this device."""
    bad = _misfit(device, dtype, *tensors)
    if bad >= 0:
        raise ValueError(f"{names.split()[bad]}: dense {dtype} of at least {tensors[2 * bad + 1]} elements on device {device} wanted, "
                         f"not {_is(tensors[2 * bad])}")


def _here(device: int, workspace) -> None:
    """The tensors' device has to be a GPU and the current one (streams and launches are its own), and the workspace has to lie there."""
    if device < 0:                                         # (before torch has been asked for a GPU, there is no current one to compare with)
        raise ValueError("tensors in host memory, but tensors on the GPU wanted")
    current = _device() if _device is not None else _torch.cuda.current_device() if _torch.cuda.is_initialized() else device
    if device != current:
        raise ValueError(f"tensors on device {device}, but the current device is {current}")
    if workspace is not None and (workspace.get_device() != device or not workspace.is_contiguous()):
        raise ValueError(f"workspace: a dense tensor on device {device} wanted, not {_is(workspace)}")


def _pool_size(params) -> int:
    return params.num_pages * params.num_kv_heads * params.page_size * params.head_dim


def _table(block_tables, rows: int) -> int:
    """Columns of a block table that has ``rows`` rows."""
    shape = block_tables.shape
    if len(shape) != 2 or shape[0] < rows:
        raise ValueError(f"block_tables: [{rows}, pages] wanted, not {tuple(shape)}")
    return shape[1]


def _rope_tensors(params, q, k, v, q_norm, k_norm, q_out, k_pool, v_pool, tokens: int):
    """Looks the tensors of a rotation call over: (device, strides or None where all of them are dense)."""
    dtype = _type(params)
    device, Hq, Hkv, D = q.get_device(), params.num_q_heads, params.num_kv_heads, params.head_dim
    a, b, c = (_row_stride(device, dtype, q, tokens, Hq, D), _row_stride(device, dtype, k, tokens, Hkv, D),
               _row_stride(device, dtype, v, tokens, Hkv, D))
    if a < 0 or b < 0 or c < 0:
        name, t, heads = ("q", q, Hq) if a < 0 else ("k", k, Hkv) if b < 0 else ("v", v, Hkv)
        raise ValueError(f"{name}: {dtype} [{tokens}, {heads}, {D}] with dense heads on device {device} wanted, not {_is(t)}")
    size = _pool_size(params)
    if q_norm is not None and k_norm is not None:
        _dense("q_out k_pool v_pool q_norm k_norm", device, dtype, q_out, tokens * Hq * D, k_pool, size, v_pool, size, q_norm, D, k_norm, D)
    else:
        _dense("q_out k_pool v_pool", device, dtype, q_out, tokens * Hq * D, k_pool, size, v_pool, size)
        for name, t in (("q_norm", q_norm), ("k_norm", k_norm)):
            if t is not None:
                _dense(name, device, dtype, t, D)
    return device, None if a == Hq * D and b == c == Hkv * D else (ctypes.c_int64 * 3)(a, b, c)


def _rope(rope):
    if not isinstance(rope, McRopeParams):
        raise TypeError(f"McRopeParams wanted, not {type(rope).__name__}")
    return rope


def mc_kv_rope_append_paged(params: McAttnParams, rope: McRopeParams, q, k, v, q_norm, k_norm, q_out, k_pool, v_pool, block_tables,
                            prefix_lens, new_lens, workspace, stream=None) -> None:
    """Enqueue head norms (``q_norm`` / ``k_norm``: weights or None), rotation and append of the new tokens' rows.

    q, k, v: [tokens, heads, head_dim] or [tokens, heads * head_dim], dense or columns of a wider projection; q_out: dense."""
    n = len(prefix_lens)
    if len(new_lens) != n:
        raise ValueError(f"{n} prefix lengths and {len(new_lens)} new lengths")
    device, strides = _rope_tensors(params, q, k, v, q_norm, k_norm, q_out, k_pool, v_pool, sum(new_lens))
    wide = _table(block_tables, n)
    _dense("block_tables", device, _torch.int32, block_tables, 0)
    _here(device, workspace)
    _enqueue("mc_kv_rope_append_paged", params, _rope(rope), q, k, v, strides, q_norm, k_norm, q_out, k_pool, v_pool, block_tables, wide,
             _ints("i", prefix_lens, n), _ints("i", new_lens, n), n, workspace, _nbytes(workspace),
             _on(stream))


def mc_kv_rope_append_run(params: McAttnParams, plan: McAttnPlan, rope: McRopeParams, q, k, v, q_norm, k_norm, q_out, k_pool, v_pool,
                          block_tables, workspace, stream=None) -> None:
    """mc_kv_rope_append_paged for a prepared batch."""
    device, strides = _rope_tensors(params, q, k, v, q_norm, k_norm, q_out, k_pool, v_pool, _plan(plan).total_new_tokens)
    wide = _table(block_tables, plan.batch)
    _dense("block_tables", device, _torch.int32, block_tables, 0)
    _here(device, workspace)
    _enqueue("mc_kv_rope_append_run", params, plan, _rope(rope), q, k, v, strides, q_norm, k_norm, q_out, k_pool, v_pool, block_tables, wide,
             workspace, _on(stream))


def mc_kv_rope_append_decode(params: McAttnParams, rope: McRopeParams, q, k, v, q_norm, k_norm, q_out, k_pool, v_pool, block_tables,
                             seq_lens, stream=None) -> None:
    """The same for one new token a row, at position ``seq_lens[r] - 1``; ``seq_lens``: int32 device tensor."""
    n = seq_lens.numel()
    device, strides = _rope_tensors(params, q, k, v, q_norm, k_norm, q_out, k_pool, v_pool, n)
    wide = _table(block_tables, n)
    _dense("seq_lens block_tables", device, _torch.int32, seq_lens, n, block_tables, 0)
    _here(device, None)
    _enqueue("mc_kv_rope_append_decode", params, _rope(rope), q, k, v, strides, q_norm, k_norm, q_out, k_pool, v_pool, block_tables, wide,
             seq_lens, n, _on(stream))


def mc_decode_attn_workspace_bytes(params: McAttnParams, batch: int) -> int:
    return int(lib().mc_decode_attn_workspace_bytes(ctypes.byref(params), batch))


def mc_decode_attn_paged(params: McAttnParams, q, k_pool, v_pool, block_tables, seq_lens, out, lse, workspace, stream=None) -> None:
    """Enqueue attention of one new token a row: q, out [rows, heads, head_dim], ``seq_lens`` int32 device tensor [rows]."""
    dtype = _type(params)
    n, heads = seq_lens.numel(), params.num_q_heads
    wide = _table(block_tables, n)
    device, size, pool = q.get_device(), n * heads * params.head_dim, _pool_size(params)
    _dense("q k_pool v_pool out", device, dtype, q, size, k_pool, pool, v_pool, pool, out, size)
    _dense("seq_lens block_tables", device, _torch.int32, seq_lens, n, block_tables, 0)
    if lse is not None:
        _dense("lse", device, _torch.float32, lse, n * heads)
    _here(device, workspace)
    _enqueue("mc_decode_attn_paged", params, q, k_pool, v_pool, block_tables, wide, seq_lens, n, out, lse, workspace, _nbytes(workspace),
             _on(stream))


def mc_kv_pages_workspace_bytes(num_pages: int, rows: int) -> int:
    return int(lib().mc_kv_pages_workspace_bytes(num_pages, rows))


def _state(ref_counts, block_tables, page_size: int, seq_lens, workspace, names: str, *more):
    """Looks a cache's bookkeeping over, and the int32 tensors that follow with what is used of each: the seven arguments that
    stand for it."""
    if _torch is None:
        _dtypes()
    rows, device = seq_lens.numel(), ref_counts.get_device()
    wide = _table(block_tables, rows)
    _dense("ref_counts block_tables seq_lens " + names, device, _torch.int32, ref_counts, 0, block_tables, 0, seq_lens, rows, *more)
    _here(device, workspace)
    return ref_counts, ref_counts.numel(), block_tables, wide, page_size, seq_lens, rows


def mc_kv_pages_fork(ref_counts, block_tables, page_size: int, seq_lens, src_rows, dst_rows, moves, report, workspace, stream=None) -> None:
    """Enqueue rows ``dst_rows`` becoming copies of ``src_rows``; all int32 device tensors, ``moves`` [n, 2], ``report`` [4]."""
    n = src_rows.numel()
    state = _state(ref_counts, block_tables, page_size, seq_lens, workspace, "src_rows dst_rows moves report", src_rows, n, dst_rows, n, moves, 2 * n, report, 4)
    _enqueue("mc_kv_pages_fork", *state, src_rows, dst_rows, n, moves, report, workspace, _nbytes(workspace), _on(stream))


def mc_kv_pages_grow(ref_counts, block_tables, page_size: int, seq_lens, add, report, workspace, stream=None) -> None:
    """Enqueue row r getting ``add[r]`` more tokens, and the pages that takes."""
    state = _state(ref_counts, block_tables, page_size, seq_lens, workspace, "add report", add, seq_lens.numel(), report, 4)
    _enqueue("mc_kv_pages_grow", *state, add, report, workspace, _nbytes(workspace), _on(stream))


def mc_kv_pages_free(ref_counts, block_tables, page_size: int, seq_lens, free_rows, report, stream=None) -> None:
    """Enqueue the listed rows becoming empty."""
    n = free_rows.numel()
    state = _state(ref_counts, block_tables, page_size, seq_lens, None, "free_rows report", free_rows, n, report, 4)
    _enqueue("mc_kv_pages_free", *state, free_rows, n, report, _on(stream))


def mc_kv_pages_compact(ref_counts, moves, report, workspace, stream=None) -> None:
    """Enqueue the list of at most ``moves.shape[0]`` moves that bring live pages to the front of the pool."""
    if _torch is None:
        _dtypes()
    n = moves.shape[0]
    device = ref_counts.get_device()
    _dense("ref_counts moves report", device, _torch.int32, ref_counts, 0, moves, 2 * n, report, 4)
    _here(device, workspace)
    _enqueue("mc_kv_pages_compact", ref_counts, ref_counts.numel(), n, moves, report, workspace, _nbytes(workspace), _on(stream))


def mc_kv_pages_remap(ref_counts, block_tables, page_size: int, seq_lens, moves, count=None, stream=None) -> None:
    """Enqueue tables and counts following ``moves`` [n, 2], of which ``count[0]`` are looked at (None: all; unused ones of -1 are passed over)."""
    n = moves.shape[0]
    if count is None:
        state = _state(ref_counts, block_tables, page_size, seq_lens, None, "moves", moves, 2 * n)
    else:
        state = _state(ref_counts, block_tables, page_size, seq_lens, None, "moves count", moves, 2 * n, count, 1)
    _enqueue("mc_kv_pages_remap", *state, moves, count, n, _on(stream))


def mc_kv_copy_pages(k_pools, v_pools, num_pages: int, page_bytes: int, moves, count=None, stream=None) -> None:
    """Enqueue the copy of the moved pages in every layer: lists of device tensors of num_pages * page_bytes bytes."""
    _dtypes()
    if len(k_pools) != len(v_pools):
        raise ValueError(f"{len(k_pools)} K pools and {len(v_pools)} V pools")
    device, n = moves.get_device(), moves.shape[0]
    _dense("moves", device, _torch.int32, moves, 2 * n)
    if count is not None:
        _dense("count", device, _torch.int32, count, 1)
    for pool in (*k_pools, *v_pools):
        if pool.get_device() != device or not pool.is_contiguous() or pool.nbytes < num_pages * page_bytes:
            raise ValueError(f"pools: {num_pages * page_bytes} dense bytes on device {device} wanted, not {_is(pool)}")
    _here(device, None)
    layers = len(k_pools)
    _enqueue("mc_kv_copy_pages", _ints("q", [t.data_ptr() for t in k_pools], layers), _ints("q", [t.data_ptr() for t in v_pools], layers),
             layers, num_pages, page_bytes, moves, count, n, _on(stream))
