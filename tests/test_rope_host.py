"""Rotation on the host: frequencies, what the calls refuse, and how the binding looks tensors over.  Nothing is launched."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2407_00079_amd import binding as B
from test_binding_calls import declarations

FAKE = 0x7F0000001000      # never dereferenced


def test_frequencies():
    plain = 500000.0 ** (-2 * np.arange(48) / 96)
    r = B.rope_params(96, B.MC_ROPE_HALF, base=500000.0)
    assert r.rotary_dim == 96 and np.allclose(list(r.inv_freq)[:48], plain, rtol=1e-14) and not any(list(r.inv_freq)[48:])
    r = B.rope_params(96, B.MC_ROPE_HALF, base=500000.0, scaling=B.MC_ROPE_LINEAR, factor=8.0)
    assert np.allclose(list(r.inv_freq)[:48], plain / 8, rtol=1e-14)
    r = B.rope_params(96, B.MC_ROPE_HALF, base=500000.0, scaling=B.MC_ROPE_BASE, factor=8.0)
    got = list(r.inv_freq)[:48]
    # the fastest pair turns as before, the slowest as it does over a context 8 times as long
    assert got[0] == 1.0 and math.isclose(got[47], plain[47] / 8, rel_tol=1e-12)
    r = B.rope_params(96, B.MC_ROPE_HALF, base=500000.0, scaling=B.MC_ROPE_BY_PARTS, factor=8.0, low=1.0, high=4.0, original_len=8192.0)
    turns = 8192 * plain / (2 * math.pi)
    share = np.clip((turns - 1) / 3, 0, 1)
    assert np.allclose(list(r.inv_freq)[:48], plain * (share + (1 - share) / 8), rtol=1e-13) and 0 < sum(share) < 48
    assert B.rope_params(0, B.MC_ROPE_PAIRS, scaling=B.MC_ROPE_BASE, factor=2.0).rotary_dim == 0


@pytest.mark.parametrize("args,status", [
    ((24, 1e4, 0, 1, 1, 4, 8192), B.MC_ERR_UNSUPPORTED), ((-16, 1e4, 0, 1, 1, 4, 8192), B.MC_ERR_UNSUPPORTED),
    ((144, 1e4, 0, 1, 1, 4, 8192), B.MC_ERR_UNSUPPORTED), ((64, 1e4, 4, 1, 1, 4, 8192), B.MC_ERR_UNSUPPORTED),
    ((64, 1e4, -1, 1, 1, 4, 8192), B.MC_ERR_UNSUPPORTED), ((64, 0.0, 0, 1, 1, 4, 8192), B.MC_ERR_SHAPE),
    ((64, math.nan, 0, 1, 1, 4, 8192), B.MC_ERR_SHAPE), ((64, 1e4, 1, 0.0, 1, 4, 8192), B.MC_ERR_SHAPE),
    ((64, 1e4, 1, math.inf, 1, 4, 8192), B.MC_ERR_SHAPE), ((64, 1e4, 3, 2.0, 4, 4, 8192), B.MC_ERR_SHAPE),
    ((64, 1e4, 3, 2.0, 1, math.nan, 8192), B.MC_ERR_SHAPE), ((64, 1e4, 3, 2.0, 1, 4, 0.0), B.MC_ERR_SHAPE),
    ((64, 1e4, 3, 2.0, -1, 4, 8192), B.MC_ERR_SHAPE), ((64, 1e4, 0, 1, 9, 4, 0), B.MC_OK)])
def test_frequencies_refused(args, status):
    r = B.McRopeParams()
    assert B.lib().mc_rope_init(ctypes.byref(r), *args) == status
    assert B.lib().mc_rope_init(None, *args) == B.MC_ERR_NULL


def call(form, *, p=None, rope=None, q=FAKE, k=FAKE, v=FAKE, strides=None, qn=FAKE, kn=FAKE, out=FAKE + 4096, kp=FAKE, vp=FAKE, bt=FAKE,
         max_pages=64, prefix=(100,), new=(5,), lens=FAKE, batch=None, ws=FAKE, ws_bytes=1 << 20):
    p = p or B.attn_params(8, 2, 128, 16, 64, "bf16")
    rope = B.rope_params(64, B.MC_ROPE_HALF) if rope is None else rope
    rope = ctypes.byref(rope) if rope else None
    strides = None if strides is None else (ctypes.c_int64 * 3)(*strides)
    n = len(prefix) if batch is None else batch
    a = (q, k, v, strides, qn, kn, out, kp, vp, bt, max_pages)
    if form == "paged":
        i32 = ctypes.c_int32 * max(1, len(prefix))
        lists = (None, None) if prefix is None else (i32(*prefix), i32(*new))
        return B.lib().mc_kv_rope_append_paged(ctypes.byref(p), rope, *a, *lists, n, ws, ws_bytes, None)
    if form == "run":
        plan = B.McAttnPlan(2, n, 0, 7, sum(new), 64, p.num_q_heads, p.num_kv_heads, p.dtype, 0)
        return B.lib().mc_kv_rope_append_run(ctypes.byref(p), ctypes.byref(plan), rope, *a, ws, None)
    return B.lib().mc_kv_rope_append_decode(ctypes.byref(p), rope, *a, lens, n, None)


def broken(**fields):
    r = B.rope_params(64, B.MC_ROPE_HALF)
    for name, value in fields.items():
        if name == "freq":
            r.inv_freq[31] = value
        else:
            setattr(r, name, value)
    return r


@pytest.mark.parametrize("form", ["paged", "run", "decode"])
@pytest.mark.parametrize("change,status", [
    (dict(rope=False), B.MC_ERR_NULL), (dict(rope=broken(rotary_dim=40)), B.MC_ERR_UNSUPPORTED),
    (dict(rope=broken(rotary_dim=144)), B.MC_ERR_UNSUPPORTED), (dict(rope=broken(rotary_dim=-16)), B.MC_ERR_UNSUPPORTED),
    (dict(rope=broken(layout=2)), B.MC_ERR_UNSUPPORTED), (dict(rope=broken(norm_eps=-1.0)), B.MC_ERR_SHAPE),
    (dict(rope=broken(norm_eps=math.nan)), B.MC_ERR_SHAPE), (dict(rope=broken(gain=0.0)), B.MC_ERR_SHAPE),
    (dict(rope=broken(gain=math.inf)), B.MC_ERR_SHAPE), (dict(rope=broken(freq=math.nan)), B.MC_ERR_SHAPE),
    (dict(rope=broken(rotary_dim=128), p=B.attn_params(8, 2, 64, 16, 64, "bf16")), B.MC_ERR_UNSUPPORTED),
    (dict(p=B.attn_params(8, 3, 128, 16, 64, "bf16")), B.MC_ERR_SHAPE), (dict(p=B.attn_params(8, 2, 96, 16, 64, "bf16")), B.MC_ERR_UNSUPPORTED),
    (dict(p=B.attn_params(8, 2, 128, 32, 64, "bf16")), B.MC_ERR_UNSUPPORTED),
    (dict(strides=(1016, 256, 256)), B.MC_ERR_SHAPE), (dict(strides=(1024, 255, 256)), B.MC_ERR_SHAPE),
    (dict(strides=(1024, 256, 260)), B.MC_ERR_ALIGN), (dict(strides=(1024, 256, 2 ** 62)), B.MC_ERR_SHAPE),
    (dict(strides=(1032, 256, 256), out=FAKE), B.MC_ERR_SHAPE),
    (dict(q=None), B.MC_ERR_NULL), (dict(k=None), B.MC_ERR_NULL), (dict(v=None), B.MC_ERR_NULL), (dict(out=None), B.MC_ERR_NULL),
    (dict(kp=None), B.MC_ERR_NULL), (dict(vp=None), B.MC_ERR_NULL), (dict(bt=None), B.MC_ERR_NULL),
    (dict(q=FAKE + 8), B.MC_ERR_ALIGN), (dict(kn=FAKE + 2), B.MC_ERR_ALIGN), (dict(bt=FAKE + 2), B.MC_ERR_ALIGN),
    (dict(max_pages=-1), B.MC_ERR_SHAPE)])
def test_refusals(form, change, status):
    assert call(form, **change) == status


def test_refusals_of_one_form():
    assert call("paged", ws=None) == B.MC_ERR_WORKSPACE and call("paged", ws_bytes=8) == B.MC_ERR_WORKSPACE
    assert call("paged", ws=FAKE + 4) == B.MC_ERR_ALIGN and call("run", ws=None) == B.MC_ERR_WORKSPACE
    assert call("paged", prefix=(-1,)) == B.MC_ERR_SHAPE and call("paged", new=(-1,)) == B.MC_ERR_SHAPE
    assert call("paged", max_pages=6) == B.MC_ERR_SHAPE and call("run", max_pages=6) == B.MC_ERR_SHAPE
    assert call("paged", prefix=(2 ** 31 - 8,), new=(16,), max_pages=2 ** 27) == B.MC_ERR_RANGE
    assert call("paged", batch=-1) == B.MC_ERR_SHAPE and call("decode", batch=-1) == B.MC_ERR_SHAPE
    assert call("decode", lens=None) == B.MC_ERR_NULL and call("decode", lens=FAKE + 1) == B.MC_ERR_ALIGN
    assert call("decode", batch=2 ** 20, max_pages=2 ** 20) == B.MC_ERR_RANGE
    assert call("decode", batch=0, q=None, lens=None) == B.MC_OK and call("paged", new=(0,), q=None, ws=None) == B.MC_OK
    p = B.attn_params(2 ** 30, 2 ** 30, 64, 16, 64, "bf16")
    assert call("decode", p=p) == B.MC_ERR_RANGE


def test_the_kinds_of_the_cache_calls():
    host, declared = {"prefix_lens", "new_lens"}, declarations()
    for function, kinds in B._CACHE_KINDS.items():
        want = ""
        for type_, name in declared[function]:
            if name in host:
                want += "I"
            elif name in ("k_pools", "v_pools"):
                want += "Q"
            elif type_.startswith(("const mc_attn_", "const mc_rope_")) or name == "strides":
                want += "s"
            else:
                want += "p" if type_.endswith("*") and name != "hip_stream" else "i"
        assert kinds == want and len(getattr(B.lib(), function).argtypes) == len(want), function


class Host(torch.Tensor):
    """A CPU tensor that says it lies on device 0."""

    def get_device(self):
        return 0


def host(shape, dtype=torch.bfloat16, strides=None):
    x = torch.empty(shape, dtype=dtype) if strides is None else torch.empty(1 << 18, dtype=dtype).as_strided(shape, strides)
    return x.as_subclass(Host)


GOOD = dict(q=(3, 8, 128), k=(3, 2, 128), v=(3, 2, 128), out=(3, 8, 128), pool=(9, 2, 16, 128), table=(3, 4), lens=(3,))


@pytest.mark.parametrize("name,tensor", [
    ("q", host((3, 8, 64))), ("q", host((2, 8, 128))), ("q", host((3, 1000))), ("q", host((3, 8, 128), torch.float32)),
    ("q", host((3, 8, 128), strides=(2048, 256, 1))), ("k", host((3, 2, 128), strides=(256, 128, 2))), ("v", torch.empty((3, 2, 128), dtype=torch.bfloat16)),
    ("out", host((3, 8, 128), strides=(2048, 128, 1))), ("out", host((2, 8, 128))), ("pool", host((8, 2, 16, 128))),
    ("pool", host((9, 2, 16, 128), torch.float16)), ("table", host((2, 4), torch.int32)), ("table", host((3, 4), torch.int64)),
    ("table", host((12,), torch.int32)), ("lens", host((3,), torch.int64)), ("lens", host((4,), torch.int32)), ("norm", host((64,)))])
def test_the_binding_refuses_tensors_that_do_not_fit(name, tensor):
    made = {n: host(s, torch.int32 if n in ("table", "lens") else torch.bfloat16) for n, s in GOOD.items()}
    made["norm"] = host((128,))
    made[name] = tensor
    p, rope = B.attn_params(8, 2, 128, 16, 9, "bf16"), B.rope_params(128, B.MC_ROPE_HALF)
    stream = type("S", (), {"cuda_stream": 0})()
    with pytest.raises(ValueError):
        B.mc_kv_rope_append_decode(p, rope, made["q"], made["k"], made["v"], made["norm"], None, made["out"], made["pool"], made["pool"],
                                   made["table"], made["lens"], stream)


def test_the_binding_refuses_other_things():
    p, stream = B.attn_params(8, 2, 128, 16, 9, "bf16"), type("S", (), {"cuda_stream": 0})()
    t = {n: host(s, torch.int32 if n in ("table", "lens") else torch.bfloat16) for n, s in GOOD.items()}
    rest = (t["q"], t["k"], t["v"], None, None, t["out"], t["pool"], t["pool"], t["table"])
    with pytest.raises(TypeError):
        B.mc_kv_rope_append_decode(p, p, *rest, t["lens"], stream)
    with pytest.raises(ValueError):
        B.mc_kv_rope_append_paged(p, B.rope_params(128, B.MC_ROPE_HALF), *rest, [1, 2], [3], None, stream)
    with pytest.raises(ValueError):                           # a plan of other lengths
        B.mc_kv_rope_append_run(p, B.McAttnPlan(2, 1, 0, 7, 5, 64, 8, 2, 0, 0), B.rope_params(128, B.MC_ROPE_HALF), *rest, None, stream)
    with pytest.raises(B.McError):
        B.rope_params(20, B.MC_ROPE_HALF)
