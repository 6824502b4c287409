"""Decode attention on the host: how the line of blocks is shared out, and what the call refuses."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2407_00079_amd import binding as B
from test_rope_host import FAKE, host

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_place_of_the_line_has_its_wave(tmp_path):
    """decode_begin and decode_wave_of for all small lines and for the largest that fit."""
    src = tmp_path / "line.cpp"
    src.write_text(r'''
#include <cstdio>
#include <cstdint>
#include <initializer_list>
#include "mc_types.h"
using namespace mc;
int main() {
  for (int64_t total = 1; total < 700; ++total)
    for (int all : {1, 8, 64, 512}) {
      const int n = decode_waves(total, all);
      if (decode_begin(total, 0, n) != 0 || decode_begin(total, n, n) != total) return 1;
      for (int w = 0; w < n; ++w) {
        const int64_t lo = decode_begin(total, w, n), hi = decode_begin(total, w + 1, n);
        if (hi <= lo || hi - lo > (total + n - 1) / n) return 2;           // each has work, none more than its share
        for (int64_t x = lo; x < hi; ++x)
          if (decode_wave_of(total, x, n) != w) return 3;
      }
    }
  const int64_t most = (int64_t)1 << 51;                                   // what the front end lets through
  for (int w = 0; w < 2048; ++w) {
    const int64_t lo = decode_begin(most - 77, w, 2048), hi = decode_begin(most - 77, w + 1, 2048);
    if (lo < 0 || hi <= lo || decode_wave_of(most - 77, lo, 2048) != w || decode_wave_of(most - 77, hi - 1, 2048) != w) return 4;
  }
  return 0;
}
''')
    exe = tmp_path / "line"
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2407_00079_amd", "csrc"), "-o", str(exe), str(src)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0


def call(p=None, q=FAKE, k=FAKE, v=FAKE, bt=FAKE, max_pages=64, lens=FAKE, batch=3, out=FAKE, lse=None, ws=FAKE, ws_bytes=1 << 30):
    p = p or B.attn_params(8, 2, 128, 16, 64, "bf16")
    return B.lib().mc_decode_attn_paged(ctypes.byref(p), q, k, v, bt, max_pages, lens, batch, out, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), B.MC_ERR_NULL), (dict(k=None), B.MC_ERR_NULL), (dict(v=None), B.MC_ERR_NULL), (dict(bt=None), B.MC_ERR_NULL),
    (dict(lens=None), B.MC_ERR_NULL), (dict(out=None), B.MC_ERR_NULL), (dict(batch=-1), B.MC_ERR_SHAPE), (dict(max_pages=-1), B.MC_ERR_SHAPE),
    (dict(q=FAKE + 8), B.MC_ERR_ALIGN), (dict(out=FAKE + 8), B.MC_ERR_ALIGN), (dict(ws=FAKE + 8), B.MC_ERR_ALIGN),
    (dict(lens=FAKE + 2), B.MC_ERR_ALIGN), (dict(lse=FAKE + 2), B.MC_ERR_ALIGN), (dict(ws=None), B.MC_ERR_WORKSPACE),
    (dict(ws_bytes=1000), B.MC_ERR_WORKSPACE), (dict(batch=2 ** 26, max_pages=1), B.MC_ERR_RANGE),
    (dict(batch=2 ** 16, max_pages=2 ** 16), B.MC_ERR_RANGE),
    (dict(p=B.attn_params(2 ** 25, 1, 128, 16, 64, "bf16"), batch=1, max_pages=2 ** 28), B.MC_ERR_RANGE),
    (dict(p=B.attn_params(8, 2, 128, 32, 64, "bf16")), B.MC_ERR_UNSUPPORTED),
    (dict(p=B.attn_params(8, 2, 128, 16, 64, "f32")), B.MC_ERR_UNSUPPORTED), (dict(p=B.attn_params(8, 3, 128, 16, 64, "bf16")), B.MC_ERR_SHAPE),
    (dict(p=B.attn_params(8, 2, 128, 16, 64, "bf16", -1.0)), B.MC_ERR_SHAPE), (dict(batch=0, q=None, lens=None, ws=None), B.MC_OK)])
def test_refusals(change, status):
    assert call(**change) == status


def test_workspace():
    p = B.attn_params(8, 2, 128, 16, 64, "bf16")
    need = B.mc_decode_attn_workspace_bytes(p, 1)
    assert 0 < need < 1 << 23 and need == B.mc_decode_attn_workspace_bytes(p, 5000)
    assert call(ws_bytes=need - 1) == B.MC_ERR_WORKSPACE
    assert B.mc_decode_attn_workspace_bytes(p, -1) == 0 and B.mc_decode_attn_workspace_bytes(B.attn_params(8, 3, 128, 16, 64, "bf16"), 1) == 0


GOOD = dict(q=(3, 8, 128), pool=(9, 2, 16, 128), table=(3, 4), lens=(3,), out=(3, 8, 128), lse=(3, 8))


@pytest.mark.parametrize("name,tensor", [
    ("q", host((3, 8, 64))), ("q", host((3, 8, 128), torch.float32)), ("q", host((3, 8, 128), strides=(2048, 128, 1))), ("q", host((2, 8, 128))),
    ("out", host((3, 8, 128), strides=(2048, 128, 1))), ("out", host((3, 8, 128), torch.float32)), ("pool", host((8, 2, 16, 128))),
    ("table", host((2, 4), torch.int32)), ("table", host((3, 4), torch.int64)), ("table", host((3, 4), torch.int32, (8, 1))),
    ("lens", host((3,), torch.int64)), ("lse", host((3, 7), torch.float32)), ("lse", host((3, 8))), ("out", torch.empty((3, 8, 128), dtype=torch.bfloat16))])
def test_the_binding_refuses_tensors_that_do_not_fit(name, tensor):
    kinds = dict(table=torch.int32, lens=torch.int32, lse=torch.float32)
    t = {n: host(s, kinds.get(n, torch.bfloat16)) for n, s in GOOD.items()}
    t[name] = tensor
    with pytest.raises(ValueError):
        B.mc_decode_attn_paged(B.attn_params(8, 2, 128, 16, 9, "bf16"), t["q"], t["pool"], t["pool"], t["table"], t["lens"], t["out"], t["lse"],
                               None, type("S", (), {"cuda_stream": 0})())


@pytest.mark.parametrize("what", ["device", "workspace", "lens"])
def test_other_devices_and_shapes_are_refused(what, monkeypatch):
    kinds = dict(table=torch.int32, lens=torch.int32, lse=torch.float32)
    t = {n: host(s, kinds.get(n, torch.bfloat16)) for n, s in GOOD.items()}
    ws = host((1 << 24,), torch.uint8)
    if what == "device":                                      # the tensors lie on device 0
        monkeypatch.setattr(B, "_device", lambda: 1)
    elif what == "workspace":
        ws = torch.empty(1 << 24, dtype=torch.uint8)
    else:
        t["lens"] = host((3, 2), torch.int32)
    with pytest.raises(ValueError):
        B.mc_decode_attn_paged(B.attn_params(8, 2, 128, 16, 9, "bf16"), t["q"], t["pool"], t["pool"], t["table"], t["lens"], t["out"], t["lse"],
                               ws, type("S", (), {"cuda_stream": 0})())


def test_by_python_as_by_the_native_caller():
    """The two looks at tensors agree, for an interpreter that the caller was not built for."""
    from paper_2407_00079_amd import _mccall
    bf16, good = torch.bfloat16, host((4, 8, 64))
    for t in (good, host((4, 8, 64), torch.float32), torch.empty((4, 8, 64), dtype=bf16), host((4, 8, 64), strides=(1024, 64, 1)), host((4, 512)),
              host((4, 512), strides=(700, 1)), host((4, 8, 64), strides=(1024, 128, 1)), host((3, 8, 64)), host((4, 4, 128)), host((2048,)),
              host((1, 8, 64), strides=(3, 64, 1)), host((4, 1, 512), strides=(600, 7, 1)), host((0, 8, 64)), host((1, 4, 8, 64))):
        for least in (0, 2048, 2049):
            assert _mccall.misfit(0, bf16, good, 2048, t, least) == B._misfit_by_python(0, bf16, good, 2048, t, least)
        for tokens, heads, dim in ((4, 8, 64), (1, 8, 64), (4, 1, 512), (0, 8, 64)):
            assert _mccall.row_stride(0, bf16, t, tokens, heads, dim) == B._row_stride_by_python(0, bf16, t, tokens, heads, dim)
    for bad in ((0, bf16, good), (0, bf16, None, 1), ("x", bf16, good, 1)):
        with pytest.raises((TypeError, AttributeError)):
            _mccall.misfit(*bad)
    with pytest.raises(TypeError):
        _mccall.row_stride(0, bf16, good, 4, 8)


def test_parameters_without_a_type():
    """Refused with the library's statuses by the wrappers, too, which look at the tensors first."""
    x, ids = torch.zeros((1, 8, 128), dtype=torch.bfloat16), torch.zeros((1, 1), dtype=torch.int32)
    p = B.attn_params(8, 8, 128, 16, 1, "bf16")
    p.dtype = 5
    for params, status in ((p, B.MC_ERR_UNSUPPORTED), (None, B.MC_ERR_NULL)):
        with pytest.raises(B.McError) as e:
            B.mc_decode_attn_paged(params, x, x, x, ids, ids[0], x, None, None)
        assert e.value.status == status
        with pytest.raises(B.McError) as e:
            B.mc_kv_rope_append_decode(params, B.rope_params(128, B.MC_ROPE_HALF), x, x, x, None, None, x, x, x, ids, ids[0])
        assert e.value.status == status
