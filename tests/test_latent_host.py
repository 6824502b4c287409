"""The cache of latent vectors on the host: what the calls refuse, workspaces, how work is cut, and how the binding looks tensors over.  Nothing
is launched."""
import ctypes
import math
import os
import random
import subprocess

import pytest
import torch

from paper_2407_00079_amd import binding as B
from test_binding_calls import declarations

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2407_00079_amd", "csrc")
FAKE = 0x7F0000001000      # never dereferenced
CALLS = ("append", "append_decode", "decode", "expand", "prefill")
BIG = 2 ** 31 - 1


def par(heads=8, latent=512, rope=64, head_dim=128, page=16, pages=64, dtype=B.MC_DTYPE_BF16, scale=0.0):
    return B.McLatentParams(heads, latent, rope, head_dim, page, dtype, pages, scale)


def call(form, *, p=None, rope=None, q=FAKE, kv=FAKE + 4096, strides=None, norm=FAKE, out=FAKE + 8192, pool=FAKE, bt=FAKE, max_pages=64, prefix=(100,),
         new=(5,), lens=FAKE, batch=None, tokens=1, k=FAKE, v=FAKE, weight=FAKE, lse=FAKE, ws=FAKE, ws_bytes=1 << 30):
    l, p = B.lib(), None if p is False else ctypes.byref(p or par())
    rope = B.rope_params(64, B.MC_ROPE_HALF) if rope is None else rope
    rope = ctypes.byref(rope) if rope else None
    n = len(new or (0,)) if batch is None else batch
    strides = None if strides is None else (ctypes.c_int64 * len(strides))(*strides)
    prefix, new = (None if x is None else (ctypes.c_int32 * max(1, len(x)))(*x) for x in (prefix, new))
    if form == "append":
        return l.mc_latent_append_paged(p, rope, q, kv, strides, norm, out, pool, bt, max_pages, prefix, new, n, ws, ws_bytes, None)
    if form == "append_decode":
        return l.mc_latent_append_decode(p, rope, q, kv, strides, norm, out, pool, bt, max_pages, lens, n, tokens, None)
    if form == "decode":
        return l.mc_latent_decode_attn_paged(p, q, pool, bt, max_pages, lens, n, tokens, out, lse, ws, ws_bytes, None)
    if form == "expand":
        return l.mc_latent_expand_paged(p, weight, pool, bt, max_pages, new, n, out, ws, ws_bytes, None)
    return l.mc_latent_prefill_attn_paged(p, q, k, v, strides, pool, bt, max_pages, prefix, new, n, out, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("form", CALLS)
@pytest.mark.parametrize("change,status", [
    (dict(p=False), B.MC_ERR_NULL), (dict(p=par(heads=0)), B.MC_ERR_SHAPE), (dict(p=par(heads=-8)), B.MC_ERR_SHAPE), (dict(p=par(pages=0)), B.MC_ERR_SHAPE),
    (dict(p=par(latent=0)), B.MC_ERR_SHAPE), (dict(p=par(latent=384)), B.MC_ERR_UNSUPPORTED), (dict(p=par(rope=32)), B.MC_ERR_UNSUPPORTED),
    (dict(p=par(head_dim=96)), B.MC_ERR_UNSUPPORTED), (dict(p=par(page=32)), B.MC_ERR_UNSUPPORTED), (dict(p=par(dtype=B.MC_DTYPE_F32)), B.MC_ERR_UNSUPPORTED),
    (dict(p=par(dtype=9)), B.MC_ERR_UNSUPPORTED), (dict(p=par(heads=1025)), B.MC_ERR_RANGE), (dict(p=par(scale=-1.0)), B.MC_ERR_SHAPE),
    (dict(p=par(scale=math.nan)), B.MC_ERR_SHAPE), (dict(p=par(scale=math.inf)), B.MC_ERR_SHAPE),
    (dict(pool=None), B.MC_ERR_NULL), (dict(bt=None), B.MC_ERR_NULL), (dict(out=None), B.MC_ERR_NULL), (dict(pool=FAKE + 8), B.MC_ERR_ALIGN),
    (dict(out=FAKE + 8), B.MC_ERR_ALIGN), (dict(bt=FAKE + 2), B.MC_ERR_ALIGN), (dict(max_pages=-1), B.MC_ERR_SHAPE), (dict(batch=-1), B.MC_ERR_SHAPE)])
def test_refusals(form, change, status):
    assert call(form, **change) == status


def broken(**fields):
    r = B.rope_params(64, B.MC_ROPE_HALF)
    for name, value in fields.items():
        if name == "freq":
            r.inv_freq[31] = value
        else:
            setattr(r, name, value)
    return r


@pytest.mark.parametrize("form", ["append", "append_decode"])
@pytest.mark.parametrize("change,status", [
    (dict(rope=False), B.MC_ERR_NULL), (dict(rope=broken(rotary_dim=48)), B.MC_ERR_UNSUPPORTED), (dict(rope=broken(layout=2)), B.MC_ERR_UNSUPPORTED),
    (dict(rope=broken(norm_eps=-1.0)), B.MC_ERR_SHAPE), (dict(rope=broken(gain=math.nan)), B.MC_ERR_SHAPE), (dict(rope=broken(freq=math.inf)), B.MC_ERR_SHAPE),
    (dict(q=None), B.MC_ERR_NULL), (dict(kv=None), B.MC_ERR_NULL), (dict(norm=FAKE + 8), B.MC_ERR_ALIGN), (dict(q=FAKE + 2), B.MC_ERR_ALIGN),
    (dict(kv=FAKE + 8), B.MC_ERR_ALIGN), (dict(strides=(512, 64, 576, 512, -8)), B.MC_ERR_SHAPE), (dict(strides=(512, 64, 576, 512, 68)), B.MC_ERR_ALIGN),
    (dict(strides=(2 ** 62, 64, 576, 512, 64)), B.MC_ERR_SHAPE), (dict(strides=(512, 64, 576, 512, 56), new=(2,), batch=2, prefix=(0, 0)), B.MC_ERR_SHAPE),
    (dict(q=FAKE, out=FAKE, strides=(512, 64, 576, 512, 128)), B.MC_ERR_SHAPE)])
def test_refusals_of_appends(form, change, status):
    if "batch" in change:
        change = dict(change, batch=None, new=(2, 2))
    assert call(form, **change) == status


def test_rows_that_would_overlap():
    """q_out from token to token and from head to head, in either order; overlaps are refused, whichever they are."""
    for out, status in (((512, 64), None), ((504, 64), B.MC_ERR_SHAPE), ((64, 5 * 64), None), ((64, 4 * 64), B.MC_ERR_SHAPE), ((0, 64), B.MC_ERR_SHAPE),
                        ((512, 0), B.MC_ERR_SHAPE), ((1024, 128), None)):
        # (the workspace's check comes behind)
        assert call("append", strides=(0, 0, 0, *out), ws=None) == (status or B.MC_ERR_WORKSPACE), out
    one = dict(strides=(0, 0, 0, 0, 0), ws=None, p=par(heads=1))
    assert call("append", new=(1,), **one) == B.MC_ERR_WORKSPACE and call("append", new=(2,), **one) == B.MC_ERR_SHAPE


def test_refusals_of_one_form():
    for form in ("append", "prefill"):
        assert call(form, prefix=None) == B.MC_ERR_NULL and call(form, new=None, batch=1) == B.MC_ERR_NULL
        assert call(form, prefix=(-1,)) == B.MC_ERR_SHAPE
        assert call(form, prefix=(BIG - 8,), new=(16,), max_pages=2 ** 27) == B.MC_ERR_RANGE
    for form in ("append", "expand", "prefill"):
        assert call(form, new=(-1,)) == B.MC_ERR_SHAPE and call(form, ws=FAKE + 8) == B.MC_ERR_ALIGN
        assert call(form, new=(64 * 16 + 1,)) == B.MC_ERR_SHAPE                                  # one page more than the table has
        assert call(form, ws=None) == B.MC_ERR_WORKSPACE and call(form, ws_bytes=8) == B.MC_ERR_WORKSPACE
        assert call(form, new=(0,), pool=None, ws=None) == B.MC_OK and call(form, batch=0, new=None, prefix=None) == B.MC_OK
        assert call(form, prefix=(0,) * 2 ** 10, new=(1,) * 2 ** 10, max_pages=2 ** 22) == B.MC_ERR_RANGE
    # many tokens in all: appends count new tokens, attention the keys
    many = dict(prefix=(2 ** 30,) * 3, new=(1, 1, 1), max_pages=2 ** 27, ws=None)
    assert call("prefill", **many) == B.MC_ERR_RANGE and call("append", **many) == B.MC_ERR_WORKSPACE
    assert call("expand", new=(2 ** 30,) * 2, max_pages=2 ** 27) == B.MC_ERR_RANGE
    for form in ("append_decode", "decode"):
        assert call(form, tokens=0) == B.MC_ERR_SHAPE and call(form, tokens=17) == B.MC_ERR_SHAPE and call(form, lens=None) == B.MC_ERR_NULL
        assert call(form, lens=FAKE + 2) == B.MC_ERR_ALIGN and call(form, batch=2 ** 20, max_pages=2 ** 20) == B.MC_ERR_RANGE
        assert call(form, batch=0, q=None, lens=None, ws=None) == B.MC_OK
    assert call("decode", q=None) == B.MC_ERR_NULL and call("decode", q=FAKE + 8) == B.MC_ERR_ALIGN and call("decode", lse=FAKE + 2) == B.MC_ERR_ALIGN
    assert call("decode", ws=None) == B.MC_ERR_WORKSPACE and call("decode", ws_bytes=1 << 20) == B.MC_ERR_WORKSPACE
    assert call("decode", batch=2 ** 26, max_pages=1) == B.MC_ERR_RANGE and call("append_decode", p=par(heads=1024), batch=BIG, max_pages=1) == B.MC_ERR_RANGE
    assert call("expand", weight=None) == B.MC_ERR_NULL and call("expand", weight=FAKE + 8) == B.MC_ERR_ALIGN
    for name in "kv":
        assert call("prefill", **{name: None}) == B.MC_ERR_NULL and call("prefill", **{name: FAKE + 8}) == B.MC_ERR_ALIGN
    for strides, status in (((2048, 256, -8, 256), B.MC_ERR_SHAPE), ((2048, 260, 2048, 256), B.MC_ERR_ALIGN), ((2 ** 26 + 8, 256, 2048, 256), B.MC_ERR_RANGE),
                            ((2048, 256, 2 ** 62, 256), B.MC_ERR_SHAPE), ((2 ** 26, 2 ** 28, 0, 0), B.MC_ERR_WORKSPACE)):
        assert call("prefill", strides=strides, ws=None) == status, strides


def test_workspaces():
    for n in (0, 1, 64, 65, 1000):
        assert 32 * max(n, 1) <= B.mc_latent_workspace_bytes(n) <= 32 * n + 64
    assert B.mc_latent_workspace_bytes(-1) == 0
    p = par(heads=16)
    l = B.lib()
    sizes = [B.mc_latent_decode_attn_workspace_bytes(p, n) for n in (0, 1, 256, 5000)]
    assert 0 < sizes[0] <= sizes[1] <= sizes[2] == sizes[3] < 1 << 26
    for bad in ((-1, 1), (1, 0), (1, 17)):
        assert B.mc_latent_decode_attn_workspace_bytes(p, *bad) == 0
    assert B.mc_latent_decode_attn_workspace_bytes(par(latent=100), 1) == 0 and l.mc_latent_decode_attn_workspace_bytes(None, 1, 1) == 0
    size = B.mc_latent_prefill_attn_workspace_bytes
    assert size(p, [], []) > 0 and size(p, [0], [0]) > 0 and size(p, [8192], [1]) > size(p, [0], [1])
    assert size(p, [-1], [1]) == 0 and size(p, [0], [-1]) == 0 and size(p, [2 ** 30] * 3, [1] * 3) == 0 and size(par(head_dim=32), [0], [1]) == 0
    assert l.mc_latent_prefill_attn_workspace_bytes(ctypes.byref(p), None, None, 1) == 0
    assert call("prefill", p=p, prefix=(8192,), new=(1,), max_pages=600, ws_bytes=size(p, [8192], [1]) - 1) == B.MC_ERR_WORKSPACE


DRIVER = r'''
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "latent_plan.h"
using namespace mc;
using namespace mc::host;
#define NEED(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)

// Stretches of a line: each has work, and they are the whole line.
static int line() {
  for (int stretches : {1, 2, 32, 85, 256})
    for (int total : {1, 2, 3, 63, 64, 65, 127, 128, 129, 1000, 12345, 1 << 20, (1 << 29) + 7})
      for (int rows : {1, 2, 7, 64, 1000}) {
        if (rows > total) continue;
        const int used = latent_used(total, rows, stretches);
        NEED(used >= 1 && used <= stretches && used <= total);
        NEED(decode_begin(total, 0, used) == 0 && decode_begin(total, used, used) == total);
        for (int w = 0; w < used; ++w) {
          const int64_t lo = decode_begin(total, w, used), hi = decode_begin(total, w + 1, used);
          NEED(lo < hi && decode_wave_of(total, lo, used) == w && decode_wave_of(total, hi - 1, used) == w);
        }
      }
  for (int64_t stacked = 1; stacked <= 16 * 1024; ++stacked) {
    const int rows = latent_tile_rows(stacked), tiles = latent_tiles(stacked);
    NEED((int64_t)rows * tiles >= stacked && (int64_t)rows * (tiles - 1) < stacked && latent_stretches(tiles) * tiles <= 256);
  }
  return 0;
}

// The work items as the kernel finds them: every piece of every row tile once, partial results beside each other.
static int items(int heads, int head_dim, const std::vector<int32_t>& prefix, const std::vector<int32_t>& fresh) {
  const mc_latent_params p = {heads, 512, 64, head_dim, 16, MC_DTYPE_BF16, 1 << 20, 0.f};
  const int32_t batch = (int32_t)prefix.size();
  const LatentPrefillLayout l = latent_prefill_layout(&p, prefix.data(), fresh.data(), batch);
  const int32_t entries = latent_entries(fresh.data(), batch);
  std::vector<LatentReq> reqs((size_t)entries);
  fill_latent_entries(&p, prefix.data(), fresh.data(), batch, reqs.data());
  fill_latent_items(entries, l.most_tiles, reqs.data());
  std::vector<int64_t> rows((size_t)batch, 0);               // of each request that some entry has
  int64_t item = 0, part = 0, cut = 0, tiles = 0, new_tiles = 0;
  for (int32_t r = 0; r < batch; ++r) tiles += latent_row_tiles(fresh[r]);
  NEED(entries <= batch || (entries <= 64 && batch <= 64));
  for (int32_t r = 0; r < entries; ++r) {
    const LatentReq& q = reqs[r];
    NEED(q.row >= 0 && q.row < batch);
    int64_t q_off = 0, k_off = 0;
    for (int i = 0; i < q.row; ++i) q_off += fresh[i], k_off += (int64_t)prefix[i] + fresh[i];
    const int64_t done = q.prefix - prefix[q.row];           // of its request, before the entry: whole row tiles
    NEED(done >= 0 && done % 256 == 0 && done + q.chunk <= fresh[q.row] && (done + q.chunk == fresh[q.row] || q.chunk % 256 == 0));
    NEED(q.q_off == q_off + done && q.k_off == k_off && q.item_off == item && q.part_off == part && q.cut_off == cut);
    rows[q.row] += q.chunk;
    NEED(entries == tiles || r == 0 || reqs[r - 1].prefix + reqs[r - 1].chunk >= q.prefix + q.chunk);
    for (int t = latent_row_tiles(q.chunk) - 1; t >= 0; --t) {
      const int keys = latent_key_tiles(q.prefix, q.chunk, t), pieces = latent_pieces(keys, l.most_tiles), height = latent_tile_height(q.chunk, t);
      NEED(height >= 1 && height <= 256 && keys >= 1 && pieces >= 1 && pieces <= keys);
      NEED((int64_t)keys * 64 >= q.prefix + (int64_t)t * 256 + height && (int64_t)(keys - 1) * 64 < q.prefix + (int64_t)t * 256 + height);
      item += pieces;
      new_tiles += 1;
      if (pieces > 1) cut += 1, part += (int64_t)pieces * height;
    }
  }
  for (int32_t r = 0; r < batch; ++r) NEED(rows[r] == fresh[r]);
  NEED(tiles == new_tiles && item == l.items && part == l.part_rows && cut == l.cut_tiles);
  NEED(l.o_off >= latent_table_bytes(batch) && l.ml_off - l.o_off >= (size_t)part * heads * head_dim * 4 && l.total - l.ml_off >= (size_t)part * heads * 8);
  NEED(item * heads <= 4 * 1024 || l.most_tiles == 0);
  return 0;
}

int main() {
  if (line() != 0) return 1;
  std::srand(7);
  for (int heads : {1, 3, 16, 128, 200, 300, 1024})
    for (int head_dim : {64, 128}) {
      if (items(heads, head_dim, {}, {}) || items(heads, head_dim, {0}, {0}) || items(heads, head_dim, {0}, {1}) ||
          items(heads, head_dim, {100000}, {1}) || items(heads, head_dim, {2000000000}, {5000}) || items(heads, head_dim, {0, 5, 0}, {0, 0, 0}))
        return 1;
      for (int n = 0; n < 60; ++n) {
        std::vector<int32_t> prefix(1 + std::rand() % 80), fresh(prefix.size());
        for (size_t i = 0; i < prefix.size(); ++i) {
          prefix[i] = std::rand() % 3 ? std::rand() % (1 << (1 + std::rand() % 17)) : 0;
          fresh[i] = std::rand() % 4 ? std::rand() % (1 << (1 + std::rand() % 13)) : 0;
        }
        if (items(heads, head_dim, prefix, fresh)) return 1;
      }
    }
  std::printf("ok\n");
  return 0;
}
'''


def test_how_work_is_cut(tmp_path):
    src, exe = tmp_path / "latent.cpp", tmp_path / "latent"
    src.write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-Wall", "-Wextra",
                    "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", str(exe), str(src), os.path.join(CSRC, "latent_plan.cpp"),
                    os.path.join(CSRC, "host_plan.cpp"), "-lpthread"], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0")
    res = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert res.returncode == 0 and res.stdout == "ok\n" and res.stderr == "", res.stdout + res.stderr


def test_the_kinds_of_the_calls():
    host, declared = {"prefix_lens", "new_lens", "lens"}, declarations()
    for function, kinds in B._LATENT_KINDS.items():
        want = ""
        for type_, name in declared[function]:
            if name in host:
                want += "I"
            elif type_.startswith(("const mc_latent_", "const mc_rope_")) or name == "strides":
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


STREAM = type("S", (), {"cuda_stream": 0})()
GOOD = dict(q=(3, 4, 64), kv=(3, 320), q_out=(3, 4, 64), norm=(256,), pool=(5, 16, 320), table=(3, 2), lens=(3,), aq=(3, 4, 320), aout=(3, 4, 256),
            lse=(3, 4), weight=(512, 256), both=(9, 4, 128), pq=(3, 4, 128), k=(9, 4, 64), v=(9, 4, 64), pout=(3, 4, 64), ws=(1 << 24,))
INTS = ("table", "lens")


def made(**change):
    t = {n: host(s, torch.int32 if n in INTS else torch.float32 if n == "lse" else torch.uint8 if n == "ws" else torch.bfloat16) for n, s in GOOD.items()}
    t.update(change)
    return t


def through(form, t, p=None, rope=None):
    p, rope = p or B.latent_params(4, 256, 64, 64, 16, 5), rope or B.rope_params(64, B.MC_ROPE_HALF)
    if form == "append":
        B.mc_latent_append_paged(p, rope, t["q"], t["kv"], t["norm"], t["q_out"], t["pool"], t["table"], [2] * 3, [1] * 3, t["ws"], STREAM)
    elif form == "append_decode":
        B.mc_latent_append_decode(p, rope, t["q"], t["kv"], t["norm"], t["q_out"], t["pool"], t["table"], t["lens"], 1, STREAM)
    elif form == "decode":
        B.mc_latent_decode_attn_paged(p, t["aq"], t["pool"], t["table"], t["lens"], 1, t["aout"], t["lse"], t["ws"], STREAM)
    elif form == "expand":
        B.mc_latent_expand_paged(p, t["weight"], t["pool"], t["table"], [3] * 3, t["both"], t["ws"], STREAM)
    else:
        B.mc_latent_prefill_attn_paged(p, t["pq"], t["k"], t["v"], t["pool"], t["table"], [2] * 3, [1] * 3, t["pout"], t["lse"], t["ws"], STREAM)


USES = dict(append=("q", "kv", "q_out", "norm", "pool", "table"), append_decode=("q", "kv", "q_out", "norm", "pool", "table", "lens"),
            decode=("aq", "aout", "pool", "table", "lens", "lse"), expand=("weight", "both", "pool", "table"),
            prefill=("pq", "k", "v", "pout", "pool", "table", "lse"))


@pytest.mark.parametrize("form,name", [(f, n) for f, names in USES.items() for n in names])
def test_the_binding_refuses_tensors_that_do_not_fit(form, name):
    """Another type, device or order, and one row too few: each is refused before anything is called."""
    shape, kind = GOOD[name], made()[name].dtype
    other = torch.int64 if name in INTS else torch.float16
    wrong = [host(shape, other), torch.empty(shape, dtype=kind)]
    if len(shape) > 1 or name not in INTS:
        wrong.append(host((shape[0] - 1, *shape[1:]), kind))
    if len(shape) > 1:
        wrong.append(host(shape, kind, tuple(2 * s for s in torch.empty(shape).stride())))
    if len(shape) == 3 and name in ("q", "q_out", "k", "v"):
        wrong.append(host((shape[0], shape[1] * shape[2]), kind))
    for t in wrong:
        with pytest.raises(ValueError):
            through(form, made(**{name: t}))


def test_the_binding_refuses_other_things(monkeypatch):
    for form in CALLS:
        with pytest.raises(TypeError):
            through(form, made(), B.attn_params(8, 2, 128, 16, 5, "bf16"))
        with pytest.raises(B.McError) as e:
            through(form, made(), par(heads=4, latent=256, head_dim=64, pages=5, dtype=B.MC_DTYPE_F32))
        assert e.value.status == B.MC_ERR_UNSUPPORTED
        if form != "append_decode":
            with pytest.raises(ValueError):
                through(form, made(ws=torch.empty(1 << 24, dtype=torch.uint8)))
    for form in ("append", "append_decode"):
        with pytest.raises(TypeError):
            through(form, made(), rope=par())
    p, t = B.latent_params(4, 256, 64, 64, 16, 5), made()
    with pytest.raises(ValueError):
        B.mc_latent_append_paged(p, B.rope_params(64, B.MC_ROPE_HALF), t["q"], t["kv"], None, t["q_out"], t["pool"], t["table"], [1, 2], [3], t["ws"], STREAM)
    with pytest.raises(ValueError):
        B.mc_latent_prefill_attn_paged(p, t["pq"], t["k"], t["v"], t["pool"], t["table"], [1, 2], [3], t["pout"], None, t["ws"], STREAM)
    with pytest.raises(B.McError) as e:
        B.mc_latent_expand_paged(None, t["weight"], t["pool"], t["table"], [3] * 3, t["both"], t["ws"], STREAM)
    assert e.value.status == B.MC_ERR_NULL
    monkeypatch.setattr(B, "_device", lambda: 1)              # the tensors lie on device 0
    for form in CALLS:
        with pytest.raises(ValueError):
            through(form, made())


def test_by_python_as_by_the_native_caller():
    from paper_2407_00079_amd import _mccall
    bf16 = torch.bfloat16
    for t in (host((4, 8, 64)), host((4, 8, 64), torch.float32), torch.empty((4, 8, 64), dtype=bf16), host((4, 8, 64), strides=(1024, 64, 1)),
              host((4, 8, 64), strides=(64, 256, 1)), host((4, 8, 64), strides=(512, 64, 2)), host((4, 512)), host((3, 8, 64)), host((4, 4, 64)),
              host((1, 8, 64), strides=(3, 64, 1)), host((4, 1, 64), strides=(600, 7, 1)), host((0, 8, 64)), host((1, 4, 8, 64))):
        for tokens, heads, dim in ((4, 8, 64), (1, 8, 64), (4, 1, 64), (0, 8, 64), (3, 8, 64)):
            assert _mccall.head_strides(0, bf16, t, tokens, heads, dim) == B._head_strides_by_python(0, bf16, t, tokens, heads, dim)
    with pytest.raises(TypeError):
        _mccall.head_strides(0, bf16, host((4, 8, 64)), 4, 8)
