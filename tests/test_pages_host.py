"""What the calls on a cache's pages refuse on the host.  Nothing is launched."""
import ctypes

import pytest
import torch

from paper_2407_00079_amd import binding as B
from test_rope_host import FAKE, host

OK = dict(rc=FAKE, pages=64, bt=FAKE, wide=8, page=16, lens=FAKE, rows=4, src=FAKE, dst=FAKE, n=2, moves=FAKE, count=FAKE, report=FAKE, ws=FAKE,
          ws_bytes=1 << 20)


def call(form, **change):
    a = dict(OK, **change)
    state = (a["rc"], a["pages"], a["bt"], a["wide"], a["page"], a["lens"], a["rows"])
    l = B.lib()
    if form == "fork":
        return l.mc_kv_pages_fork(*state, a["src"], a["dst"], a["n"], a["moves"], a["report"], a["ws"], a["ws_bytes"], None)
    if form == "grow":
        return l.mc_kv_pages_grow(*state, a["src"], a["report"], a["ws"], a["ws_bytes"], None)
    if form == "free":
        return l.mc_kv_pages_free(*state, a["src"], a["n"], a["report"], None)
    if form == "remap":
        return l.mc_kv_pages_remap(*state, a["moves"], a["count"], a["n"], None)
    return l.mc_kv_pages_compact(a["rc"], a["pages"], a["n"], a["moves"], a["report"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("form", ["fork", "grow", "free", "remap"])
@pytest.mark.parametrize("change,status", [
    (dict(rc=None), B.MC_ERR_NULL), (dict(bt=None), B.MC_ERR_NULL), (dict(lens=None), B.MC_ERR_NULL), (dict(rc=FAKE + 2), B.MC_ERR_ALIGN),
    (dict(bt=FAKE + 1), B.MC_ERR_ALIGN), (dict(lens=FAKE + 3), B.MC_ERR_ALIGN), (dict(pages=0), B.MC_ERR_SHAPE), (dict(pages=-1), B.MC_ERR_SHAPE),
    (dict(rows=-1), B.MC_ERR_SHAPE), (dict(wide=-1), B.MC_ERR_SHAPE), (dict(page=0), B.MC_ERR_SHAPE), (dict(pages=2 ** 31), B.MC_ERR_RANGE),
    (dict(rows=2 ** 20, wide=2 ** 20), B.MC_ERR_RANGE), (dict(wide=2 ** 20, page=2 ** 20, rows=1), B.MC_ERR_RANGE)])
def test_the_state(form, change, status):
    assert call(form, **change) == status


@pytest.mark.parametrize("form,change,status", [
    ("fork", dict(src=None), B.MC_ERR_NULL), ("fork", dict(dst=None), B.MC_ERR_NULL), ("fork", dict(moves=None), B.MC_ERR_NULL),
    ("fork", dict(report=None), B.MC_ERR_NULL), ("fork", dict(n=-1), B.MC_ERR_SHAPE), ("fork", dict(n=5), B.MC_ERR_SHAPE),
    ("fork", dict(ws=None), B.MC_ERR_WORKSPACE), ("fork", dict(ws_bytes=20), B.MC_ERR_WORKSPACE), ("fork", dict(ws=FAKE + 4), B.MC_ERR_ALIGN),
    ("fork", dict(moves=FAKE + 2), B.MC_ERR_ALIGN), ("fork", dict(n=0, src=None, ws=None), B.MC_OK),
    ("grow", dict(src=None), B.MC_ERR_NULL), ("grow", dict(report=None), B.MC_ERR_NULL), ("grow", dict(ws=None), B.MC_ERR_WORKSPACE),
    ("grow", dict(src=FAKE + 2), B.MC_ERR_ALIGN), ("grow", dict(rows=0, src=None), B.MC_OK),
    ("free", dict(src=None), B.MC_ERR_NULL), ("free", dict(report=None), B.MC_ERR_NULL), ("free", dict(n=-1), B.MC_ERR_SHAPE),
    ("free", dict(report=FAKE + 2), B.MC_ERR_ALIGN), ("free", dict(n=0, src=None), B.MC_OK), ("free", dict(rows=0), B.MC_OK),
    ("remap", dict(moves=None), B.MC_ERR_NULL), ("remap", dict(n=-1), B.MC_ERR_SHAPE), ("remap", dict(count=FAKE + 2), B.MC_ERR_ALIGN),
    ("remap", dict(n=0, moves=None), B.MC_OK), ("remap", dict(rows=0, rc=None), B.MC_ERR_NULL),
    ("compact", dict(rc=None), B.MC_ERR_NULL), ("compact", dict(moves=None), B.MC_ERR_NULL), ("compact", dict(report=None), B.MC_ERR_NULL),
    ("compact", dict(pages=0), B.MC_ERR_SHAPE), ("compact", dict(n=-1), B.MC_ERR_SHAPE), ("compact", dict(pages=2 ** 30), B.MC_ERR_RANGE),
    ("compact", dict(ws=None), B.MC_ERR_WORKSPACE), ("compact", dict(ws_bytes=4), B.MC_ERR_WORKSPACE), ("compact", dict(moves=FAKE + 1), B.MC_ERR_ALIGN),
    ("compact", dict(n=0, moves=None), B.MC_OK)])
def test_refusals(form, change, status):
    assert call(form, **change) == status


def test_workspace():
    assert B.mc_kv_pages_workspace_bytes(64, 4) >= 4 + 3 * 16 and B.mc_kv_pages_workspace_bytes(1 << 20, 0) >= 1024
    assert B.mc_kv_pages_workspace_bytes(0, 4) == 0 and B.mc_kv_pages_workspace_bytes(64, -1) == 0 and B.mc_kv_pages_workspace_bytes(2 ** 31, 1) == 0


def copy_pages(k=(FAKE,), v=(FAKE,), layers=1, pages=64, page_bytes=4096, moves=FAKE, count=None, n=2):
    lists = [None if x is None else (ctypes.c_int64 * max(1, len(x)))(*x) for x in (k, v)]
    return B.lib().mc_kv_copy_pages(*lists, layers, pages, page_bytes, moves, count, n, None)


@pytest.mark.parametrize("change,status", [
    (dict(k=None), B.MC_ERR_NULL), (dict(v=None), B.MC_ERR_NULL), (dict(k=(0,)), B.MC_ERR_NULL), (dict(moves=None), B.MC_ERR_NULL),
    (dict(v=(FAKE + 8,)), B.MC_ERR_ALIGN), (dict(moves=FAKE + 2), B.MC_ERR_ALIGN), (dict(count=FAKE + 2), B.MC_ERR_ALIGN),
    (dict(page_bytes=4100), B.MC_ERR_ALIGN), (dict(page_bytes=-16), B.MC_ERR_SHAPE), (dict(layers=-1), B.MC_ERR_SHAPE), (dict(n=-1), B.MC_ERR_SHAPE),
    (dict(pages=0), B.MC_ERR_SHAPE), (dict(layers=129, k=(FAKE,) * 129, v=(FAKE,) * 129), B.MC_ERR_RANGE), (dict(pages=2 ** 31), B.MC_ERR_RANGE),
    (dict(layers=0, k=None, v=None), B.MC_OK), (dict(n=0, moves=None), B.MC_OK), (dict(page_bytes=0), B.MC_OK)])
def test_copies_refused(change, status):
    assert copy_pages(**change) == status


def i32(*shape):
    return host(shape, torch.int32)


def test_the_binding_refuses_tensors_that_do_not_fit():
    good = dict(counts=i32(64), tables=i32(4, 8), lens=i32(4), src=i32(2), dst=i32(2), moves=i32(2, 2), report=i32(4), add=i32(4), rows=i32(9))
    stream = type("S", (), {"cuda_stream": 0})()
    calls = dict(
        fork=lambda t: B.mc_kv_pages_fork(t["counts"], t["tables"], 16, t["lens"], t["src"], t["dst"], t["moves"], t["report"], None, stream),
        grow=lambda t: B.mc_kv_pages_grow(t["counts"], t["tables"], 16, t["lens"], t["add"], t["report"], None, stream),
        free=lambda t: B.mc_kv_pages_free(t["counts"], t["tables"], 16, t["lens"], t["rows"], t["report"], stream),
        compact=lambda t: B.mc_kv_pages_compact(t["counts"], t["moves"], t["report"], None, stream),
        remap=lambda t: B.mc_kv_pages_remap(t["counts"], t["tables"], 16, t["lens"], t["moves"], t["dst"], stream))
    uses = dict(counts="fork grow free compact remap", tables="fork grow free remap", lens="fork grow free remap", moves="fork compact remap",
                report="fork grow free compact", src="fork", dst="fork remap", add="grow", rows="free")
    for name, forms in uses.items():
        for form in forms.split():
            bad = [host(good[name].shape, torch.int64), torch.empty(good[name].shape, dtype=torch.int32)]
            if name in ("report", "add", "dst") and form != "remap":
                bad.append(i32(1))
            if name == "tables":
                bad += [i32(3, 8), i32(32), host((4, 8), torch.int32, (16, 1))]
            if name == "moves":
                bad.append(host((2, 2), torch.int32, (1, 2)))
            for b in bad:
                with pytest.raises(ValueError):
                    calls[form](dict(good, **{name: b}))


def test_the_binding_refuses_pools_that_do_not_fit():
    stream, moves = type("S", (), {"cuda_stream": 0})(), i32(2, 2)
    pool = host((64, 2048))
    for k, v in (([pool], []), ([host((63, 2048))], [pool]), ([pool], [torch.empty((64, 2048), dtype=torch.bfloat16)]),
                 ([host((64, 1024), strides=(1100, 1))], [host((64, 1024))])):
        with pytest.raises(ValueError):
            B.mc_kv_copy_pages(k, v, 64, 4096, moves, None, stream)
