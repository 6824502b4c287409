"""The cache calls refuse tensors in host memory, all of them alike or not: the kernels would follow their addresses."""
import pytest
import torch

from paper_2407_00079_amd import binding as B


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


P = B.attn_params(8, 2, 128, 16, 9, "bf16")
Q, KV, POOL = (torch.zeros(s, dtype=torch.bfloat16) for s in ((3, 8, 128), (3, 2, 128), (9, 2, 16, 128)))
STATE, STREAM, WS = (i32(64), i32(4, 8), 16, i32(4)), type("S", (), {"cuda_stream": 0})(), torch.zeros(1 << 23, dtype=torch.uint8)
ROPE = (Q, KV, KV, None, None, Q, POOL, POOL, i32(3, 4))
CALLS = dict(
    paged=lambda r: B.mc_kv_rope_append_paged(P, r, *ROPE, [0, 0, 0], [1, 1, 1], WS, STREAM),
    run=lambda r: B.mc_kv_rope_append_run(P, B.McAttnPlan(2, 3, 0, 3, 3, 1, 8, 2, 0, 0), r, *ROPE, WS, STREAM),
    tokens=lambda r: B.mc_kv_rope_append_decode(P, r, *ROPE, i32(3), STREAM),
    decode=lambda r: B.mc_decode_attn_paged(P, Q, POOL, POOL, i32(3, 4), i32(3), Q.clone(), None, WS, STREAM),
    fork=lambda r: B.mc_kv_pages_fork(*STATE, i32(2), i32(2), i32(2, 2), i32(4), WS, STREAM),
    grow=lambda r: B.mc_kv_pages_grow(*STATE, i32(4), i32(4), WS, STREAM),
    free=lambda r: B.mc_kv_pages_free(*STATE, i32(2), i32(4), STREAM),
    compact=lambda r: B.mc_kv_pages_compact(i32(64), i32(2, 2), i32(4), WS, STREAM),
    remap=lambda r: B.mc_kv_pages_remap(*STATE, i32(2, 2), None, STREAM),
    copy=lambda r: B.mc_kv_copy_pages([POOL], [POOL], 9, 8192, i32(2, 2), None, STREAM))


@pytest.mark.parametrize("name", CALLS)
def test_tensors_in_host_memory(name, monkeypatch):
    def enqueued(*_):
        raise AssertionError("handed to the library")

    rope = B.rope_params(128, B.MC_ROPE_HALF)
    monkeypatch.setattr(B, "_enqueue", enqueued)
    with pytest.raises(ValueError, match="GPU"):
        CALLS[name](rope)
