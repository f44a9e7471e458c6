"""Heads that lie more than 2^31 elements apart in memory: offsets of every operator in 64 bits."""
import math

import pytest
import torch

from paper_2609_37001_b200 import binding as B

GRID, TILE, TOKENS = (2, 16, 33), (1, 8, 16), 1056
APART = (1 << 31) + 128 * 1000   # elements between heads


@pytest.fixture(scope="module")
def far():
    """Three tensors [2, TOKENS, 128] in one buffer, and copies of them close together."""
    buf = torch.empty(APART + 4 * TOKENS * 128, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    views = [torch.as_strided(buf, (2, TOKENS, 128), (APART, 128, 1), i * TOKENS * 128) for i in range(4)]
    for v in views[:3]:
        v.copy_(torch.randn(v.shape, device="cuda", generator=g))
    return views, [v.clone(memory_format=torch.contiguous_format) for v in views[:3]]


@pytest.mark.gpu
def test_norm_rope(far):
    (q, k, dq, out), (qc, kc, dqc) = far
    how = dict(norm="token", q_weight=torch.full((2, 128), 1.5, device="cuda"))
    want = B.psa_qk_norm_rope(qc, None, GRID, **how)[0]
    assert torch.equal(B.psa_qk_norm_rope(q, None, GRID, **how)[0], want)
    out.zero_()
    B.psa_qk_norm_rope(qc, None, GRID, out=(out, None), **how)
    assert torch.equal(out, want)
    for a, b in zip(B.psa_qk_norm_rope_bwd(dq, None, k, None, GRID, **how), B.psa_qk_norm_rope_bwd(dqc, None, kc, None, GRID, **how)):
        assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.gpu
def test_select_and_lists(far):
    (q, k, v, out), (qc, kc, vc) = far
    lists = B.psa_select_blocks(q, k, GRID, TILE, 3)
    assert all(torch.equal(a, b) for a, b in zip(lists, B.psa_select_blocks(qc, kc, GRID, TILE, 3)))
    scale = 1.0 / math.sqrt(128.0)
    want, want_lse = B.psa_attn_fwd_lists(qc, kc, vc, *lists, GRID, TILE, scale)
    out.zero_()
    got, lse = B.psa_attn_fwd_lists(q, k, v, *lists, GRID, TILE, scale, out=out)
    assert B.psa_last_device_status() == (0, 0)
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
