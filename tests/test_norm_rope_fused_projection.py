"""q, k and v as one projection leaves them, side by side in a token: norm and rotation hand q and k on with the strides that v
has, which every attention call asks for."""
import math

import pytest
import torch

from paper_2609_37001_b200 import binding as B
from paper_2609_37001_b200 import ulysses as U

GRID, TILE, HEADS, SCALE = (4, 16, 32), (1, 16, 16), 4, 1.0 / math.sqrt(128.0)
PARAMS = [(2, 0, 0, 2, 0, 0), (1, 1, 2, 3, 0, 0), (1, 0, 0, 8, 0, 0), (3, 0, 1, 1, 0, 0)]


def projection(tokens, seed, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((tokens, 3, HEADS, 128), device="cuda", generator=g).to(dtype)
    return [x[:, i].transpose(0, 1) for i in range(3)]


def apart(*tensors):
    return [x.contiguous() for x in tensors]


def test_new_tensors_have_the_strides_of_what_they_are_like():
    fused = torch.empty((2, 10, 3, 4, 128))[:, :, 1].transpose(1, 2)
    for x in (torch.empty((3, 5, 128)), torch.empty((5, 3, 128)).transpose(0, 1), torch.empty((3, 5, 136))[..., :128], fused, fused[:, :1], fused[0],
              torch.empty((3, 0, 128)), torch.empty((1, 1, 128)).as_strided((1, 1, 128), (7, 9, 1))):
        for dtype in (None, torch.bfloat16):
            for y in B._new_outputs(x, dtype, True):
                assert y.shape == x.shape and y.stride() == x.stride() and y.dtype == (dtype or x.dtype)
    # elements that share memory: heads half a row apart, tokens half a row apart
    for strides in ((64, 512, 1), (1024, 64, 1), (128, 128, 1)):
        x = torch.empty(8192).as_strided((2, 5, 128), strides)
        y, none = B._new_outputs(x, None, False)
        assert none is None and y.shape == x.shape and len(set((y.stride(0) * a + y.stride(1) * b) for a in range(2) for b in range(5))) == 10
        assert sorted(y.stride()) in ([1, 128, 256], [1, 128, 640])


@pytest.mark.gpu
def test_attention_takes_them():
    n = math.prod(GRID)
    q, k, v = projection(n, 1)
    q1, k1 = B.psa_qk_norm_rope(q, k, GRID, norm="token")
    assert q1.stride() == v.stride() and k1.stride() == v.stride()
    q2, k2 = B.psa_qk_norm_rope(*apart(q, k), GRID, norm="token")
    assert torch.equal(q1, q2) and torch.equal(k1, k2)
    got, want = (B.psa_attn_fwd(*x, PARAMS, GRID, TILE, SCALE) for x in ((q1, k1, v), apart(q1, k1, v)))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    lists = B.psa_select_blocks(q1, k1, GRID, TILE, 3)
    got, want = (B.psa_attn_fwd_lists(*x, *lists, GRID, TILE, SCALE) for x in ((q1, k1, v), apart(q1, k1, v)))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_joint_and_batched_attention_take_them():
    text, n = 40, math.prod(GRID)
    q, k, v = projection(n + text, 2)
    q1, k1 = B.psa_qk_norm_rope(q, k, GRID, n_text=text)
    got, want = (B.psa_attn_fwd_joint(*x, PARAMS, GRID, TILE, SCALE, text) for x in ((q1, k1, v), apart(q1, k1, v)))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    x = torch.randn((2, n, 3, HEADS, 128), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).bfloat16()
    q, k, v = (x[:, :, i].transpose(1, 2) for i in range(3))
    q1, k1 = B.psa_qk_norm_rope(q, k, GRID)
    out, lse = B.psa_attn_fwd_batched(q1, k1, v, PARAMS, GRID, TILE, SCALE)
    for b in range(2):   # (samples in one piece each are one launch of all their heads, which may share items otherwise: sample by sample)
        want = B.psa_attn_fwd(*apart(q1[b], k1[b], v[b]), PARAMS, GRID, TILE, SCALE)
        assert torch.equal(out[b], want[0]) and torch.equal(lse[b], want[1])


@pytest.mark.gpu
def test_the_head_sharded_call_takes_them():
    q, k, v = projection(math.prod(GRID), 4)
    got, want = (U.psa_attn_fwd_ulysses(*x, PARAMS, GRID, TILE, SCALE, norm_rope=dict(norm="token")) for x in ((q, k, v), apart(q, k, v)))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_inputs_that_share_memory_get_outputs_that_do_not():
    """Windows of one row of channels, each half a window further: as inputs these are in order."""
    buf = torch.randn(64 * 1024, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)).bfloat16()
    q = buf.as_strided((2, 30, 128), (16 * 1024, 128, 1))
    same = buf.as_strided((2, 30, 128), (128, 128, 1))   # head 1 is head 0 one token on
    for x in (q, same):
        got, _ = B.psa_qk_norm_rope(x, None, (2, 3, 5), norm="token")
        want, _ = B.psa_qk_norm_rope(x.contiguous(), None, (2, 3, 5), norm="token")
        assert torch.equal(got, want)
