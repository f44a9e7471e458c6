"""Calls with `stream=`: what they allocate is memory of that stream.  Memory of the current stream that was dropped may still be in
use by kernels queued there, behind which nothing orders a call on another stream; and a result that is dropped while the current stream
still reads it is not written by the next call."""
import math

import pytest
import torch

from paper_2609_37001_b200 import binding as B

pytestmark = pytest.mark.gpu
GRID, TILE, HEADS, SCALE = (4, 16, 32), (1, 16, 16), 4, 1.0 / math.sqrt(128.0)
TOKENS = math.prod(GRID)
PARAMS = [(2, 0, 0, 2, 0, 0), (1, 1, 2, 3, 0, 0), (1, 0, 0, 8, 0, 0), (3, 0, 1, 1, 0, 0)]


@pytest.fixture(scope="module")
def data():
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((HEADS, TOKENS, 128), device="cuda", generator=g).bfloat16() for _ in range(3))
    w = 1 + 0.2 * torch.randn((HEADS, 128), device="cuda", generator=g)
    _, row_ptr, col_idx = B.psa_mask_build(PARAMS, GRID, TILE)
    torch.cuda.synchronize()
    return q, k, v, w, row_ptr, col_idx


# more than one allocation in a call: scratch and weight sums come from the same stream
CALLS = {
    "mask_build": lambda d, s: B.psa_mask_build(PARAMS, GRID, TILE, stream=s),
    "attn_fwd": lambda d, s: B.psa_attn_fwd(*d[:3], PARAMS, GRID, TILE, SCALE, stream=s),
    "attn_fwd_batched": lambda d, s: B.psa_attn_fwd_batched(*(x.unsqueeze(0) for x in d[:3]), PARAMS, GRID, TILE, SCALE, stream=s),
    "attn_fwd_joint": lambda d, s: B.psa_attn_fwd_joint(*(x[:, :TOKENS - 8] for x in d[:3]), PARAMS, (3, 16, 32), TILE, SCALE, TOKENS // 4 - 8, stream=s),
    "search_losses": lambda d, s: (B.psa_search_losses(*(x[0] for x in d[:3]), PARAMS, GRID, TILE, SCALE, stream=s),),
    "qk_norm_rope": lambda d, s: B.psa_qk_norm_rope(*d[:2], GRID, q_weight=d[3], k_weight=d[3], stream=s),
    "qk_norm_rope_bwd": lambda d, s: B.psa_qk_norm_rope_bwd(d[2], d[2], *d[:2], GRID, q_weight=d[3], k_weight=d[3], stream=s),
    "select_blocks": lambda d, s: B.psa_select_blocks(*d[:2], GRID, TILE, 3, stream=s),
    "attn_fwd_lists": lambda d, s: B.psa_attn_fwd_lists(*d[:3], *d[4:], GRID, TILE, SCALE, stream=s),
}


def places(tensors):
    return {x.untyped_storage().data_ptr() for x in tensors}


@pytest.mark.parametrize("name", CALLS)
def test_dropped_memory_of_the_current_stream_is_left_alone(data, name):
    call, side = CALLS[name], torch.cuda.Stream()
    want = [x.clone() for x in call(data, None)]
    torch.cuda.synchronize()
    fresh = call(data, None)   # on the current stream: its memory, all of it, and then dropped
    held = places(fresh)
    sizes = [(x.untyped_storage().nbytes()) for x in fresh]
    torch.cuda.synchronize()
    del fresh
    got = call(data, side)
    torch.cuda.synchronize()
    assert not places(got) & held
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    del got
    # the same while the current stream is still busy with what it dropped
    late = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    torch.cuda._sleep(20_000_000)
    for x in late:
        x.fill_(7)
    del late, x
    got = call(data, side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("name", CALLS)
def test_dropped_results_are_not_written_while_the_current_stream_reads_them(data, name):
    call, side = CALLS[name], torch.cuda.Stream()
    got = call(data, side)
    torch.cuda.current_stream().wait_stream(side)
    want = [x.clone() for x in got]
    torch.cuda._sleep(20_000_000)
    late = [x.clone() for x in got]   # queued, not yet begun
    held = places(got)
    del got
    again = call(data, side)
    assert not places(again) & held
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, late, again))
