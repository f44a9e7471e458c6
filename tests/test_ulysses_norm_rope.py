"""The head-sharded call with norm and rotation in front: each rank treats its own tokens, at their place in the sequence (two
gloo ranks on CPU with plain functions in the place of the kernels; one rank with the kernels)."""
import os

import pytest
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

from paper_2609_37001_b200 import ulysses as U
from test_norm_rope import _root, _rotate, _turns, _weight
from test_ulysses_gloo import D, GRID, NH, PARAMS, SCALE, TILE, _free_port, _full_inputs, _oracle_attn

DIMS = (4, 4, 8)


def _plain(q, k, grid, first_token=0, norm="token", q_weight=None, k_weight=None):
    angle = _turns(grid, DIMS, (2, 0, 0), (1, 1, 1), first_token, q.shape[1])
    return [_rotate(x * _root(x, norm, 1e-6) * _weight(w), angle, "halves") for x, w in ((q, q_weight), (k, k_weight))]


def _options():
    g = torch.Generator().manual_seed(6)
    return dict(norm="token", q_weight=1 + 0.2 * torch.randn((NH, D), generator=g), k_weight=1 + 0.2 * torch.randn((NH, D), generator=g))


def _worker(rank, world, port, out):
    os.environ["MASTER_ADDR"] = "127.0.0.1"
    os.environ["MASTER_PORT"] = str(port)
    dist.init_process_group("gloo", rank=rank, world_size=world)
    try:
        q, k, v = _full_inputs()
        lc = q.shape[1] // world
        sl = slice(rank * lc, (rank + 1) * lc)
        o, lse = U.psa_attn_fwd_ulysses(*(t[:, sl].contiguous() for t in (q, k, v)), PARAMS, GRID, TILE, SCALE, attn_fn=_oracle_attn,
                                        norm_rope=_options(), norm_rope_fn=_plain)
        ro, rl = _oracle_attn(*_plain(q, k, GRID, **_options()), v, PARAMS, GRID, TILE, SCALE)
        same = torch.isinf(lse) == torch.isinf(rl[:, sl])
        out.put((rank, float((o - ro[:, sl]).abs().max()), bool(same.all()), float((lse - rl[:, sl])[torch.isfinite(lse)].abs().max())))
        dist.barrier()
    finally:
        dist.destroy_process_group()


def test_two_ranks_match_the_whole_sequence():
    world, port = 2, _free_port()
    ctx = mp.get_context("spawn")
    queue = ctx.Queue()
    procs = [ctx.Process(target=_worker, args=(r, world, port, queue)) for r in range(world)]
    for p in procs:
        p.start()
    got = sorted(queue.get(timeout=180) for _ in range(world))
    for p in procs:
        p.join(timeout=60)
        assert p.exitcode == 0
    for _, off, same, lse_off in got:
        assert off < 1e-12 and same and lse_off < 1e-12


def test_options_that_name_tokens_are_refused():
    q, k, v = _full_inputs()
    for bad in (dict(first_token=0), dict(n_text=3), dict(out=(q, k))):
        with pytest.raises(ValueError):
            U.psa_attn_fwd_ulysses(q, k, v, PARAMS, GRID, TILE, SCALE, attn_fn=_oracle_attn, norm_rope=bad, norm_rope_fn=_plain)


@pytest.mark.gpu
def test_one_rank_calls_the_kernels():
    from paper_2609_37001_b200 import binding as B
    grid, tile = (4, 12, 16), (1, 8, 16)
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn((2, 768, 128), device="cuda", generator=g).bfloat16() for _ in range(3))
    params = [(2, 0, 0, 2, 0, 0), (1, 1, 2, 3, 0, 0)]
    how = dict(dims=(16, 56, 56), norm="token", q_weight=torch.randn(128, device="cuda", generator=g), k_weight=torch.ones(128, device="cuda"))
    got = U.psa_attn_fwd_ulysses(q, k, v, params, grid, tile, 0.088, norm_rope=how)
    want = B.psa_attn_fwd(*B.psa_qk_norm_rope(q, k, grid, **how), v, params, grid, tile, 0.088)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
