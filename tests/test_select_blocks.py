"""psa_select_blocks: the lists are whole numbers and equal to those of the definition in 64 bits, ties included."""
import ctypes
import math

import pytest
import torch

from paper_2609_37001_b200 import binding as B


def blocks_of_tokens(grid, tile):
    """Block of every token, and the number of blocks."""
    n = [-(-g // b) for g, b in zip(grid, tile)]
    t, h, w = (torch.arange(g) // b for g, b in zip(grid, tile))
    return ((t[:, None, None] * n[1] + h[None, :, None]) * n[2] + w[None, None, :]).reshape(-1), n[0] * n[1] * n[2]


def reference(q, k, grid, tile, keep, keep_self=False):
    """Lists [heads][blocks] of the definition."""
    block, nb = blocks_of_tokens(grid, tile)
    tokens = torch.bincount(block, minlength=nb).double()
    lists = []
    for h in range(q.shape[0]):
        sq, sk = (torch.zeros((nb, 128), dtype=torch.float64).index_add_(0, block, x[h].cpu().double()) for x in (q, k))
        s = sq @ sk.t() / tokens
        s = torch.where(s.isnan(), -math.inf, s)
        order = s.sort(dim=1, descending=True, stable=True).indices.tolist()
        if keep_self:   # before any other, one with an infinite score too
            order = [[i] + [j for j in row if j != i] for i, row in enumerate(order)]
        lists.append([sorted(row[:keep[h]]) for row in order])
    return lists


def check(got, lists):
    row_ptr, col_idx = (x.cpu().tolist() for x in got)
    flat = [row for head in lists for row in head]
    assert len(row_ptr) == len(flat) + 1 and row_ptr[0] == 0
    for r, row in enumerate(flat):
        assert col_idx[row_ptr[r]:row_ptr[r + 1]] == row, r
    assert len(col_idx) >= row_ptr[-1]


def normal(heads, tokens, seed, layout="head"):
    x = torch.randn((heads, tokens, 128), generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()
    return x if layout == "head" else x.transpose(0, 1).contiguous().transpose(0, 1)


# grid, tile, heads, keep, layout
CASES = [
    ((8, 16, 16), (2, 8, 16), 2, 3, "head"), ((5, 30, 52), (1, 30, 8), 3, 11, "token"), ((4, 9, 7), (1, 7, 9), 2, 1, "head"),
    ((7, 5, 3), (3, 5, 2), 1, 6, "head"), ((1, 1, 1), (1, 16, 16), 2, 1, "head"), ((1, 3, 2), (2, 8, 8), 1, 1, "head"),
    ((3, 17, 33), (1, 1, 1), 1, 100, "head"), ((2, 40, 60), (1, 2, 2), 2, [7, 300], "token"), ((9, 20, 33), (6, 8, 8), 3, [1, 20, 13], "head"),
    ((21, 45, 80), (1, 15, 16), 2, 79, "head"), ((5, 18, 38), (1, 1, 1), 1, 3420, "head"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%s-%s" % ("x".join(map(str, c[0])), "x".join(map(str, c[1])), c[3]))
@pytest.mark.parametrize("keep_self", [False, True])
def test_lists_are_those_of_the_definition(case, keep_self):
    grid, tile, heads, keep, layout = case
    q, k = (normal(heads, math.prod(grid), s, layout) for s in (1, 2))
    each = [keep] * heads if isinstance(keep, int) else keep
    got = B.psa_select_blocks(q, k, grid, tile, keep, keep_self=keep_self)
    check(got, reference(q, k, grid, tile, each, keep_self))
    again = B.psa_select_blocks(q, k, grid, tile, keep, keep_self=keep_self)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.gpu
@pytest.mark.parametrize("values", ["zeros", "signs", "few", "same"])
def test_equal_scores_go_to_the_lowest_block(values):
    """Scores that are equal exactly, between blocks that are equal and blocks that are not."""
    grid, tile, heads = (6, 16, 24), (1, 8, 8), 2
    g = torch.Generator().manual_seed(3)
    shape = (heads, math.prod(grid), 128)
    if values == "zeros":
        q = k = torch.zeros(shape)
    elif values == "signs":   # sums of +-1: whole numbers, the scores as well
        q, k = (torch.randint(0, 2, shape, generator=g) * 2.0 - 1.0 for _ in range(2))
        q[:, :, 4:] = 0
    elif values == "few":     # four kinds of blocks, -0 among them
        block, nb = blocks_of_tokens(grid, tile)
        kinds = torch.randn((heads, 4, 128), generator=g)
        kinds[:, 0] = -0.0
        q, k = kinds[:, block % 4], kinds[:, block % 3]
    else:
        q = k = torch.randn((heads, 1, 128), generator=g).expand(shape)
    q, k = (x.to(torch.bfloat16).cuda().contiguous() for x in (q, k))
    for keep in (1, 5, 17, 36):
        check(B.psa_select_blocks(q, k, grid, tile, keep), reference(q, k, grid, tile, [keep] * heads))


@pytest.mark.gpu
def test_values_that_are_not_finite():
    """NaN scores count as -infinity; every row still has its number of blocks."""
    grid, tile = (4, 16, 16), (1, 8, 8)
    q, k = (normal(2, 1024, s) for s in (1, 2))
    k[0, 0, 0], k[0, 300, 5], k[1, 700, 9], q[1, 0, 3] = math.inf, math.nan, -math.inf, math.nan
    for keep_self in (False, True):
        for keep in (1, 9, 16):
            check(B.psa_select_blocks(q, k, grid, tile, keep, keep_self=keep_self), reference(q, k, grid, tile, [keep] * 2, keep_self))
    big = torch.full((1, 1024, 128), torch.finfo(torch.bfloat16).max, dtype=torch.bfloat16, device="cuda")
    big[0, ::3] *= -1
    small = torch.full_like(big, 2.0 ** -133)   # (a subnormal value)
    for a, b in ((big, big), (small, big), (small, small)):
        check(B.psa_select_blocks(a, b, grid, tile, 5), reference(a, b, grid, tile, [5]))


@pytest.mark.gpu
def test_more_heads_than_a_launch_takes():
    grid, tile, heads = (2, 4, 4), (1, 2, 2), 131
    q, k = (normal(heads, 32, s) for s in (1, 2))
    keep = [1 + h % 8 for h in range(heads)]
    check(B.psa_select_blocks(q, k, grid, tile, keep), reference(q, k, grid, tile, keep))


@pytest.mark.gpu
def test_captured_with_buffers_of_the_caller():
    grid, tile, heads, keep = (3, 20, 30), (1, 10, 8), 2, 4
    q, k = (normal(heads, 1800, s) for s in (1, 2))
    nb = 3 * 2 * 4
    out = (torch.empty(heads * nb + 1, dtype=torch.int32, device="cuda"), torch.full((heads * nb * keep + 5,), -7, dtype=torch.int32, device="cuda"))
    scratch = torch.empty(B.psa_select_scratch_bytes(heads, grid, tile), dtype=torch.uint8, device="cuda")
    B.psa_select_blocks(q, k, grid, tile, keep, out=out, scratch=scratch)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.psa_select_blocks(q, k, grid, tile, keep, out=out, scratch=scratch)
    for s in (5, 6):
        q.copy_(normal(heads, 1800, s))
        graph.replay()
        check(out, reference(q, k, grid, tile, [keep] * heads))
        assert (out[1][-5:] == -7).all()


def test_refusals():
    f = B.lib().psa_select_blocks
    keep = (ctypes.c_int32 * 2)(1, 4)

    def call(q=4096, k=8192, heads=2, tile=(1, 8, 8), grid=(1, 16, 16), strides=(128 * 256, 128), d=128, keep=keep, row_ptr=64, col_idx=128, room=20,
             scratch=256):
        return f(q, k, B._problem(heads, tile, 1.0, *strides, d), *grid, keep, 0, row_ptr, col_idx, room, scratch, None)

    bad = B.PSA_ERR_INVALID_ARG
    for over in (dict(q=None), dict(k=None), dict(keep=None), dict(row_ptr=None), dict(col_idx=None), dict(scratch=None), dict(q=4104), dict(row_ptr=66),
                 dict(scratch=264), dict(heads=0), dict(tile=(0, 8, 8)), dict(grid=(0, 16, 16)), dict(strides=(128 * 256, 132)),
                 dict(strides=(64, 128)), dict(keep=(ctypes.c_int32 * 2)(0, 1)), dict(keep=(ctypes.c_int32 * 2)(1, 5))):
        assert call(**over) == bad, over
    assert call(d=64) == B.PSA_ERR_UNSUPPORTED
    assert call(grid=(1, 60, 60), tile=(1, 1, 1)) == B.PSA_ERR_UNSUPPORTED   # more blocks than it takes
    assert call(room=19) == B.PSA_ERR_CAPACITY
    q = torch.zeros((2, 4, 128), dtype=torch.bfloat16)
    for args in ((q, q[:1], (1, 2, 2), (1, 1, 1), 1), (q, q, (1, 2, 3), (1, 1, 1), 1), (q, q, (1, 2, 2), (1, 1, 1), 1)):   # (the last: no device tensors)
        with pytest.raises(ValueError):
            B.psa_select_blocks(*args)
