"""Attention over lists of key blocks against the definition in 64 bits.

Tolerances: probabilities are rounded to bf16 (2^-8 of each) before they meet the values, the output is rounded once more.  A score
is a sum of 128 products in 32 bits, off by at most 128 u of the sum of their magnitudes (u = 2^-24) -- which moves a probability by
that, relative, and lse by that -- and the exponential by 4 u.  A row's sum over n keys rounds n times.
"""
import math

import pytest
import torch

from paper_2609_37001_b200 import binding as B
from test_select_blocks import blocks_of_tokens
from test_select_blocks import reference as select_reference

U = 2.0 ** -24
SCALE = 1.0 / math.sqrt(128.0)


def tensors(heads, tokens, seed, layout="head"):
    g = torch.Generator().manual_seed(seed)
    got = []
    for _ in range(3):
        x = torch.randn((heads, tokens, 128), generator=g).to(torch.bfloat16).cuda()
        got.append(x if layout == "head" else x.transpose(0, 1).contiguous().transpose(0, 1))
    return got


def pack(lists):
    """(row_ptr, col_idx) of lists [heads][blocks]."""
    flat = [row for head in lists for row in head]
    ptr = torch.tensor([0] + [len(r) for r in flat], dtype=torch.int64).cumsum(0).to(torch.int32)
    return ptr.cuda(), torch.tensor([j for r in flat for j in r], dtype=torch.int32).cuda()


def random_lists(heads, nb, seed, kind, keep=None):
    g = torch.Generator().manual_seed(seed)
    lists = []
    for _ in range(heads):
        rows = []
        for _ in range(nb):
            n = {"none": 0, "one": 1, "all": nb, "ragged": int(torch.randint(0, nb + 1, (), generator=g)), "even": keep}[kind]
            if kind == "ragged" and int(torch.randint(0, 4, (), generator=g)) == 0:
                n = 0
            rows.append(sorted(torch.randperm(nb, generator=g)[:n].tolist()))
        lists.append(rows)
    return lists


def check(out, lse, q, k, v, lists, grid, tile, text=0, scale=SCALE):
    block, nb = blocks_of_tokens(grid, tile)
    n_video = math.prod(grid)
    members = [torch.nonzero(block == b).squeeze(1) for b in range(nb)]
    texts = torch.arange(n_video, n_video + text)
    for h in range(q.shape[0]):
        qh, kh, vh = (x[h].cpu().double() for x in (q, k, v))
        jobs = [(members[b], torch.cat([members[j] for j in lists[h][b]] + [texts]).long()) for b in range(nb)]
        if text:
            jobs.append((texts, torch.arange(n_video + text)))
        for rows, keys in jobs:
            o, m = out[h].cpu()[rows].double(), lse[h].cpu()[rows].double()
            if keys.numel() == 0:
                assert (o == 0).all() and (m == -math.inf).all()
                continue
            s = qh[rows] @ kh[keys].t() * scale
            p = s.softmax(1)
            want, met = p @ vh[keys], p @ vh[keys].abs()
            score = 128 * U * scale * float((qh[rows].abs() @ kh[keys].abs().t()).max()) + 4 * U
            off = (o - want).abs()
            limit = (2.0 ** -8 + 2 * score + keys.numel() * U) * met + 2.0 ** -8 * want.abs() + 1e-30
            assert (off <= limit).all(), (h, float((off / limit).max()))
            ref = s.logsumexp(1)
            assert ((m - ref).abs() <= score + (keys.numel() + 16) * U + 8 * U * ref.abs()).all()


# grid, tile, heads, kind, keep, text, layout
CASES = [
    ((8, 16, 16), (2, 8, 16), 2, "even", 3, 0, "head"),
    ((8, 16, 16), (2, 8, 16), 2, "ragged", None, 0, "token"),
    ((4, 30, 20), (1, 30, 8), 3, "ragged", None, 0, "head"),      # blocks cut at the width, 240 tokens
    ((3, 45, 33), (1, 15, 16), 2, "ragged", None, 37, "token"),   # a 112-token slab; text
    ((7, 17, 35), (3, 8, 16), 2, "ragged", None, 0, "head"),      # three slabs, edge blocks of fewer
    ((5, 9, 9), (6, 8, 8), 2, "all", None, 0, "head"),            # one block along the frames, which it exceeds
    ((2, 40, 40), (1, 8, 16), 4, "ragged", None, 0, "head"),      # one slab a block
    ((2, 40, 40), (1, 8, 16), 1, "one", None, 200, "token"),
    ((1, 1, 1), (1, 16, 16), 1, "all", None, 0, "head"),          # one token
    ((1, 1, 1), (1, 8, 16), 2, "none", None, 1, "head"),          # one token of text
    ((3, 16, 48), (1, 16, 16), 3, "none", None, 0, "head"),
    ((3, 16, 48), (1, 16, 16), 40, "ragged", None, 130, "head"),  # more items than run at once
    ((6, 32, 33), (1, 32, 4), 20, "ragged", None, 0, "head"),
    ((11, 30, 52), (1, 30, 8), 3, "even", 77, 0, "head"),         # every block of long lists
    ((5, 32, 48), (1, 16, 16), 5, "all", None, 0, "head"),        # two CTAs an item, more of them than run at once
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%s-%dx%s-%d" % ("x".join(map(str, c[0])), "x".join(map(str, c[1])), c[2], c[3], c[5]))
def test_against_the_definition(case):
    grid, tile, heads, kind, keep, text, layout = case
    n = math.prod(grid)
    q, k, v = tensors(heads, n + text, 1, layout)
    nb = blocks_of_tokens(grid, tile)[1]
    lists = random_lists(heads, nb, 2, kind, keep)
    row_ptr, col_idx = pack(lists)
    out, lse = B.psa_attn_fwd_lists(q, k, v, row_ptr, col_idx, grid, tile, SCALE, n_text=text)
    assert B.psa_last_device_status() == (0, 0)
    check(out, lse, q, k, v, lists, grid, tile, text)
    again = B.psa_attn_fwd_lists(q, k, v, row_ptr, col_idx, grid, tile, SCALE, n_text=text)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.gpu
def test_all_ways_of_handing_out_items():
    seen = set()
    for grid, tile, heads, kind in (((8, 16, 16), (2, 8, 16), 2, "all"), ((3, 16, 48), (1, 16, 16), 40, "ragged"), ((4, 16, 16), (1, 16, 16), 30, "one"),
                                    ((4, 32, 48), (1, 8, 16), 20, "ragged"), ((4, 31, 47), (1, 8, 16), 20, "ragged")):
        q, k, v = tensors(heads, math.prod(grid), 5)
        lists = random_lists(heads, blocks_of_tokens(grid, tile)[1], 6, kind)
        out, lse = B.psa_attn_fwd_lists(q, k, v, *pack(lists), grid, tile, SCALE)
        seen.add(B.psa_last_attn_launch()[1])
        check(out, lse, q, k, v, lists, grid, tile)
    assert seen == {"ticket", "ticket_short", "direct", "shared_direct"}


@pytest.mark.gpu
@pytest.mark.parametrize("tile", [(1, 16, 16), (3, 8, 16), (1, 8, 16)])
def test_lists_of_a_stripe_mask(tile):
    """The lists that psa_mask_build writes give what psa_attn_fwd gives, up to the order of its sums."""
    grid, params = (6, 32, 40), [(1, 0, 3, 3, 1, 5), (2, 1, 0, 4, 0, 0), (9, 0, 0, 99, 0, 0)]
    q, k, v = tensors(3, math.prod(grid), 7)
    _, row_ptr, col_idx = B.psa_mask_build(params, grid, tile)
    out, lse = B.psa_attn_fwd_lists(q, k, v, row_ptr, col_idx, grid, tile, SCALE)
    want, want_lse = B.psa_attn_fwd(q, k, v, params, grid, tile, SCALE)
    assert (out.float() - want.float()).abs().max() <= 2 ** -6 * v.float().abs().max()
    inside = want_lse > -math.inf
    assert torch.equal(inside, lse > -math.inf) and (lse - want_lse)[inside].abs().max() <= 1e-4


@pytest.mark.gpu
def test_a_layer():
    """Norm and rotation, choice, attention, as they are used together."""
    grid, tile, heads, text, keep = (5, 30, 20), (1, 15, 16), 3, 40, 6
    n = math.prod(grid)
    g = torch.Generator().manual_seed(9)
    qkv = torch.randn((n + text, 3, heads, 128), generator=g).to(torch.bfloat16).cuda()
    q, k, v = (qkv[:, i].transpose(0, 1) for i in range(3))
    w = (1.0 + 0.2 * torch.randn((heads, 128), generator=g)).cuda()
    v = v.contiguous()
    q, k = B.psa_qk_norm_rope(q, k, grid, norm="token", q_weight=w, k_weight=w, n_text=text, out=(torch.empty_like(v), torch.empty_like(v)))
    row_ptr, col_idx = B.psa_select_blocks(q[:, :n], k[:, :n], grid, tile, keep, keep_self=True)
    out, lse = B.psa_attn_fwd_lists(q, k, v, row_ptr, col_idx, grid, tile, SCALE, n_text=text)
    lists = select_reference(q[:, :n], k[:, :n], grid, tile, [keep] * heads, True)
    assert col_idx.cpu().tolist() == [j for head in lists for row in head for j in row]
    check(out, lse, q, k, v, lists, grid, tile, text)


@pytest.mark.gpu
def test_keys_outside_the_lists_are_not_read():
    """Values that are not finite in blocks that no list of a head has do not reach it."""
    grid, tile = (4, 16, 32), (1, 16, 16)
    q, k, v = tensors(2, math.prod(grid), 11)
    lists = [[[j for j in range(8) if j != 3] for _ in range(8)] for _ in range(2)]
    want = B.psa_attn_fwd_lists(q, k, v, *pack(lists), grid, tile, SCALE)
    at = blocks_of_tokens(grid, tile)[0] == 3
    for x, value in ((k, math.inf), (v, math.nan)):
        x[:, at.cuda()] = value
    got = B.psa_attn_fwd_lists(q, k, v, *pack(lists), grid, tile, SCALE)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_graphs_and_streams():
    """Two captured calls of other lists, each with its scratch, replayed at once on two streams beside an eager call before."""
    grid, tile, heads = (3, 16, 48), (1, 16, 16), 30
    q, k, v = tensors(heads, math.prod(grid), 13)
    graphs = []
    for seed in (1, 2):
        lists = random_lists(heads, 9, seed, "ragged")
        ptr_col = pack(lists)
        want = B.psa_attn_fwd_lists(q, k, v, *ptr_col, grid, tile, SCALE)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = B.psa_attn_fwd_lists(q, k, v, *ptr_col, grid, tile, SCALE)
        graphs.append((graph, got, want, ptr_col))
    B.psa_shutdown()   # (the library's workspace is none of theirs)
    for _ in range(3):
        for graph, got, want, _ in graphs:
            got[0].zero_()
            graph.replay()
    torch.cuda.synchronize()
    assert B.psa_last_device_status() == (0, 0)
    for _, got, want, _ in graphs:
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    _, got, want, ptr_col = graphs[0]
    out, lse = B.psa_attn_fwd_lists(q, k, v, *ptr_col, grid, tile, SCALE, stream=side)
    side.synchronize()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [1, 40])
@pytest.mark.parametrize("fault", ["negative", "beyond", "twice", "descending", "row_before", "row_behind", "row_backwards", "row_long"])
def test_bad_lists_are_reported_and_left_out(heads, fault):
    """What the caller's lists may not hold is caught by the kernel before any address is made of it."""
    grid, tile = (3, 16, 48), (1, 16, 16)
    q, k, v = tensors(heads, math.prod(grid), 17)
    lists = [[[0, 2, 5, 7] for _ in range(9)] for _ in range(heads)]
    row_ptr, col_idx = pack(lists)
    row, head = 4, heads - 1
    r = head * 9 + row
    start = int(row_ptr[r])
    lists[head][row] = [0, 2, 7]
    if fault in ("negative", "beyond", "twice"):
        col_idx[start + 2] = {"negative": -1, "beyond": 9, "twice": 2}[fault]
        lists[head][row] = {"negative": [0, 2, 7], "beyond": [0, 2], "twice": [0, 2, 7]}[fault]   # (7 is not behind 9)
    elif fault == "descending":
        col_idx[start + 3] = 1
        lists[head][row] = [0, 2, 5]
    else:   # a row's end is the next one's beginning: the last row's end, or two rows
        if fault == "row_before":
            row_ptr[0] = -4
            head, row = 0, 0
        elif fault == "row_behind":
            row_ptr[-1] += 1
            head, row = heads - 1, 8
        elif fault == "row_backwards":
            row_ptr[-1] = row_ptr[-2] - 1
            head, row = heads - 1, 8
        else:
            col_idx = torch.cat([col_idx, torch.arange(8, dtype=torch.int32, device="cuda")])
            row_ptr[-1] += 8
            head, row = heads - 1, 8
        lists = [[[0, 2, 5, 7] for _ in range(9)] for _ in range(heads)]
        lists[head][row] = []
    out, lse = B.psa_attn_fwd_lists(q, k, v, row_ptr, col_idx, grid, tile, SCALE)
    status, detail = B.psa_last_device_status()
    assert status == B.PSA_ERR_INVALID_ARG and detail == (0x600 if fault.startswith("row") else 0x601)
    check(out, lse, q, k, v, lists, grid, tile)
    good = pack([[[1] for _ in range(9)] for _ in range(heads)])
    B.psa_attn_fwd_lists(q, k, v, *good, grid, tile, SCALE)
    assert B.psa_last_device_status() == (0, 0)


def test_refusals():
    f, size = B.lib().psa_attn_fwd_lists, B.lib().psa_attn_fwd_lists_scratch_bytes

    def call(q=4096, k=8192, v=16384, out=32768, lse=64, row_ptr=128, col_idx=256, n=4, heads=2, tile=(1, 16, 16), scale=0.1, strides=(128 * 256, 128),
             d=128, text=0, grid=(1, 16, 16), scratch=512):
        return f(q, k, v, out, lse, row_ptr, col_idx, n, B._problem(heads, tile, scale, *strides, d), text, *grid, scratch, None)

    for over in (dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(lse=None), dict(row_ptr=None), dict(col_idx=None), dict(scratch=None),
                 dict(n=-1), dict(q=4104), dict(out=32776), dict(lse=66), dict(row_ptr=129), dict(col_idx=254 + 4 - 1), dict(scratch=520), dict(out=4096),
                 dict(scale=0.0), dict(scale=math.nan), dict(text=-1), dict(heads=0), dict(grid=(1, 0, 16)), dict(strides=(128 * 256, 132)),
                 dict(strides=(64, 128))):
        assert call(**over) == B.PSA_ERR_INVALID_ARG, over
    for over in (dict(d=64), dict(tile=(1, 10, 10)), dict(tile=(1, 4, 4)), dict(n=1 << 31)):
        assert call(**over) == B.PSA_ERR_UNSUPPORTED, over
    assert size(B._problem(2, (1, 16, 16), 1.0, 0, 128), 0, 1, 16, 16) >= 2 * 16
    assert size(B._problem(2, (1, 10, 10), 1.0, 0, 128), 0, 1, 16, 16) == B.PSA_ERR_UNSUPPORTED
    q = torch.zeros((1, 4, 128), dtype=torch.bfloat16)
    ptr = torch.zeros(5, dtype=torch.int32)
    for args in ((q, q, q, ptr, ptr, (1, 2, 3)), (q, q[:, :2], q, ptr, ptr, (1, 2, 2)), (q, q, q, ptr, ptr, (1, 2, 2))):   # (the last: no device tensors)
        with pytest.raises(ValueError):
            B.psa_attn_fwd_lists(*args, (1, 16, 16), 0.1)
