"""Weight gradients over many tokens: every token, head and block is in the sum, once.

Whole numbers: x of +-1 has the root mean square 1, dy is a small whole number and nothing turns, so that every term and every sum, below
2^24, is exact in 32 bits in whatever order.  Values in general: a thread adds up its tokens (at least half as many blocks run as there are
SMs, or a block has one set of tokens; a set is of 64 threads at least, 8 a head and tensor, so of 4 tokens for one head and 2 for two), the block adds up its
tokens and, for a shared weight, its heads (8 or as many as there are heads, and one more where a thread has two heads), the sum over blocks is in 64 bits
and rounds once.  Every term is off
by 40 roundings (root and rotation: see the forward pass)."""
import pytest
import torch

from paper_2609_37001_b200 import binding as B
from test_norm_rope import U, WIDE_TIME, _formula, _turns

# type, heads, batch, tokens, norm, weight a head
CASES = [
    (torch.bfloat16, 24, 1, 3100, "head", False), (torch.bfloat16, 20, 700, 3, "token", False), (torch.float32, 1, 1, 50001, "head", False),
    (torch.bfloat16, 12, 2, 2501, "head", True), (torch.float16, 12, 2, 2501, "token", False), (torch.bfloat16, 40, 1, 1999, "token", True),
    (torch.float32, 57, 1, 611, "token", False), (torch.bfloat16, 64, 1, 777, "head", False), (torch.bfloat16, 65, 1, 777, "token", True),
    (torch.bfloat16, 127, 1, 500, "head", False), (torch.float32, 128, 3, 167, "token", False), (torch.float16, 128, 1, 500, "token", True),
    (torch.bfloat16, 3, 1, 4001, "head", False), (torch.bfloat16, 8, 1, 3000, "token", True), (torch.bfloat16, 9, 1, 3000, "token", False),
]
ids = [("%s-%d-%dx%d-%s-%s" % (str(c[0])[6:], c[1], c[2], c[3], c[4], "each" if c[5] else "shared")) for c in CASES]


def _call(x, dy, w, grid, two, **how):
    with_k = (dy[1], x[0], x[1]) if two else (None, x[0], None)
    return B.psa_qk_norm_rope_bwd(dy[0], *with_k, grid, q_weight=w, k_weight=w if two else None, **how)[2:]


@pytest.mark.gpu
@pytest.mark.parametrize("two", [True, False], ids=["qk", "q"])
@pytest.mark.parametrize("case", CASES, ids=ids)
def test_whole_numbers(case, two):
    dtype, heads, batch, tokens, norm, each = case
    g = torch.Generator(device="cuda").manual_seed(heads + tokens)
    shape = (batch, heads, tokens, 128)
    x = [(torch.randint(0, 2, shape, device="cuda", generator=g) * 2 - 1).to(dtype) for _ in range(2)]
    dy = [torch.randint(-2, 3, shape, device="cuda", generator=g).to(dtype) for _ in range(2)]
    w = torch.full((heads, 128) if each else (128,), 1.5, device="cuda")
    got = _call(x, dy, w, (1, 1, tokens), two, dims=(0, 0, 0), norm=norm, eps=0.0)
    for i in range(2 if two else 1):
        terms = (x[i].double() * dy[i].double())
        assert (terms != 0).any(-1).all()   # a row left out or taken twice shows
        want = terms.sum((0, 2) if each else (0, 1, 2))
        assert want.abs().max() < 2 ** 24 and torch.equal(got[i].double(), want)
    assert two or got[1] is None


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=ids)
def test_values_in_general(case):
    dtype, heads, batch, tokens, norm, each = case
    g = torch.Generator(device="cuda").manual_seed(heads + tokens + 1)
    shape = (batch, heads, tokens, 128)
    x, dy = ([torch.randn(shape, device="cuda", generator=g).to(dtype) for _ in range(2)] for _ in range(2))
    w = 1 + 0.3 * torch.randn((heads, 128) if each else (128,), device="cuda", generator=g)
    grid = (1, 1, tokens)
    got = _call(x, dy, w, grid, True, dims=WIDE_TIME, norm=norm, eps=1e-6)
    angle = _turns(grid, WIDE_TIME, (0, 0, 0), (1, 1, 1), 0, tokens).cuda()
    blocks = torch.cuda.get_device_properties(0).multi_processor_count // 2
    depth = -(-batch * tokens // (blocks * max(1, 4 // heads))) + heads + 9
    over = (0, 2) if each else (0, 1, 2)
    for i in range(2):
        how = dict(norm=norm, pairs="interleaved")
        _, terms, _, met = _formula(x[i].double(), None, dy[i].double(), angle, how)   # (terms of dw do not depend on the weights)
        off = (got[i].double() - terms.sum(over)).abs()
        limit = (depth + 40) * U * met.sum(over) + U * terms.sum(over).abs()
        assert (off <= limit).all(), float((off / limit).max())
        # a definition that leaves out the last token, or the first head's, is told apart
        assert (terms[-1:, :, -1:].sum(over).abs() > 2 * limit).any()
        if not each and heads > 1:
            assert (terms[:, :1].sum(over).abs() > 2 * limit).any()
