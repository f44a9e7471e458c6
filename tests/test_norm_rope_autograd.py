"""psa_qk_norm_rope where a gradient is required: autograd gets the one of psa_qk_norm_rope_bwd, whatever the gradients of the outputs look like."""
import pytest
import torch

from paper_2609_37001_b200 import binding as B
from test_norm_rope import EPS, THETA, WIDE_SPACE, WIDE_TIME, _formula, _make, _root, _rotate, _turns, _weight

GRID, TEXT, HEADS = (2, 3, 4), 3, 5
TOKENS = 27


# ------------------------------------------------------------------------------------- on the CPU, plain functions for the kernels
def _plain(q, k, grid, q_weight=None, k_weight=None, out_dtype=None, norm="head", pairs="interleaved", dims=(4, 8, 4), n_text=0, **how):
    assert not torch.is_grad_enabled()
    angle = _turns(grid, dims, (1, 0, 2), (1, 1, 1), 0, q.shape[-2])
    return tuple(None if x is None else _rotate(x * _root(x, norm, EPS) * _weight(w), angle, pairs) for x, w in ((q, q_weight), (k, k_weight)))


def _plain_bwd(dq_out, dk_out, q, k, grid, q_weight=None, k_weight=None, norm="head", pairs="interleaved", dims=(4, 8, 4), n_text=0, **how):
    assert dk_out is None or dk_out.stride() == dq_out.stride()
    assert all(B._as_it_lies(g) for g in (dq_out, dk_out) if g is not None)
    angle = _turns(grid, dims, (1, 0, 2), (1, 1, 1), 0, dq_out.shape[-2])
    got = [(None, None) if g is None else _formula(torch.empty(0) if x is None else x, w, g, angle, dict(norm=norm, pairs=pairs))[:2]
           for x, w, g in ((q, q_weight, dq_out), (k, k_weight, dk_out))]
    return got[0][0], got[1][0], None if q_weight is None else got[0][1], None if k_weight is None else got[1][1]


@pytest.mark.parametrize("norm,pairs,weights,two", [("head", "interleaved", 1, True), ("token", "halves", 2, True), ("none", "halves", 0, True),
                                                    ("token", "interleaved", 0, False), ("head", "halves", 2, False)])
def test_against_differences(monkeypatch, norm, pairs, weights, two):
    apply = B._NormRope.apply
    monkeypatch.setattr(B, "psa_qk_norm_rope", _plain)
    monkeypatch.setattr(B, "psa_qk_norm_rope_bwd", _plain_bwd)
    g = torch.Generator().manual_seed(1)
    q, k = (torch.randn((2, 6, 128), generator=g, dtype=torch.float64).requires_grad_() for _ in range(2))
    shape = {0: None, 1: (128,), 2: (2, 128)}[weights]
    qw, kw = (None if shape is None else (1 + 0.3 * torch.randn(shape, generator=g, dtype=torch.float64)).requires_grad_() for _ in range(2))
    if not two:
        k = kw = None
    leaves = [x for x in (q, k, qw, kw) if x is not None]

    def call(*leaves):
        got = iter(leaves)
        q, k, qw, kw = (None if x is None else next(got) for x in (q0, k0, qw0, kw0))
        return tuple(y for y in apply(q, k, qw, kw, (1, 2, 2), None, dict(norm=norm, pairs=pairs, stream=None)) if y is not None)

    q0, k0, qw0, kw0 = q, k, qw, kw
    assert torch.autograd.gradcheck(call, leaves, fast_mode=True)


def test_the_head_sharded_call_keeps_no_graph():
    """Attention behind it is forward only."""
    from paper_2609_37001_b200 import ulysses as U
    from test_ulysses_gloo import GRID, PARAMS, SCALE, TILE, _full_inputs, _oracle_attn
    q, k, v = _full_inputs()
    w = torch.ones(q.shape[-1], dtype=q.dtype).requires_grad_()
    seen = []

    def attn_fn(q, k, *more):
        seen.append(q.requires_grad or k.requires_grad)
        return _oracle_attn(q, k, *more)

    U.psa_attn_fwd_ulysses(q, k, v, PARAMS, GRID, TILE, SCALE, attn_fn=attn_fn, norm_rope=dict(q_weight=w),
                           norm_rope_fn=lambda q, k, grid, first_token, q_weight: (q * q_weight, k * q_weight))
    assert seen == [False]


# ------------------------------------------------------------------------------------- the kernels
# type, out type, norm, weights, weight type, pairs, dims, layout, two
CASES = [
    (torch.bfloat16, None, "token", (HEADS, 128), torch.float32, "interleaved", WIDE_TIME, "fused", True),
    (torch.float32, None, "head", (128,), torch.float32, "halves", WIDE_SPACE, "head", True),
    (torch.float32, torch.bfloat16, "none", None, None, "interleaved", WIDE_TIME, "token", True),
    (torch.float16, None, "none", None, None, "halves", WIDE_SPACE, "head", True),
    (torch.bfloat16, None, "head", (128,), torch.bfloat16, "interleaved", WIDE_TIME, "token", False),
    (torch.float16, torch.bfloat16, "token", None, None, "interleaved", WIDE_TIME, "head", True),
]


def _case(case, seed=1):
    dt, odt, norm, shape, wdt, pairs, dims, layout, two = case
    q, k = (_make((HEADS, TOKENS, 128), dt, layout, seed + i).detach().requires_grad_() for i in range(2))
    g = torch.Generator().manual_seed(seed + 5)
    qw, kw = (None if shape is None else (1 + 0.3 * torch.randn(shape, generator=g)).to(wdt).cuda().requires_grad_() for _ in range(2))
    if not two:
        k = kw = None
    how = dict(dims=dims, norm=norm, pairs=pairs, n_text=TEXT, q_weight=qw, k_weight=kw)
    dq, dk = (_make((HEADS, TOKENS, 128), odt or dt, "head", seed + 7 + i) for i in range(2))
    return q, k, how, odt, dq, dk if two else None


def _direct(q, k, how, dq, dk):
    with torch.no_grad():
        got = B.psa_qk_norm_rope_bwd(dq, dk, q, k, GRID, **how)
    return [None if x is None else x.to(y.dtype) for x, y in zip(got, (q, k, how["q_weight"], how["k_weight"]))]


def _leaves(q, k, how):
    return q, k, how["q_weight"], how["k_weight"]


def _same(leaves, want):
    for x, g in zip(leaves, want):
        if x is not None:
            assert x.grad.dtype == x.dtype and torch.equal(x.grad, g)


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%s-%s" % (str(c[0])[6:], c[2], c[5]))
def test_gradients_are_those_of_the_call(case):
    q, k, how, odt, dq, dk = _case(case)
    got = B.psa_qk_norm_rope(q, k, GRID, out_dtype=odt, **how)
    with torch.no_grad():
        want = B.psa_qk_norm_rope(q, k, GRID, out_dtype=odt, **how)
    for a, b in zip(got, want):
        assert (a is None and b is None) or (a.requires_grad and not b.requires_grad and torch.equal(a, b) and a.stride() == b.stride())
    torch.autograd.backward([y for y in got if y is not None], [g for g in (dq, dk) if g is not None])
    _same(_leaves(q, k, how), _direct(q, k, how, dq, dk))


@pytest.mark.gpu
def test_against_the_formula():
    """The whole way, from a projection's q and k to its gradient, against autograd in 64 bits."""
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn((TOKENS, 3, HEADS, 128), generator=g).cuda().requires_grad_()
    w = (1 + 0.3 * torch.randn((HEADS, 128), generator=g)).cuda().requires_grad_()
    dy = torch.randn((2, HEADS, TOKENS, 128), generator=g)
    q, k = (qkv[:, i].transpose(0, 1) for i in (0, 1))
    y = B.psa_qk_norm_rope(q, k, GRID, dims=WIDE_TIME, norm="token", n_text=TEXT, q_weight=w, k_weight=w)
    sum((a * b.cuda()).sum() for a, b in zip(y, dy)).backward()
    x, w64 = qkv.detach().cpu().double().requires_grad_(), w.detach().cpu().double().requires_grad_()
    angle = _turns(GRID, WIDE_TIME, (0, 0, 0), (1, 1, 1), 0, TOKENS, THETA)
    total = 0
    for i in (0, 1):
        t = x[:, i].transpose(0, 1)
        total = total + (_rotate(t * _root(t, "token", EPS) * w64[:, None], angle, "interleaved") * dy[i].double()).sum()
    total.backward()
    u = 2.0 ** -24
    assert (qkv.grad[:, 2] == 0).all()
    for i in (0, 1):   # 160 u of the magnitudes that meet, as the call itself, and the rounding to 32 bits
        _, _, met, w_met = _formula(x.detach()[:, i].transpose(0, 1), w64.detach(), dy[i].double(), angle, dict(norm="token", pairs="interleaved"))
        off = (qkv.grad[:, i].cpu().double() - x.grad[:, i]).abs().transpose(0, 1)
        assert (off <= 160 * u * met + u * x.grad[:, i].abs().transpose(0, 1)).all()
    assert ((w.grad.cpu().double() - w64.grad).abs() <= 2 * (TOKENS + 160) * u * 2 * w_met.max()).all()


@pytest.mark.gpu
def test_gradients_of_every_shape():
    """One value for all (of a sum), other strides for q than for k, an output that nothing reads."""
    case = CASES[0]
    for kind in ("sum", "strides", "one"):
        q, k, how, odt, dq, dk = _case(case, 11)
        got = B.psa_qk_norm_rope(q, k, GRID, **how)
        if kind == "sum":
            (got[0].sum() + 2 * got[1].sum()).backward()
            dq, dk = torch.ones_like(dq), torch.full_like(dk, 2.0)
        elif kind == "strides":
            torch.autograd.backward(got, (dq, dk.transpose(0, 1).contiguous().transpose(0, 1)))
        else:
            got[1].backward(dk)
            dq = torch.zeros_like(dk)
        _same(_leaves(q, k, how), _direct(q, k, how, dq, dk))


@pytest.mark.gpu
def test_on_another_stream():
    case = CASES[0]
    q, k, how, odt, dq, dk = _case(case, 13)
    want = _direct(q, k, how, dq, dk)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = B.psa_qk_norm_rope(q, k, GRID, stream=side, **how)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(20_000_000)   # the outputs' gradients are late
    torch.autograd.backward(got, [dq + 0, dk + 0])
    _same(_leaves(q, k, how), want)


@pytest.mark.gpu
def test_where_no_gradient_is_required():
    q, k, how, odt, dq, dk = _case(CASES[0])
    with torch.no_grad():
        assert not any(y.requires_grad for y in B.psa_qk_norm_rope(q, k, GRID, **how))
    plain = dict(how, q_weight=how["q_weight"].detach(), k_weight=how["k_weight"].detach())
    assert not any(y.requires_grad for y in B.psa_qk_norm_rope(q.detach(), k.detach(), GRID, **plain))
    out = (torch.empty_like(dq), torch.empty_like(dk))
    got = B.psa_qk_norm_rope(q, k, GRID, out=out, **how)
    assert got[0] is out[0] and not any(y.requires_grad for y in got)
    # weights alone, q and k alone
    for leaf in (dict(), plain):
        a, b = (q.detach(), k.detach()) if not leaf else (q, k)
        for x in _leaves(q, k, how):
            x.grad = None
        torch.autograd.backward(B.psa_qk_norm_rope(a, b, GRID, **(leaf or how)), (dq, dk))
        want = _direct(q, k, how, dq, dk)
        rows = slice(2, 4) if not leaf else slice(0, 2)
        _same(_leaves(q, k, how)[rows], want[rows])
        assert all(x.grad is None for i, x in enumerate(_leaves(q, k, how)) if not rows.start <= i < rows.stop)


@pytest.mark.gpu
def test_second_derivatives_are_refused():
    q, k, how, odt, dq, dk = _case(CASES[1])
    got = B.psa_qk_norm_rope(q, k, GRID, **how)
    first = torch.autograd.grad(got[0], q, dq, create_graph=True)[0]
    with pytest.raises(RuntimeError):
        first.sum().backward()


@pytest.mark.gpu
def test_forward_and_gradient_captured_together():
    """Leaves that no other graph knows, and gradients as results."""
    q, k, how, odt, dq, dk = _case(CASES[0], 17)
    _direct(q, k, how, dq, dk)   # (the first call on a device is not captured)
    with torch.no_grad():
        B.psa_qk_norm_rope(q, k, GRID, **how)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = torch.autograd.grad(B.psa_qk_norm_rope(q, k, GRID, **how), _leaves(q, k, how), (dq, dk))
    for s in (21, 22):
        with torch.no_grad():
            q.copy_(_make((HEADS, TOKENS, 128), torch.bfloat16, "fused", s))
        graph.replay()
        for a, b in zip(got, _direct(q, k, how, dq, dk)):
            assert torch.equal(a, b)
