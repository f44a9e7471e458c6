"""Norm and three-axis rotation of queries and keys, and their gradient, against the definition in 64 bits.

Tolerances count roundings (u = 2^-24, half a step of fp32): the output's own half step relative to the value, and for the
32-bit arithmetic a number of u of the magnitudes that meet in a value.  Forward: the mean of squares goes through at most 8 *
4 (channels and heads of a lane) + 4 (lanes) + 12 (half warps of a token) additions, which the root halves, the root itself is off
by 4 u, weight and norm multiply 2 more, cos and sin are off by 4 u (fraction of a turn, function), a rotation rounds 3 times:
under 24 + 4 + 2 + 4 + 3 < 40.  Gradient: the rotation (7), the same root three times over (3 * 28), the mean of h * x (48 + 9)
and 4 more operations: under 160.  A weight's sum over n tokens and heads: at most n additions of terms that are off by 40 u.
"""
import math

import pytest
import torch

from paper_2609_37001_b200 import binding as B

U = 2.0 ** -24
THETA, EPS = 10000.0, 1e-6
WIDE_TIME, WIDE_SPACE, PART = (44, 42, 42), (16, 56, 56), (16, 24, 24)


def _half_step(dtype):
    return torch.finfo(dtype).eps / 2


def _turns(grid, dims, origin, step, first, tokens, theta=THETA):
    """Angles [tokens, pairs] in 64 bits; text tokens: 0."""
    T, H, W = grid
    angle = torch.zeros((tokens, sum(dims) // 2), dtype=torch.float64)
    for n in range(tokens):
        i = first + n
        if i >= T * H * W:
            continue
        p = 0
        for axis, index in enumerate((i // (H * W), i // W % H, i % W)):
            for j in range(dims[axis] // 2):
                angle[n, p] = (origin[axis] + step[axis] * index) * theta ** (-2.0 * j / dims[axis])
                p += 1
    return angle


def _pair(n, pairs):
    return (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if pairs == "interleaved" else (slice(0, n), slice(n, 2 * n))


def _rotate(x, angle, pairs):
    a, b = _pair(angle.shape[1], pairs)
    y = x.clone()
    y[..., a] = x[..., a] * angle.cos() - x[..., b] * angle.sin()
    y[..., b] = x[..., a] * angle.sin() + x[..., b] * angle.cos()
    return y


def _met(x, n, pairs):
    """Magnitudes that meet in a rotated value: |a| + |b| of its pair."""
    a, b = _pair(n, pairs)
    y = x.abs().clone()
    y[..., a] = y[..., b] = x[..., a].abs() + x[..., b].abs()
    return y


def _root(x, norm, eps):
    if norm == "none":
        return torch.ones_like(x[..., :1])
    mean = x.square().mean(-1, keepdim=True) if norm == "head" else x.square().mean((-3, -1), keepdim=True)
    return 1.0 / (mean + eps).sqrt()


def _weight(w):
    return torch.ones((), dtype=torch.float64) if w is None else (w.double() if w.dim() == 1 else w.double()[:, None, :])


def _make(shape, dtype, layout, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = (scale * torch.randn(shape, generator=g)).to(dtype)
    if layout == "head":
        return x.cuda()
    if layout == "token":
        return x.transpose(-3, -2).contiguous().cuda().transpose(-3, -2)
    *b, h, n, d = shape   # fused: the middle one of three
    buf = torch.zeros((*b, n, 3, h, d), dtype=dtype, device="cuda")
    view = buf[..., 1, :, :].transpose(-3, -2)
    view.copy_(x)
    return view


# type, out type, heads, batch, grid, text, (first, tokens), norm, weights, dims, pairs, layout, origin, step
CASES = [
    (torch.bfloat16, torch.bfloat16, 2, 0, (2, 3, 5), 0, None, "head", "shared", WIDE_TIME, "interleaved", "head", (0, 0, 0), (1, 1, 1)),
    (torch.bfloat16, torch.bfloat16, 12, 2, (3, 5, 7), 9, None, "token", "heads", WIDE_TIME, "interleaved", "token", (0, 0, 0), (1, 1, 1)),
    (torch.float16, torch.float16, 5, 0, (4, 3, 11), 0, None, "none", None, WIDE_SPACE, "halves", "fused", (250000, -17, 3), (0.5, 1.25, 1)),
    (torch.float32, torch.float32, 3, 2, (2, 7, 9), 3, None, "head", "heads", PART, "halves", "head", (17, 0, 0), (1, 1, 1)),
    (torch.float32, torch.bfloat16, 40, 0, (1, 4, 6), 2, None, "token", "shared", PART, "interleaved", "token", (0, 0, 0), (1, 1, 1)),
    (torch.float16, torch.bfloat16, 33, 3, (1, 3, 4), 0, None, "token", None, WIDE_TIME, "halves", "head", (0, 0, 0), (1, 1, 1)),
    (torch.bfloat16, torch.bfloat16, 128, 0, (1, 1, 3), 1, None, "token", "heads", (2, 0, 4), "interleaved", "head", (5, 5, 5), (2, 2, 2)),
    (torch.bfloat16, torch.bfloat16, 1, 0, (1, 1, 1), 0, None, "head", None, WIDE_TIME, "interleaved", "head", (0, 0, 0), (1, 1, 1)),
    (torch.bfloat16, torch.bfloat16, 7, 2, (3, 4, 5), 20, (37, 41), "head", "shared", WIDE_SPACE, "interleaved", "fused", (0, 0, 0), (1, 1, 1)),
    (torch.float32, torch.float32, 2, 0, (5, 20, 31), 0, (1000, 1), "none", None, (128, 0, 0), "interleaved", "head", (1e6, 0, 0), (1, 1, 1)),
    (torch.bfloat16, torch.bfloat16, 24, 0, (5, 20, 31), 0, None, "head", "shared", (0, 0, 0), "halves", "head", (0, 0, 0), (1, 1, 1)),
    (torch.bfloat16, torch.bfloat16, 56, 0, (2, 4, 41), 0, None, "token", "heads", WIDE_TIME, "interleaved", "head", (0, 0, 0), (1, 1, 1)),
    (torch.float32, torch.float32, 57, 0, (2, 4, 41), 0, None, "token", "heads", WIDE_SPACE, "halves", "head", (0, 0, 0), (1, 1, 1)),
    (torch.float16, torch.float16, 64, 2, (2, 4, 21), 1, None, "head", "shared", WIDE_TIME, "interleaved", "token", (0, 0, 0), (1, 1, 1)),
    (torch.bfloat16, torch.bfloat16, 65, 0, (2, 4, 41), 0, None, "token", "heads", WIDE_TIME, "interleaved", "head", (0, 0, 0), (1, 1, 1)),
    (torch.bfloat16, torch.bfloat16, 3, 3000, (1, 1, 2), 0, (1, 1), "head", "heads", WIDE_TIME, "interleaved", "token", (0, 0, 0), (1, 1, 1)),
    (torch.bfloat16, torch.bfloat16, 20, 700, (1, 1, 3), 0, None, "token", "shared", WIDE_TIME, "interleaved", "head", (0, 0, 0), (1, 1, 1)),
    (torch.float32, torch.float32, 128, 0, (1, 13, 31), 5, None, "token", "heads", WIDE_TIME, "interleaved", "head", (0, 0, 0), (1, 1, 1)),
    (torch.float32, torch.float32, 127, 2, (1, 3, 71), 0, None, "head", "heads", PART, "halves", "token", (0, 0, 0), (1, 1, 1)),
    (torch.bfloat16, torch.bfloat16, 17, 0, (3, 20, 31), 40, None, "token", "heads", WIDE_TIME, "interleaved", "head", (0, 0, 0), (1, 1, 1)),
]


def _problem(case):
    dt, odt, heads, batch, grid, text, part, norm, weights, dims, pairs, layout, origin, step = case
    first, tokens = part or (0, grid[0] * grid[1] * grid[2] + text)
    shape = ((batch,) if batch else ()) + (heads, tokens, 128)
    q, k = (_make(shape, dt, layout, seed) for seed in (1, 2))
    q_out_grad, k_out_grad = (_make(shape, odt, "token" if layout == "head" else "head", seed) for seed in (3, 4))
    wdt = {torch.float16: torch.float16, torch.bfloat16: torch.bfloat16}.get(dt, torch.float32) if heads % 2 else torch.float32
    wshape = {"shared": (128,), "heads": (heads, 128)}.get(weights)
    qw, kw = (None if wshape is None else (1.0 + 0.3 * torch.randn(wshape, generator=torch.Generator().manual_seed(s))).to(wdt).cuda() for s in (5, 6))
    how = dict(dims=dims, theta=THETA, norm=norm, q_weight=qw, k_weight=kw, eps=EPS, pairs=pairs, origin=origin, step=step, n_text=text, first_token=first)
    return (q, k), (q_out_grad, k_out_grad), (qw, kw), _turns(grid, dims, origin, step, first, tokens), how


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%dx%s-%s-%s" % (str(c[0])[6:], c[2], "x".join(map(str, c[4])), c[7], c[10]))
def test_forward(case):
    x, _, w, angle, how = _problem(case)
    got = B.psa_qk_norm_rope(*x, case[4], out_dtype=case[1], **how)
    for y, x, w in zip(got, x, w):
        assert y.shape == x.shape and y.dtype == case[1]
        xd, wd = x.cpu().double(), _weight(None if w is None else w.cpu())
        u = xd * _root(xd, how["norm"], EPS) * wd
        want = _rotate(u, angle, how["pairs"])
        off = (y.cpu().double() - want).abs()
        limit = _half_step(case[1]) * want.abs() + 40 * U * _met(u, angle.shape[1], how["pairs"]) + torch.finfo(case[1]).tiny * _half_step(case[1]) * 2
        assert (off <= limit).all(), (off / limit).max()


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%dx%s-%s-%s" % (str(c[0])[6:], c[2], "x".join(map(str, c[4])), c[7], c[10]))
def test_gradient(case):
    """Against the gradient's formula in 64 bits (which test_formula_is_the_gradient holds against differences)."""
    x, dy, w, angle, how = _problem(case)
    got = B.psa_qk_norm_rope_bwd(*dy, *x, case[4], **how)
    again = B.psa_qk_norm_rope_bwd(*dy, *x, case[4], **how)
    for a, b in zip(got, again):   # sums in a fixed order
        assert (a is None and b is None) or torch.equal(a, b)
    for i in (0, 1):
        xd, gd = x[i].cpu().double(), dy[i].cpu().double()
        dx, dw, met, dw_met = _formula(xd, None if w[i] is None else w[i].cpu(), gd, angle, how)
        off = (got[i].cpu().double() - dx).abs()
        limit = _half_step(case[0]) * dx.abs() + 160 * U * met + torch.finfo(case[0]).tiny * _half_step(case[0]) * 2
        assert got[i].dtype == case[0] and (off <= limit).all(), (off / limit).max()
        if w[i] is None:
            assert got[2 + i] is None
            continue
        terms = xd.numel() / w[i].numel()
        assert got[2 + i].dtype == torch.float32 and got[2 + i].shape == w[i].shape
        off = (got[2 + i].cpu().double() - dw).abs()
        assert (off <= (terms + 40) * U * dw_met).all()


def _formula(x, w, dy, angle, how):
    """dx, dw, and the magnitudes that meet in them."""
    norm, pairs, wd = how["norm"], how["pairs"], _weight(w)
    g = _rotate(dy, -angle, pairs)
    g_met = _met(dy, angle.shape[1], pairs)
    if norm == "none":
        return g, None, g_met, None
    r = _root(x, norm, EPS)
    axes = (-1,) if norm == "head" else (-3, -1)
    h = g * wd
    dx = r * (h - x * r * r * (h * x).mean(axes, keepdim=True))
    met = r * (g_met * wd.abs() + x.abs() * r * r * (g_met * wd.abs() * x.abs()).mean(axes, keepdim=True))
    dw, dw_met = g * x * r, g_met * x.abs() * r
    if w is not None:
        over = tuple(i for i in range(x.dim() - 1) if w.dim() == 1 or i != x.dim() - 3)
        dw, dw_met = dw.sum(over), dw_met.sum(over)
    return dx, dw, met, dw_met


@pytest.mark.parametrize("norm,pairs,weights", [("head", "interleaved", 1), ("token", "halves", 2), ("none", "halves", 0), ("token", "interleaved", 1)])
def test_formula_is_the_gradient(norm, pairs, weights):
    """The formula that the kernels are tested against, against central differences (no GPU)."""
    g = torch.Generator().manual_seed(7)
    grid, dims = (2, 2, 3), (8, 16, 8)
    x, dy, dx, dw = (torch.randn((3, 14, 128), generator=g, dtype=torch.float64) for _ in range(4))
    w = None if weights == 0 else 1.0 + 0.3 * torch.randn((128,) if weights == 1 else (3, 128), generator=g, dtype=torch.float64)
    dw = None if w is None else torch.randn(w.shape, generator=g, dtype=torch.float64)
    angle = _turns(grid, dims, (3, 1, 0), (1, 0.5, 2), 0, 14)
    how = dict(norm=norm, pairs=pairs)

    def y(x, w):
        return (_rotate(x * _root(x, norm, EPS) * _weight(w), angle, pairs) * dy).sum()

    gx, gw, _, _ = _formula(x, w, dy, angle, how)
    h = 1e-5
    slope = (y(x + h * dx, w) - y(x - h * dx, w)) / (2 * h)
    assert math.isclose(float((gx * dx).sum()), float(slope), rel_tol=1e-7, abs_tol=1e-7)
    if w is not None:
        slope = (y(x, w + h * dw) - y(x, w - h * dw)) / (2 * h)
        assert math.isclose(float((gw * dw).sum()), float(slope), rel_tol=1e-7, abs_tol=1e-7)


@pytest.mark.gpu
def test_differences_of_the_kernels():
    """The gradient kernel against differences of the forward kernel, fp32."""
    grid, shape = (2, 3, 4), (3, 24, 128)
    how = dict(dims=PART, norm="token", pairs="halves", origin=(9, 0, 0))
    x, dx, dy = (_make(shape, torch.float32, "head", s) for s in (1, 2, 3))
    w = (1.0 + 0.3 * torch.randn((3, 128), generator=torch.Generator().manual_seed(4))).cuda()
    dq, _, dw, _ = B.psa_qk_norm_rope_bwd(dy, None, x, None, grid, q_weight=w, **how)
    h = 2.0 ** -6

    def value(t):
        return (B.psa_qk_norm_rope(x + t * dx, None, grid, q_weight=w, **how)[0].double() * dy.double()).sum()

    # second-order error h^2 / 6 of a third derivative that is of the order of the slopes of 9216 unit terms; fp32 rounding 9216^.5 u / h
    slope = (value(h) - value(-h)) / (2 * h)
    assert abs(float((dq.double() * dx.double()).sum() - slope)) <= 9216 ** 0.5 * h * h + 9216 * U / h
    q1 = B.psa_qk_norm_rope(x, None, grid, q_weight=w + h, **how)[0].double()
    q0 = B.psa_qk_norm_rope(x, None, grid, q_weight=w - h, **how)[0].double()
    slope = ((q1 - q0) * dy.double()).sum() / (2 * h)   # linear in the weights
    assert abs(float(dw.double().sum() - slope)) <= 9216 * 40 * U / h


@pytest.mark.gpu
def test_in_place_parts_and_layouts_agree():
    """In place, token by token, k alone or q alone, padded strides, and another stream: the same bits."""
    grid, text, heads = (3, 4, 5), 7, 6
    n = 67
    how = dict(dims=WIDE_TIME, norm="token", n_text=text)
    q, k = (_make((heads, n, 128), torch.bfloat16, "head", s) for s in (1, 2))
    qw, kw = (torch.randn((heads, 128), device="cuda", generator=torch.Generator(device="cuda").manual_seed(s)) for s in (1, 2))
    want = B.psa_qk_norm_rope(q, k, grid, q_weight=qw, k_weight=kw, **how)
    alone = B.psa_qk_norm_rope(k, None, grid, q_weight=kw, **how)
    assert alone[1] is None and torch.equal(alone[0], want[1])
    for first in range(0, n, 13):
        part = [x[:, first:first + 13] for x in (q, k)]
        got = B.psa_qk_norm_rope(*part, grid, q_weight=qw, k_weight=kw, first_token=first, **how)
        assert all(torch.equal(a, b[:, first:first + 13]) for a, b in zip(got, want))
    wide = [torch.full((heads, n + 3, 136), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    out = [x[:, 1:n + 1, :128] for x in wide]
    B.psa_qk_norm_rope(q, k, grid, q_weight=qw, k_weight=kw, out=out, **how)
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    for x in wide:   # what lies around the tokens is left as it was
        x[:, 1:n + 1, :128] = 9.0
        assert (x == 9.0).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = B.psa_qk_norm_rope(q, k, grid, q_weight=qw, k_weight=kw, stream=side, **how)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    q1, k1 = q.clone(), k.clone()
    got = B.psa_qk_norm_rope(q1, k1, grid, q_weight=qw, k_weight=kw, out=(q1, k1), **how)
    assert got[0] is q1 and torch.equal(q1, want[0]) and torch.equal(k1, want[1])


@pytest.mark.gpu
def test_captured_and_replayed():
    grid, heads = (2, 5, 7), 3
    q, k, dq, dk = (_make((heads, 70, 128), torch.bfloat16, "head", s) for s in (1, 2, 3, 4))
    w = torch.randn(128, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    how = dict(q_weight=w, k_weight=w)
    graph = torch.cuda.CUDAGraph()
    B.psa_qk_norm_rope(q, k, grid, **how)
    with torch.cuda.graph(graph):
        y = B.psa_qk_norm_rope(q, k, grid, **how)
        d = B.psa_qk_norm_rope_bwd(dq, dk, q, k, grid, **how)
    for s in (11, 12):
        q.copy_(_make((heads, 70, 128), torch.bfloat16, "head", s))
        graph.replay()
        want = (*B.psa_qk_norm_rope(q, k, grid, **how), *B.psa_qk_norm_rope_bwd(dq, dk, q, k, grid, **how))
        assert all(torch.equal(a, b) for a, b in zip((*y, *d), want))


@pytest.mark.gpu
def test_values_that_are_not_finite_stay_in_their_rows():
    grid, heads = (1, 2, 4), 3
    q = _make((heads, 8, 128), torch.bfloat16, "head", 1)
    want = B.psa_qk_norm_rope(q, None, grid, norm="head")[0]
    bad = q.clone()
    bad[1, 3, 5], bad[2, 7, 0] = math.inf, math.nan
    got = B.psa_qk_norm_rope(bad, None, grid, norm="head")[0]
    rows = torch.ones((heads, 8), dtype=torch.bool, device="cuda")
    rows[1, 3] = rows[2, 7] = False
    assert torch.equal(got[rows], want[rows]) and got[~rows].isnan().any(1).all()
    # rotation alone: within the pair; channels that are not rotated keep theirs
    got = B.psa_qk_norm_rope(bad, None, grid, dims=(2, 0, 0), norm="none")[0]
    assert got[1, 3, 5] == math.inf and torch.equal(got[1, 3, 6:], bad[1, 3, 6:])
    # zeros with eps 0 in one token: that token's rows only
    zero = q.clone()
    zero[:, 2] = 0
    got = B.psa_qk_norm_rope(zero, None, grid, norm="token", eps=0.0)[0]
    assert got[:, 2].isnan().all() and not got[:, [0, 1, 3, 4, 5, 6, 7]].isnan().any()


@pytest.mark.gpu
def test_no_tokens():
    q = torch.empty((2, 0, 128), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(128, device="cuda")
    y, _ = B.psa_qk_norm_rope(q, q, (1, 2, 2), q_weight=w, k_weight=w, first_token=4)
    assert y.shape == q.shape
    _, _, dw, _ = B.psa_qk_norm_rope_bwd(q, q, q, q, (1, 2, 2), q_weight=w, k_weight=w)
    assert (dw == 0).all()


def _args(**over):
    a = dict(n_batch=1, n_heads=2, head_dim=128, dtype=0, out_dtype=0, norm=1, weight_dtype=2, weight_heads=1, eps=1e-6, n_tokens=4, first=0, text=0,
             stride=(0, 512, 128), out_stride=(0, 512, 128), grad_stride=(0, 512, 128), dims=(44, 42, 42), pairs=0, theta=1e4, origin=(0, 0, 0),
             step=(1, 1, 1), grid=(1, 2, 2), q=4096, k=8192, q_out=16384, k_out=32768, qw=65536, kw=65536)
    assert not set(over) - set(a)
    a.update(over)
    prob = B._pack_qk(a["n_batch"], a["n_heads"], a["head_dim"], a["dtype"], a["out_dtype"], a["norm"], a["weight_dtype"], a["weight_heads"], a["eps"], 0,
                      a["n_tokens"], a["first"], a["text"], *a["stride"], *a["out_stride"], *a["grad_stride"])
    rope = B._pack_rope(*a["dims"], a["pairs"], a["theta"], *a["origin"], *a["step"])
    return a, prob, rope


INVALID, UNSUPPORTED = B.PSA_ERR_INVALID_ARG, B.PSA_ERR_UNSUPPORTED
REFUSED = [
    (dict(grid=(0, 2, 2)), INVALID), (dict(grid=(1 << 16, 1 << 15, 1)), INVALID), (dict(n_heads=0), INVALID), (dict(n_batch=0), INVALID),
    (dict(head_dim=64), UNSUPPORTED), (dict(n_heads=129), UNSUPPORTED), (dict(n_tokens=5), INVALID), (dict(first=1), INVALID), (dict(first=-1), INVALID),
    (dict(text=-1), INVALID), (dict(n_tokens=-1), INVALID), (dict(dtype=3), INVALID), (dict(out_dtype=1), UNSUPPORTED), (dict(dtype=1, out_dtype=2), UNSUPPORTED),
    (dict(norm=3), INVALID), (dict(norm=0), INVALID), (dict(weight_heads=3), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=math.nan), INVALID),
    (dict(dims=(43, 42, 42)), INVALID), (dict(dims=(64, 64, 2)), INVALID), (dict(dims=(-2, 4, 4)), INVALID), (dict(pairs=2), INVALID),
    (dict(pairs=1, dims=(2, 4, 4)), UNSUPPORTED), (dict(theta=0.0), INVALID), (dict(theta=math.inf), INVALID), (dict(origin=(math.nan, 0, 0)), INVALID),
    (dict(step=(1, math.inf, 1)), INVALID), (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(k_out=None), INVALID), (dict(q=4104), INVALID),
    (dict(q_out=16392), INVALID), (dict(qw=65540), INVALID), (dict(stride=(0, 512, 132)), INVALID), (dict(stride=(0, 512, 0)), INVALID),
    (dict(stride=(0, 0, 128)), INVALID), (dict(n_batch=2), INVALID), (dict(out_stride=(0, 508, 128)), INVALID),
    (dict(k_out=16384), INVALID), (dict(k_out=4096), INVALID), (dict(q_out=8192), INVALID), (dict(q_out=4096, out_stride=(0, 1024, 128)), INVALID), (dict(k_out=8192, dtype=2), INVALID), (dict(k=None, k_out=None), INVALID),
]


@pytest.mark.parametrize("over,status", REFUSED, ids=lambda x: "-".join(x) if isinstance(x, dict) else "")
def test_refusals(over, status):
    a, prob, rope = _args(**over)
    got = B.lib().psa_qk_norm_rope(a["q"], a["k"], a["q_out"], a["k_out"], a["qw"], a["kw"], prob, rope, *a["grid"], None)
    assert got == status


@pytest.mark.parametrize("change", ["scratch", "one_dw", "alias", "same", "no_q", "grad_stride", "dw_align", "none_with_weight"])
def test_gradient_refusals(change):
    a, prob, rope = _args(**{"grad_stride": dict(grad_stride=(0, 512, 4)), "none_with_weight": dict(norm=0)}.get(change, {}))
    p = dict(dqo=4096, dko=8192, q=1 << 14, k=1 << 15, dq=1 << 16, dk=1 << 17, qw=1 << 18, kw=1 << 18, dqw=1 << 19, dkw=1 << 20, scratch=1 << 21)
    p.update({"scratch": dict(scratch=None), "one_dw": dict(dkw=None), "alias": dict(dq=1 << 14), "same": dict(dk=1 << 16), "no_q": dict(q=None),
              "dw_align": dict(dqw=(1 << 19) + 2)}.get(change, {}))
    got = B.lib().psa_qk_norm_rope_bwd(p["dqo"], p["dko"], p["q"], p["k"], p["dq"], p["dk"], p["qw"], p["kw"], p["dqw"], p["dkw"], prob, rope, *a["grid"],
                                       p["scratch"], None)
    assert got == INVALID


def test_binding_refusals():
    q = torch.zeros((2, 4, 128), dtype=torch.bfloat16)
    for bad in (dict(norm="rms"), dict(pairs="odd"), dict(norm="none", q_weight=torch.ones(128)), dict(q_weight=torch.ones(64), k_weight=torch.ones(64)),
                dict(q_weight=torch.ones(128)), dict(out=(q,)), {}):   # (the last one: no device tensors)
        with pytest.raises(ValueError):
            B.psa_qk_norm_rope(q, q.clone(), (1, 2, 2), **bad)
    with pytest.raises(ValueError):
        B.psa_qk_norm_rope(q, q.float(), (1, 2, 2))
    with pytest.raises(ValueError):
        B.psa_qk_norm_rope(q.transpose(1, 2), None, (1, 2, 2))
    with pytest.raises(ValueError):
        B.psa_qk_norm_rope_bwd(q, None, None, None, (1, 2, 2))
