"""Operators next to the stripe attention: what a layer does to its queries and keys before attention (norm and rotary positions
on the time, height and width axes, with the gradient), and attention over key blocks chosen for each query block from pooled scores.

A case names one operator ("op") and its problem.  Plain forms are elementary tensor operations; with `own` set, `run` calls the
library instead.

    listed()  the fixed cases         draw(rng)  one more of the same ranges
    prepare() inputs on the device    run()      one pass
    work()    bytes and operations a pass cannot do without
    exact()   what a pass returns, from the definition in 64 bits
"""
import math

import torch

own = False   # True: the library's operators instead of the plain forms

D = 128   # channels of a head
SCALE = 1.0 / math.sqrt(D)
THETA = 10000.0
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
# channels of a head that turn with the frame, the row and the column
DIMS = {"wide_time": (44, 42, 42), "wide_space": (16, 56, 56), "part": (16, 24, 24)}
# mask blocks that attention takes, as in perf/cases.py
TILES = [(1, 8, 16), (2, 8, 8), (1, 32, 4), (1, 16, 16), (1, 15, 16), (1, 30, 8), (2, 32, 4), (2, 8, 16), (1, 14, 16), (1, 12, 16),
         (3, 8, 16), (6, 8, 8), (3, 32, 4)]


def _case(name, op, grid, heads, **more):
    T, H, W = grid
    case = {"op": op, "T": T, "H": H, "W": W, "heads": heads, "batch": 1, "text": 0, "layout": "head"}
    if name:
        case["name"] = name
    case.update(more)
    return case


def _norm(name, op, grid, heads, **more):
    base = {"type": "bf16", "norm": "head", "weights": "shared", "dims": "wide_time", "pairs": "interleaved", "origin": 0, "step": 1.0,
            "first": 0, "tokens": 0}
    base.update(more)
    return _case(name, op, grid, heads, **base)


def _blocks_case(name, op, grid, tile, heads, keep, **more):
    bt, bh, bw = tile
    return _case(name, op, grid, heads, bt=bt, bh=bh, bw=bw, keep=keep, **more)


def listed():
    return [
        # A few latent frames, two heads: launches and host work are all there is.
        _norm("norm_rope_tiny", "norm_rope", (8, 16, 16), 2),
        # The 1.3B model at 480p: conditional and unconditional sample, norm over all heads of a token, heads interleaved.
        _norm("norm_rope_480p_cfg", "norm_rope", (21, 30, 52), 12, batch=2, norm="token", weights="heads", layout="token"),
        # A multimodal layer at 768p: 115,200 video tokens, the prompt's 256 text tokens (normed, not rotated) behind them.
        _norm("norm_rope_768p_text", "norm_rope", (30, 48, 80), 24, text=256, dims="wide_space"),
        # Rotation alone of one of eight ranks' tokens, far into a long video that is made piece by piece, channels in halves.
        _norm("rope_far_720p_shard", "norm_rope", (21, 45, 80), 40, type="fp16", norm="none", pairs="halves", origin=100_000, first=9450, tokens=9450),
        # Fine-tuning a layer: the gradient at 480p, one weight for all heads.
        _norm("norm_rope_bwd_480p", "norm_rope_bwd", (21, 30, 52), 12),
        # The same of the 14B model at 720p, as its projections leave q and k, a weight for each channel of all heads.
        _norm("norm_rope_bwd_720p", "norm_rope_bwd", (21, 45, 80), 40, norm="token", weights="heads", layout="fused"),
        # Choosing 3 of 8 blocks on a few latent frames.
        _blocks_case("select_tiny", "select", (8, 16, 16), (2, 8, 16), 2, 3),
        # One 480p layer in token layout; the last blocks along the width hold 4 of 8 columns.
        _blocks_case("select_480p", "select", (21, 30, 52), (1, 30, 8), 12, 37, layout="token"),
        # One 768p layer, 450 blocks a head.
        _blocks_case("select_768p", "select", (30, 48, 80), (1, 16, 16), 24, 112),
        # Attention over lists on a few latent frames.
        _blocks_case("lists_tiny", "lists", (8, 16, 16), (2, 8, 16), 2, 3, rows="even"),
        # One 480p layer, lists of 0 to 74 blocks (a few query blocks have none).
        _blocks_case("lists_480p_ragged", "lists", (21, 30, 52), (1, 30, 8), 12, 37, rows="ragged"),
        # The headline layer's shape with a quarter of the blocks: the largest case.
        _blocks_case("lists_720p", "lists", (21, 45, 80), (1, 15, 16), 40, 79, rows="even"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(["norm_rope", "norm_rope", "norm_rope_bwd", "select", "lists", "lists"])
        heads = _log_int(rng, 1, 40)
        if op in ("norm_rope", "norm_rope_bwd"):
            grid = (_log_int(rng, 1, 33), _log_int(rng, 1, 48), _log_int(rng, 1, 80))
            batch = rng.choice([1, 1, 2, 3])
            tokens = grid[0] * grid[1] * grid[2]
            text = rng.choice([0, 0, _log_int(rng, 1, 512)])
            if heads * (tokens + text) * batch > 3_000_000:
                continue
            norm = rng.choice(["head", "head", "token", "none"])
            case = _norm(None, op, grid, heads, batch=batch, text=text, norm=norm, type=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                         weights=rng.choice(["shared", "heads", "none"]) if norm != "none" else "none", dims=rng.choice(sorted(DIMS)),
                         pairs=rng.choice(["interleaved", "halves"]), origin=rng.choice([0, 0, 17, -3, 250_000]),
                         step=rng.choice([1.0, 1.0, 0.5, 1.25]), layout=rng.choice(["head", "token", "fused"]))
            if rng.random() < 0.3 and tokens + text > 1:   # a rank's part of the tokens
                case["tokens"] = rng.randint(1, tokens + text)
                case["first"] = rng.randint(0, tokens + text - case["tokens"])
            return case
        tile = rng.choice(TILES)
        grid = [_log_int(rng, 2, 33), _log_int(rng, 12, 48), _log_int(rng, 12, 80)]
        if rng.random() < 0.4:
            grid = [-(-x // b) * b for x, b in zip(grid, tile)]
        nb = 1
        for x, b in zip(grid, tile):
            nb *= -(-x // b)
        tokens = grid[0] * grid[1] * grid[2]
        keep = max(1, min(nb, int(round(nb * rng.choice([0.05, 0.1, 0.2, 0.3, 0.5])))))
        case = _blocks_case(None, op, tuple(grid), tile, heads, keep, layout=rng.choice(["head", "token"]))
        if op == "lists":
            case["rows"] = rng.choice(["even", "ragged"])
            case["text"] = rng.choice([0, 0, _log_int(rng, 16, 512)])
            if work(case)["flops"] > 1.0e13:
                continue
        elif heads * tokens > 2_700_000:
            continue
        return case


# ---------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _tensors(case, gen, dtype, count, tokens):
    """`count` tensors [batch, heads, tokens, D], standard normal, in the case's layout."""
    b, h = case["batch"], case["heads"]
    if case["layout"] == "fused":   # what one projection leaves: q, k and v of a token side by side
        x = torch.empty((b, tokens, 3, h, D), dtype=dtype, device="cuda")
        for part in x:
            part.normal_(generator=gen)
        return [x[:, :, i].transpose(1, 2) for i in range(count)]
    got = []
    for _ in range(count):
        shape = (b, tokens, h, D) if case["layout"] == "token" else (b, h, tokens, D)
        x = torch.empty(shape, dtype=dtype, device="cuda")
        for part in x:
            part.normal_(generator=gen)
        got.append(x.transpose(1, 2) if case["layout"] == "token" else x)
    return got


def _norm_tokens(case):
    return case["tokens"] or case["T"] * case["H"] * case["W"] + case["text"]


def _block_grid(case):
    return tuple(-(-case[x] // case[b]) for x, b in (("T", "bt"), ("H", "bh"), ("W", "bw")))


def _add_structure(x, case, gen):
    """A component that neighbouring tokens share, so that pooled scores tell blocks apart as those of a real layer do."""
    T, H, W = case["T"], case["H"], case["W"]
    for axis, n in ((2, T), (3, H), (4, W)):
        shape = [1, case["heads"], 1, 1, 1, D]
        shape[axis] = n
        wave = 0.3 * torch.randn(shape, generator=gen, device="cuda")
        for b in range(x.shape[0]):
            for h in range(case["heads"]):
                y = x[b, h, :T * H * W].view(T, H, W, D)
                y += wave[0, h].to(x.dtype)


def _lists(case, gen):
    """Lists of key blocks: `keep` of them for every query block, or from none to twice as many."""
    nt, nh, nw = _block_grid(case)
    nb, heads, keep = nt * nh * nw, case["heads"], case["keep"]
    rank = torch.rand((heads, nb, nb), generator=gen, device="cuda").argsort(dim=2).argsort(dim=2)
    if case["rows"] == "ragged":
        count = torch.randint(0, min(2 * keep, nb) + 1, (heads, nb, 1), generator=gen, device="cuda")
    else:
        count = torch.full((heads, nb, 1), keep, device="cuda")
    mask = rank < count
    row_ptr = torch.zeros(heads * nb + 1, dtype=torch.int32, device="cuda")
    row_ptr[1:] = mask.sum(dim=2).reshape(-1).cumsum(0)
    return row_ptr, mask.nonzero()[:, 2].to(torch.int32).contiguous()


def prepare(case, seed):
    gen = _generator(seed)
    op = case["op"]
    state = {"case": case}
    if op in ("norm_rope", "norm_rope_bwd"):
        dtype, n = TYPES[case["type"]], _norm_tokens(case)
        state["q"], state["k"] = _tensors(case, gen, dtype, 2, n)
        if op == "norm_rope_bwd":
            grads = dict(case, layout="head" if case["layout"] == "fused" else case["layout"])
            state["dq_out"], state["dk_out"] = _tensors(grads, gen, dtype, 2, n)
        shape = {"shared": (D,), "heads": (case["heads"], D)}.get(case["weights"])
        for name in ("q_weight", "k_weight"):
            state[name] = None if shape is None else 1.0 + 0.2 * torch.randn(shape, generator=gen, device="cuda")
        return state
    n = case["T"] * case["H"] * case["W"] + case["text"]
    tensors = _tensors(case, gen, torch.bfloat16, 2 if op == "select" else 3, n)
    if op == "select":
        for x in tensors:
            _add_structure(x, case, gen)
    else:
        state["row_ptr"], state["col_idx"] = _lists(case, gen)
    state["qkv"] = [x[0] for x in tensors]
    return state


# ---------------------------------------------------------------------------------------------- plain forms
def _turn(case, dtype, device):
    """cos and sin of every pair of every token [tokens, pairs]: angles in 64 bits, as positions may be far."""
    T, H, W, dims = case["T"], case["H"], case["W"], DIMS[case["dims"]]
    i = case["first"] + torch.arange(_norm_tokens(case), device=device)
    video = (i < T * H * W).unsqueeze(1)
    at = (i // (H * W), i // W % H, i % W)
    angles = []
    for index, d in zip(at, dims):
        freq = THETA ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=device) / d)
        angles.append((case["origin"] + case["step"] * index.double()).unsqueeze(1) * freq)
    angle = torch.where(video, torch.cat(angles, 1), 0.0)
    return angle.cos().to(dtype), angle.sin().to(dtype)


def _rotate(x, cos, sin, pairs):
    n = cos.shape[1]
    y = x.clone()
    if pairs == "interleaved":
        a, b = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
        y[..., 0:2 * n:2] = a * cos - b * sin
        y[..., 1:2 * n:2] = a * sin + b * cos
    else:
        a, b = x[..., :n], x[..., n:2 * n]
        y[..., :n] = a * cos - b * sin
        y[..., n:2 * n] = a * sin + b * cos
    return y


def _weight(w):
    return 1.0 if w is None else (w if w.dim() == 1 else w[None, :, None, :])


def _inverse_norm(x, norm):
    """1 / root mean square of a head's channels, or of all channels of a token."""
    if norm == "none":
        return 1.0
    mean = (x * x).mean(dim=-1, keepdim=True)
    if norm == "token":
        mean = mean.mean(dim=1, keepdim=True)
    return (mean + EPS).rsqrt()


def _plain_norm_rope(state):
    case, got = state["case"], []
    cos, sin = _turn(case, torch.float32, "cuda")
    for name in ("q", "k"):
        x = state[name].float()
        u = x * _inverse_norm(x, case["norm"])
        if case["norm"] != "none":
            u = u * _weight(state[name + "_weight"])
        got.append(_rotate(u, cos, sin, case["pairs"]).to(state[name].dtype))
    return got


def _plain_norm_rope_bwd(state):
    case, got, sums = state["case"], [], []
    cos, sin = _turn(case, torch.float32, "cuda")
    for name in ("q", "k"):
        g = _rotate(state["d" + name + "_out"].float(), cos, -sin, case["pairs"])
        if case["norm"] == "none":
            got.append(g.to(state[name].dtype))
            sums.append(None)
            continue
        x, w = state[name].float(), state[name + "_weight"]
        r = _inverse_norm(x, case["norm"])
        h = g * _weight(w)
        s = (h * x).mean(dim=-1, keepdim=True)
        if case["norm"] == "token":
            s = s.mean(dim=1, keepdim=True)
        got.append((r * (h - x * (r * r * s))).to(state[name].dtype))
        if w is None:
            sums.append(None)
        else:   # long sums
            sums.append((g * (x * r)).sum(dim=(0, 1, 2) if w.dim() == 1 else (0, 2), dtype=torch.float64).float())
    return got + [s for s in sums if s is not None]


def _pool(x, case):
    """Sums over the tokens of each block [heads, blocks, D] in 64 bits (values next to a border), and the blocks' tokens."""
    nt, nh, nw = _block_grid(case)
    bt, bh, bw = case["bt"], case["bh"], case["bw"]
    sums = torch.empty((case["heads"], nt * nh * nw, D), dtype=torch.float64, device=x.device)
    full = torch.zeros((nt * bt, nh * bh, nw * bw, D), dtype=torch.float64, device=x.device)
    for h in range(case["heads"]):
        full[:case["T"], :case["H"], :case["W"]] = x[h].reshape(case["T"], case["H"], case["W"], D)
        sums[h] = full.view(nt, bt, nh, bh, nw, bw, D).sum(dim=(1, 3, 5)).view(-1, D)
    sizes = []
    for n, b, extent in ((nt, bt, case["T"]), (nh, bh, case["H"]), (nw, bw, case["W"])):
        sizes.append((extent - b * torch.arange(n, dtype=torch.float64, device=x.device)).clamp(max=b))
    tokens = sizes[0][:, None, None] * sizes[1][None, :, None] * sizes[2][None, None, :]
    return sums, tokens.reshape(-1)


def _plain_select(state):
    case = state["case"]
    (q, tokens), (k, _) = (_pool(x, case) for x in state["qkv"])
    scores = q @ k.transpose(1, 2) / tokens
    scores = torch.where(scores.isnan(), -math.inf, scores)
    order = scores.sort(dim=2, descending=True, stable=True).indices[:, :, :case["keep"]]   # ties: the lowest index first
    nb = scores.shape[1]
    row_ptr = case["keep"] * torch.arange(case["heads"] * nb + 1, dtype=torch.int32, device="cuda")
    return row_ptr, order.sort(dim=2).values.to(torch.int32).reshape(-1)


def _block_tokens(case, device):
    """Token of every place of every block [blocks, places], -1 beyond the grid."""
    nt, nh, nw = _block_grid(case)
    t = torch.arange(nt * case["bt"], device=device).view(nt, 1, 1, case["bt"], 1, 1)
    h = torch.arange(nh * case["bh"], device=device).view(1, nh, 1, 1, case["bh"], 1)
    w = torch.arange(nw * case["bw"], device=device).view(1, 1, nw, 1, 1, case["bw"])
    i = (t * case["H"] + h) * case["W"] + w
    return torch.where((t < case["T"]) & (h < case["H"]) & (w < case["W"]), i, -1).reshape(nt * nh * nw, -1)


def _plain_lists(state):
    case, (q, k, v) = state["case"], state["qkv"]
    heads, text = case["heads"], case["text"]
    n_video = case["T"] * case["H"] * case["W"]
    places = _block_tokens(case, "cuda")
    nb, size = places.shape
    counts = (state["row_ptr"][1:] - state["row_ptr"][:-1]).view(heads, nb).long()
    most = min(2 * case["keep"], nb) if case["rows"] == "ragged" else case["keep"]
    # listed blocks as a rectangle, nb (a block without tokens) in the places that a row leaves empty
    slot = torch.arange(most, device="cuda")
    start = state["row_ptr"][:-1].view(heads, nb, 1).long()
    at = (start + slot).clamp(max=state["col_idx"].numel() - 1)
    listed_blocks = torch.where(slot < counts.unsqueeze(2), state["col_idx"][at].long(), nb)
    places = torch.cat([places, places.new_full((1, size), -1)])
    out = torch.empty((heads, n_video + text, D), dtype=q.dtype, device="cuda")
    lse = torch.empty((heads, n_video + text), dtype=torch.float32, device="cuda")
    step = max(1, 2 ** 28 // (most * size * (size + D)))
    for h in range(heads):
        qh, kh, vh = (x[h].float() for x in (q, k, v))
        for b in range(0, nb, step):
            rows = places[b:min(b + step, nb)]
            keys = places[listed_blocks[h, b:b + rows.shape[0]]].view(rows.shape[0], -1)
            if text:
                keys = torch.cat([keys, torch.arange(n_video, n_video + text, device="cuda").expand(rows.shape[0], text)], 1)
            s = SCALE * (qh[rows.clamp(min=0)] @ kh[keys.clamp(min=0)].transpose(1, 2))
            s = torch.where((keys >= 0).unsqueeze(1), s, -math.inf)
            m = s.amax(dim=2, keepdim=True)
            m = torch.where(m == -math.inf, 0.0, m)
            p = (s - m).exp()
            total = p.sum(dim=2, keepdim=True)
            o = (p @ vh[keys.clamp(min=0)]) / torch.where(total > 0, total, 1.0)
            real = rows >= 0
            out[h, rows[real]] = o[real].to(out.dtype)
            lse[h, rows[real]] = (m + total.log()).squeeze(2)[real]
        if text:
            s = SCALE * (qh[n_video:] @ kh.t())
            m = s.amax(dim=1, keepdim=True)
            p = (s - m).exp()
            total = p.sum(dim=1, keepdim=True)
            out[h, n_video:] = (p @ vh / total).to(out.dtype)
            lse[h, n_video:] = (m + total.log()).squeeze(1)
    return out, lse


# ---------------------------------------------------------------------------------------------- one pass
def _own_run(state):
    from paper_2609_37001_b200 import binding as psa
    case = state["case"]
    op, grid = case["op"], (case["T"], case["H"], case["W"])
    if op in ("norm_rope", "norm_rope_bwd"):
        weights = ("q_weight", "k_weight") if case["norm"] != "none" else ()   # (rotation alone has none)
        how = dict(dims=DIMS[case["dims"]], theta=THETA, norm=case["norm"], **{w: state[w] for w in weights}, eps=EPS,
                   pairs=case["pairs"], origin=(case["origin"],) * 3, step=(case["step"],) * 3, n_text=case["text"], first_token=case["first"])
        if op == "norm_rope":
            return psa.psa_qk_norm_rope(state["q"], state["k"], grid, **how)
        got = psa.psa_qk_norm_rope_bwd(state["dq_out"], state["dk_out"], state["q"], state["k"], grid, **how)
        return [x for x in got if x is not None]
    tile = (case["bt"], case["bh"], case["bw"])
    if op == "select":
        return psa.psa_select_blocks(*state["qkv"], grid, tile, case["keep"])
    return psa.psa_attn_fwd_lists(*state["qkv"], state["row_ptr"], state["col_idx"], grid, tile, SCALE, n_text=case["text"])


def run(state):
    if own:
        return _own_run(state)
    plain = {"norm_rope": _plain_norm_rope, "norm_rope_bwd": _plain_norm_rope_bwd, "select": _plain_select, "lists": _plain_lists}
    return plain[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------- work and definition
def work(case):
    op, heads = case["op"], case["heads"]
    if op in ("norm_rope", "norm_rope_bwd"):
        values = case["batch"] * heads * _norm_tokens(case) * D
        size = 4 if case["type"] == "fp32" else 2
        tensors = 4 if op == "norm_rope" else (4 if case["norm"] == "none" else 6)   # (a rotation's gradient needs no q and k)
        weights = {"shared": D, "heads": heads * D}.get(case["weights"], 0) * 4 * (2 if op == "norm_rope" else 4)
        return {"bytes": tensors * values * size + weights, "flops": (12 if op == "norm_rope" else 24) * 2 * values}
    nt, nh, nw = _block_grid(case)
    nb, tokens = nt * nh * nw, case["T"] * case["H"] * case["W"]
    if op == "select":
        lists = 4 * (heads * nb + 1 + heads * nb * case["keep"])
        return {"bytes": 2 * heads * tokens * D * 2 + lists, "flops": 2 * heads * (tokens + nb * nb) * D}
    text, every = case["text"], tokens + case["text"]
    # attended pairs, a listed block taken as one of average size
    mean = min(2 * case["keep"], nb) / 2 if case["rows"] == "ragged" else case["keep"]
    pairs = heads * (tokens * mean * tokens / nb + 2.0 * tokens * text + float(text) * text)
    return {"bytes": heads * every * (4 * D * 2 + 4) + 4 * heads * nb * (mean + 1), "flops": 4 * D * pairs}


def _complex_turn(case, device):
    """exp(i angle) [tokens, pairs] by positions one axis at a time."""
    T, H, W, dims = case["T"], case["H"], case["W"], DIMS[case["dims"]]
    i = torch.arange(T * H * W + case["text"], device=device)
    grid = torch.stack([i // (H * W), (i % (H * W)) // W, i % W]).double()
    parts = []
    for axis, d in enumerate(dims):
        j = torch.arange(d // 2, dtype=torch.float64, device=device)
        angle = torch.outer(case["origin"] + case["step"] * grid[axis], torch.exp(-math.log(THETA) * 2.0 * j / d))
        angle[T * H * W:] = 0.0
        parts.append(torch.polar(torch.ones_like(angle), angle))
    turn = torch.cat(parts, 1)
    return turn[case["first"]:case["first"] + _norm_tokens(case)]


def _exact_norm_rope(x, w, case, turn):
    if case["norm"] == "head":
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)
    elif case["norm"] == "token":
        x = x / torch.sqrt(x.square().mean((1, 3), keepdim=True) + EPS)
    if w is not None and case["norm"] != "none":
        x = x * (w if w.dim() == 1 else w.unsqueeze(1))
    n = turn.shape[1]
    if case["pairs"] == "interleaved":
        z = torch.view_as_complex(x[..., :2 * n].reshape(*x.shape[:-1], n, 2)) * turn
        return torch.cat([torch.view_as_real(z).flatten(-2), x[..., 2 * n:]], -1)
    z = torch.complex(x[..., :n], x[..., n:2 * n]) * turn
    return torch.cat([z.real, z.imag, x[..., 2 * n:]], -1)


def _exact_lists(state):
    """Query block by query block, over the tokens of its listed blocks."""
    case, (q, k, v) = state["case"], state["qkv"]
    heads, text, n_video = case["heads"], case["text"], case["T"] * case["H"] * case["W"]
    i = torch.arange(n_video, device="cuda")
    t, h, w = i // (case["H"] * case["W"]), i // case["W"] % case["H"], i % case["W"]
    _, nh, nw = _block_grid(case)
    block = (t // case["bt"] * nh + h // case["bh"]) * nw + w // case["bw"]
    nb = int(block.max()) + 1
    members = [torch.nonzero(block == b).squeeze(1) for b in range(nb)]
    text_tokens = torch.arange(n_video, n_video + text, device="cuda")
    ptr, col = state["row_ptr"].tolist(), state["col_idx"].tolist()
    out = torch.zeros((heads, n_video + text, D), dtype=torch.float64, device="cuda")
    lse = torch.full((heads, n_video + text), -math.inf, dtype=torch.float64, device="cuda")
    for head in range(heads):
        qh, kh, vh = (x[head].double() for x in (q, k, v))

        def attend(rows, keys):
            if keys.numel() == 0:
                return
            s = qh[rows] @ kh[keys].t() * SCALE
            lse[head, rows] = torch.logsumexp(s, 1)
            out[head, rows] = torch.softmax(s, 1) @ vh[keys]

        for b in range(nb):
            mine = col[ptr[head * nb + b]:ptr[head * nb + b + 1]]
            attend(members[b], torch.cat([members[j] for j in mine] + [text_tokens]))
        if text:
            attend(text_tokens, torch.arange(n_video + text, device="cuda"))
    return out, lse


def exact(case, seed):
    op = case["op"]
    if op == "lists" and work(case)["flops"] > 6e13:   # over some 20 seconds
        return None
    state = prepare(case, seed)
    if op in ("norm_rope", "norm_rope_bwd"):
        turn, got, sums = _complex_turn(case, "cuda"), [], []
        for name in ("q", "k"):
            x, w = state[name].double(), state[name + "_weight"]
            w = None if w is None else w.double()
            if op == "norm_rope":
                got.append(_exact_norm_rope(x, w, case, turn))
                continue
            leaves = [x.requires_grad_()] + ([] if w is None else [w.requires_grad_()])
            y = _exact_norm_rope(x, w, case, turn)
            grads = torch.autograd.grad(y, leaves, state["d" + name + "_out"].double())
            got.append(grads[0])
            sums.extend(grads[1:])
        return got + sums
    if op == "select":
        case, (q, k) = state["case"], state["qkv"]
        i = torch.arange(case["T"] * case["H"] * case["W"], device="cuda")
        t, h, w = i // (case["H"] * case["W"]), i // case["W"] % case["H"], i % case["W"]
        nt, nh, nw = _block_grid(case)
        nb = nt * nh * nw
        block = (t // case["bt"] * nh + h // case["bh"]) * nw + w // case["bw"]
        rows = []
        for head in range(case["heads"]):
            pooled = [torch.zeros((nb, D), dtype=torch.float64, device="cuda").index_add_(0, block, x[head].double()) for x in (q, k)]
            s = torch.einsum("ic,jc->ij", *pooled) / torch.bincount(block, minlength=nb)
            s = s.masked_fill(s.isnan(), -math.inf)
            kept = torch.argsort(-s, dim=1, stable=True)[:, :case["keep"]]
            rows.append(torch.zeros((nb, nb), dtype=torch.bool, device="cuda").scatter_(1, kept, True).nonzero()[:, 1])
        return torch.arange(0, case["heads"] * nb * case["keep"] + 1, case["keep"], dtype=torch.int32, device="cuda"), torch.cat(rows).to(torch.int32)
    return _exact_lists(state)
