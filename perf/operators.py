"""Operators around the block-scaled FP8 linear layer: casts and products with a scale for each block of 128, the embedding in
front of the first block with its gradient, and the norm and clipping of the gradients that a step leaves.

`run` computes them in elementary torch operations where `own` is false, and through paper_2505_20524_amd.fog where it is true.
"""
import math

import torch

own = False

E4M3, E5M2 = 0, 1
FP8_MAX = {E4M3: 448.0, E5M2: 57344.0}
FP8_DTYPE = {E4M3: torch.float8_e4m3fn, E5M2: torch.float8_e5m2}
BLOCK = 128
DY_STD = 1e-3            # output gradient of a linear layer
MAX_NORM = 1.0

# the costliest listed cases bound the drawn ones
MAX_LINEAR = 8192 * 4096 * 14336
MAX_CAST = 8192 * 12288
MAX_EMBED = 16384 * 4096
MAX_TABLE = 131072 * 4096
MAX_GRADS = 4 * (12288 * 4096 + 4096 * 4096 + 3 * 14336 * 4096)


def listed():
    return [
        # one token's activations on their way into a product: launch and latency are all there is
        {"name": "cast 1x4096 rows", "kind": "cast", "rows": 1, "cols": 4096, "fmt": E4M3, "form": "row"},
        # the output gradient of an 8B-scale block's widest projection, for the data gradient and the weight gradient
        {"name": "cast 8192x12288 both", "kind": "cast", "rows": 8192, "cols": 12288, "fmt": E5M2, "form": "both"},
        # a projection for a single token: cast of the activations, product with a resident weight
        {"name": "token 1x4096x4096", "kind": "token", "M": 1, "N": 4096, "K": 4096},
        # the up projection of an 8B-scale block for a batch of sequences that each take one token
        {"name": "token 24x14336x4096", "kind": "token", "M": 24, "N": 14336, "K": 4096},
        # a training step's layer whose token count and feature sizes fit no tile and no block
        {"name": "linear 1777x3088x2064", "kind": "linear", "M": 1777, "N": 3088, "K": 2064, "backward": True},
        # the largest layer of an 8B-scale block: casts, forward, data gradient, weight gradient
        {"name": "linear 8192x4096x14336", "kind": "linear", "M": 8192, "N": 4096, "K": 14336, "backward": True},
        # the rows of one decoding step
        {"name": "embed 24x2048", "kind": "embed", "T": 24, "V": 32000, "H": 2048, "cast": True, "pad": 0.0},
        # two sequences of 4096 tokens at an 8B-scale block's width
        {"name": "embed 8192x4096", "kind": "embed", "T": 8192, "V": 131072, "H": 4096, "cast": True, "pad": 0.0},
        # a short padded batch, gradient in bf16 like the products' weight gradients
        {"name": "embed grad 777x2064", "kind": "embed_grad", "T": 777, "V": 32000, "H": 2064, "type": "bf16", "pad": 0.2},
        # four sequences of 4096 tokens, gradient in 32 bits
        {"name": "embed grad 16384x4096", "kind": "embed_grad", "T": 16384, "V": 131072, "H": 4096, "type": "f32", "pad": 0.0},
        # a small model: many gradients, most of them gains of a few hundred bytes
        {"name": "clip 49 small", "kind": "clip", "layers": 6, "hidden": 512, "inner": 2048, "type": "bf16"},
        # the weight gradients of four blocks at 8B scale
        {"name": "clip 4 blocks", "kind": "clip", "layers": 4, "hidden": 4096, "inner": 14336, "type": "bf16"},
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _by16(rng, lo, hi):
    return 16 * max(1, round(_log(rng, lo, hi) / 16))


def draw(rng):
    kind = rng.choice(["cast", "cast", "token", "token", "linear", "linear", "linear", "embed", "embed_grad", "embed_grad", "clip"])
    if kind == "cast":
        while True:
            rows, cols = round(_log(rng, 1, 16384)), round(_log(rng, 128, 14336))
            if rng.random() < 0.7:
                cols = 16 * max(1, round(cols / 16))
            if rows * cols <= MAX_CAST:
                return {"kind": kind, "rows": rows, "cols": cols, "fmt": rng.choice([E4M3, E5M2]), "form": rng.choice(["row", "both", "both", "tile"])}
    if kind == "token":
        return {"kind": kind, "M": rng.randint(1, 64), "N": _by16(rng, 256, 14336), "K": _by16(rng, 256, 14336)}
    if kind == "linear":
        while True:
            M, N, K = round(_log(rng, 64, 16384)), _by16(rng, 256, 14336), _by16(rng, 256, 14336)
            if 64 * 256 * 256 <= M * N * K <= MAX_LINEAR:
                return {"kind": kind, "M": M, "N": N, "K": K, "backward": rng.random() < 0.75}
    if kind in ("embed", "embed_grad"):
        while True:
            T, V, H = round(_log(rng, 1, 65536)), round(_log(rng, 256, 200000)), round(_log(rng, 256, 8192))
            if rng.random() < 0.8:
                H = 16 * max(1, round(H / 16))
            if T * H <= MAX_EMBED and V * H <= MAX_TABLE:
                break
        case = {"kind": kind, "T": T, "V": V, "H": H, "pad": rng.choice([0.0, 0.0, 0.3])}
        case.update({"cast": rng.random() < 0.7} if kind == "embed" else {"type": rng.choice(["bf16", "f32"])})
        return case
    while True:
        layers, hidden, inner = rng.randint(1, 6), 8 * round(_log(rng, 256, 4096) / 8), 8 * round(_log(rng, 512, 14336) / 8)
        if layers * sum(math.prod(s) for s in _layer(hidden, inner)) <= MAX_GRADS:
            return {"kind": kind, "layers": layers, "hidden": hidden, "inner": inner, "type": rng.choice(["bf16", "bf16", "f32"])}


# ---------------------------------------------------------------------------------------------- inputs
def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    return torch.randn(shape, device="cuda", generator=g).mul_(std).to(dtype)


def _activations(g, rows, cols):
    """Normal values with two channels fifty times larger: the outliers of trained activations."""
    x = torch.randn((rows, cols), device="cuda", generator=g)
    x[:, torch.randperm(cols, device="cuda", generator=g)[:2]] *= 50.0
    return x.to(torch.bfloat16)


def _tokens(g, T, V, pad):
    """Ids whose frequency falls like one over their rank, as words' do; a share of -1 behind short sequences."""
    u = torch.rand(T, device="cuda", generator=g, dtype=torch.float64)
    t = (torch.exp(u * math.log(V + 1)) - 1).long().clamp_(0, V - 1)
    t = torch.randperm(V, device="cuda", generator=g)[t]
    return torch.where(torch.rand(T, device="cuda", generator=g) < pad, torch.full_like(t, -1), t)


def _layer(hidden, inner):
    """Gradients of a block: projections of attention and of the gated feed-forward half, two gains of the post-norms, two scalars' vector."""
    return [(3 * hidden, hidden), (hidden, hidden), (inner, hidden), (inner, hidden), (hidden, inner), (hidden,), (hidden,), (2,)]


def _bytes(*shape):
    return torch.empty(shape, dtype=torch.uint8, device="cuda")


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    st, kind = {"case": case, "kept": {}}, case["kind"]
    if kind == "cast":
        rows, cols = case["rows"], case["cols"]
        st["x"] = _activations(g, rows, cols) if case["fmt"] == E4M3 else _normal(g, (rows, cols), DY_STD)
        st["out"] = _cast_room(rows, cols, case["form"])
    elif kind == "token":
        M, N, K = case["M"], case["N"], case["K"]
        # the weight as the program keeps it: its codes and the scales of its 128 x 128 blocks
        st["x"], st["w"] = _activations(g, M, K), _cast_plain(_normal(g, (N, K), 0.02), E4M3, "tile")
        st["out"], st["Y"] = _cast_room(M, K, "row"), torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    elif kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        st["X"], st["W"] = _activations(g, M, K), _normal(g, (N, K), 0.02)
        st["Y"] = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
        st["Xq"], st["Wq"] = _cast_room(M, K, "both" if case["backward"] else "row"), _cast_room(N, K, "tile")
        if case["backward"]:
            st["dY"], st["dYq"] = _normal(g, (M, N), DY_STD), _cast_room(M, N, "both")
            st["dX"], st["dW"] = torch.empty_like(st["X"]), torch.empty_like(st["W"])
    elif kind == "embed":
        T, V, H = case["T"], case["V"], case["H"]
        st["tokens"], st["table"] = _tokens(g, T, V, case["pad"]), _normal(g, (V, H), 0.02)
        st["factor"] = math.sqrt(H)
        # the scale a history of such rows gives
        st["scale"], st["amax"] = torch.full((1,), 448.0 / (0.02 * 6.0 * math.sqrt(H)), device="cuda"), torch.zeros(1, device="cuda")
        st["x"], st["q"] = torch.empty((T, H), dtype=torch.bfloat16, device="cuda"), _bytes(T, H)
    elif kind == "embed_grad":
        T, V, H = case["T"], case["V"], case["H"]
        st["tokens"], st["dx"], st["factor"] = _tokens(g, T, V, case["pad"]), _normal(g, (T, H), DY_STD), math.sqrt(H)
        st["dE"] = torch.empty((V, H), dtype=torch.bfloat16 if case["type"] == "bf16" else torch.float32, device="cuda")
    else:
        dtype = torch.bfloat16 if case["type"] == "bf16" else torch.float32
        shapes = _layer(case["hidden"], case["inner"]) * case["layers"] + [(case["hidden"],)]
        st["grads"] = [_normal(g, s, 1e-2, dtype) for s in shapes]
        st["clipped"] = [torch.empty_like(t) for t in st["grads"]]
        st["norm"], st["sumsq"] = torch.empty(1, device="cuda"), torch.empty(1, dtype=torch.float64, device="cuda")
    return st


def _cast_room(rows, cols, form):
    """Where a cast goes: codes of the tensor's shape, one scale byte for each block."""
    if form == "tile":
        return {"q": _bytes(rows, cols), "s": _bytes(_blocks(rows), _blocks(cols))}
    out = {"q_row": _bytes(rows, cols), "s_row": _bytes(_blocks(cols), rows)}
    if form == "both":
        out.update(q_col=_bytes(rows, cols), s_col=_bytes(_blocks(rows), cols))
    return out


# ---------------------------------------------------------------------------------------------- plain form
def _padded(x):
    rows, cols = x.shape
    return torch.nn.functional.pad(x, (0, -cols % BLOCK, 0, -rows % BLOCK))


def _exponent(amax, fmt):
    """k of the block's scale 2^k: the largest with amax 2^k <= FP8MAX (= 0.875 * 2^9 or 0.875 * 2^16)."""
    m, e = torch.frexp(amax)
    k = (9 if fmt == E4M3 else 16) - e - (m > 0.875).int()
    return torch.where((amax > 0) & torch.isfinite(amax), k.clamp(-126, 126), torch.zeros_like(k))


def _pow2(k):
    """2^k in 32 bits from its exponent field (-127 < k < 128)."""
    return ((k.int() + 127) << 23).view(torch.float32)


def _codes(x32, k, fmt):
    return (x32 * _pow2(k)).clamp(-FP8_MAX[fmt], FP8_MAX[fmt]).to(FP8_DTYPE[fmt])


def _cast_plain(x, fmt, form):
    """Codes (as FP8 values) and scale bytes of one form of the block cast: along rows, along columns, by tiles."""
    rows, cols = x.shape
    p = _padded(x.float())
    nr, nc = p.shape[0] // BLOCK, p.shape[1] // BLOCK
    p = p.view(nr, BLOCK, nc, BLOCK)
    dims = {"row": (3,), "col": (1,), "tile": (1, 3)}[form]
    k = _exponent(p.abs().amax(dim=dims, keepdim=True), fmt)
    q = _codes(p, k, fmt).view(torch.uint8).reshape(nr * BLOCK, nc * BLOCK)[:rows, :cols].contiguous().view(FP8_DTYPE[fmt])
    e = (127 - k).to(torch.uint8)
    if form == "row":        # [blocks of columns][rows]
        return q, e.reshape(nr * BLOCK, nc)[:rows].t().contiguous()
    if form == "col":        # [blocks of rows][columns]
        return q, e.reshape(nr, nc * BLOCK)[:, :cols].contiguous()
    return q, e.reshape(nr, nc)


def _values(q, s, form):
    """The 32-bit values that codes and scale bytes stand for."""
    rows, cols = q.shape
    inv = _pow2(s.int() - 127)
    if form == "row":
        inv = inv.t().repeat_interleave(BLOCK, dim=1)[:, :cols]
    elif form == "col":
        inv = inv.repeat_interleave(BLOCK, dim=0)[:rows]
    else:
        inv = inv.repeat_interleave(BLOCK, dim=0)[:rows].repeat_interleave(BLOCK, dim=1)[:, :cols]
    return q.float() * inv


def _run_plain(st):
    case, kind = st["case"], st["case"]["kind"]
    if kind == "cast":
        x, fmt = st["x"], case["fmt"]
        if case["form"] == "tile":
            return dict(zip(("q", "s"), _cast_plain(x, fmt, "tile")))
        out = dict(zip(("q_row", "s_row"), _cast_plain(x, fmt, "row")))
        if case["form"] == "both":
            out.update(zip(("q_col", "s_col"), _cast_plain(x, fmt, "col")))
        return out
    if kind == "token":
        return {"Y": (_values(*_cast_plain(st["x"], E4M3, "row"), "row") @ _values(*st["w"], "tile").t()).to(torch.bfloat16)}
    if kind == "linear":
        W = _values(*_cast_plain(st["W"], E4M3, "tile"), "tile")
        out = {"Y": (_values(*_cast_plain(st["X"], E4M3, "row"), "row") @ W.t()).to(torch.bfloat16)}
        if case["backward"]:
            out["dX"] = (_values(*_cast_plain(st["dY"], E5M2, "row"), "row") @ W).to(torch.bfloat16)
            X, dY = _values(*_cast_plain(st["X"], E4M3, "col"), "col"), _values(*_cast_plain(st["dY"], E5M2, "col"), "col")
            out["dW"] = (dY.t() @ X).to(torch.bfloat16)
        return out
    if kind == "embed":
        t = st["tokens"]
        x = torch.where((t >= 0).unsqueeze(1), st["table"][t.clamp(min=0)].float() * st["factor"], torch.zeros((), device="cuda")).to(torch.bfloat16)
        out = {"x": x, "amax": x.float().abs().amax().reshape(1)}
        if case["cast"]:
            out["q"] = (x.float() * st["scale"]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
        return out
    if kind == "embed_grad":
        t, dE = st["tokens"], torch.zeros(st["dE"].shape, device="cuda")
        dE.index_add_(0, t.clamp(min=0), torch.where((t >= 0).unsqueeze(1), st["dx"].float() * st["factor"], torch.zeros((), device="cuda")))
        return {"dE": dE.to(st["dE"].dtype)}
    norm = torch.stack([t.float().square().sum(dtype=torch.float64) for t in st["grads"]]).sum().sqrt()
    c = torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm)).float()
    return {"norm": norm.float().reshape(1), "grads": [(t.float() * c).to(t.dtype) for t in st["grads"]]}


# ---------------------------------------------------------------------------------------------- the framework's calls
def _kept(st, name, size):
    """A workspace that the program keeps between its calls."""
    if name not in st["kept"]:
        st["kept"][name] = torch.empty(max(size(), 16), dtype=torch.uint8, device="cuda")
    return st["kept"][name]


def _run_own(st):
    from paper_2505_20524_amd import fog
    case, kind = st["case"], st["case"]["kind"]
    if kind == "cast":
        fmt, o = case["fmt"], st["out"]
        if case["form"] == "tile":
            fog.quantize_tile(st["x"], fmt, o["q"], o["s"])
        else:
            fog.quantize_block(st["x"], fmt, **o)
        return {k: v.view(FP8_DTYPE[fmt]) if k[0] == "q" else v for k, v in o.items()}
    if kind == "token":
        M, N, K, o, w = case["M"], case["N"], case["K"], st["out"], st["w"]
        ws = _kept(st, "ws", lambda: fog.fp8_gemm_block_workspace(fog.NT, M, N, K))
        fog.quantize_block(st["x"], E4M3, **o)
        fog.fp8_gemm_block(fog.NT, M, N, K, o["q_row"], E4M3, fog.VECTOR, o["s_row"], w[0], E4M3, fog.TILE, w[1], st["Y"], workspace=ws)
        return {"Y": st["Y"]}
    if kind == "linear":
        M, N, K, X, W = case["M"], case["N"], case["K"], st["Xq"], st["Wq"]
        fog.quantize_block(st["X"], E4M3, **X)
        fog.quantize_tile(st["W"], E4M3, W["q"], W["s"])
        ws = _kept(st, "ws", lambda: max(fog.fp8_gemm_block_workspace(fog.NT, M, N, K), fog.fp8_gemm_block_workspace(fog.NN, M, K, N),
                                         fog.fp8_gemm_block_workspace(fog.TN, N, K, M)))
        fog.fp8_gemm_block(fog.NT, M, N, K, X["q_row"], E4M3, fog.VECTOR, X["s_row"], W["q"], E4M3, fog.TILE, W["s"], st["Y"], workspace=ws)
        if not case["backward"]:
            return {"Y": st["Y"]}
        dY = st["dYq"]
        fog.quantize_block(st["dY"], E5M2, **dY)
        fog.fp8_gemm_block(fog.NN, M, K, N, dY["q_row"], E5M2, fog.VECTOR, dY["s_row"], W["q"], E4M3, fog.TILE, W["s"], st["dX"], workspace=ws)
        fog.fp8_gemm_block(fog.TN, N, K, M, dY["q_col"], E5M2, fog.VECTOR, dY["s_col"], X["q_col"], E4M3, fog.VECTOR, X["s_col"], st["dW"], workspace=ws)
        return {"Y": st["Y"], "dX": st["dX"], "dW": st["dW"]}
    if kind == "embed":
        q = st["q"] if case["cast"] else None
        fog.embed_quantize(st["tokens"], st["table"], st["factor"], E4M3, st["scale"], st["x"], q=q, amax_out=st["amax"])
        out = {"x": st["x"], "amax": st["amax"]}
        if case["cast"]:
            out["q"] = q.view(torch.float8_e4m3fn)
        return out
    if kind == "embed_grad":
        ws = _kept(st, "ws", lambda: fog.embed_grad_workspace(case["T"], case["V"], case["H"]))
        fog.embed_grad(st["tokens"], st["dx"], st["factor"], st["dE"], ws)
        return {"dE": st["dE"]}
    ws = _kept(st, "ws", lambda: fog.grad_sumsq_workspace(len(st["grads"])))
    if "jobs" not in st["kept"]:
        st["kept"]["jobs"] = fog.make_grad_jobs(list(zip(st["grads"], st["clipped"])))
    fog.grad_sumsq(st["kept"]["jobs"], st["sumsq"], ws)
    fog.grad_clip(st["kept"]["jobs"], st["sumsq"], MAX_NORM, st["norm"])
    return {"norm": st["norm"], "grads": list(st["clipped"])}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------------------------- work
def work(case):
    kind = case["kind"]
    if kind == "cast":
        n, both = case["rows"] * case["cols"], case["form"] == "both"
        return {"bytes": n * (4 if both else 3) + n // BLOCK * (2 if both else 1), "flops": 0}
    if kind == "token":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": 2 * M * K + N * K + 2 * M * N, "flops": 2 * M * N * K}
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        nbytes = 2 * (M * K + N * K + M * N)
        if case["backward"]:
            nbytes += 2 * (M * N + M * K + N * K)
        return {"bytes": nbytes, "flops": 2 * M * N * K * (3 if case["backward"] else 1)}
    if kind == "embed":
        T, H = case["T"], case["H"]
        return {"bytes": 8 * T + T * H * (5 if case["cast"] else 4), "flops": 0}
    if kind == "embed_grad":
        T, V, H = case["T"], case["V"], case["H"]
        return {"bytes": 8 * T + 2 * T * H + (2 if case["type"] == "bf16" else 4) * V * H, "flops": T * H}
    n = case["layers"] * sum(math.prod(s) for s in _layer(case["hidden"], case["inner"])) + case["hidden"]
    # the norm has to be known before the first gradient is scaled: read twice, written once
    return {"bytes": 3 * (2 if case["type"] == "bf16" else 4) * n, "flops": 3 * n}


# ---------------------------------------------------------------------------------------------- the same in 64 bits
def _grid64(v, fmt):
    """64-bit values rounded to the FP8 grid, ties to even, saturating: 3 or 2 places behind the leading bit, fewer below the smallest normal."""
    places, low = (3, -6) if fmt == E4M3 else (2, -14)
    step = torch.exp2((torch.frexp(v).exponent - 1).clamp(min=low).double() - places)
    return (torch.round(v / step) * step).clamp(-FP8_MAX[fmt], FP8_MAX[fmt])


def _cast64(x, fmt, rows_of_block, cols_of_block):
    """(codes' values, exponents k by block) for blocks of rows_of_block x cols_of_block."""
    rows, cols = x.shape
    br, bc = -(-rows // rows_of_block), -(-cols // cols_of_block)
    p = torch.zeros((br * rows_of_block, bc * cols_of_block), dtype=torch.float64, device="cuda")
    p[:rows, :cols] = x
    t = p.view(br, rows_of_block, bc, cols_of_block).permute(0, 2, 1, 3)
    top = t.reshape(br, bc, -1).abs().max(dim=2).values
    k = torch.floor(torch.log2(FP8_MAX[fmt] / top.clamp(min=1e-300)))
    k = torch.where(top * torch.exp2(k + 1) <= FP8_MAX[fmt], k + 1, k)
    k = torch.where(top * torch.exp2(k) > FP8_MAX[fmt], k - 1, k)
    k = torch.where(top > 0, k.clamp(-126, 126), torch.zeros_like(k))
    q = _grid64(t * torch.exp2(k)[:, :, None, None], fmt)
    back = lambda z: z.permute(0, 2, 1, 3).reshape(br * rows_of_block, bc * cols_of_block)[:rows, :cols]  # noqa: E731
    return back(q), k, back(q * torch.exp2(-k)[:, :, None, None])


def exact(case, seed):
    st, kind = prepare(case, seed), case["kind"]
    if kind == "cast":
        if case["form"] == "tile":
            q, k, _ = _cast64(st["x"], case["fmt"], BLOCK, BLOCK)
            return {"q": q, "s": (127 - k).to(torch.uint8)}
        q, k, _ = _cast64(st["x"], case["fmt"], 1, BLOCK)
        out = {"q_row": q, "s_row": (127 - k).to(torch.uint8).t().contiguous()}
        if case["form"] == "both":
            q, k, _ = _cast64(st["x"], case["fmt"], BLOCK, 1)
            out.update(q_col=q, s_col=(127 - k).to(torch.uint8))
        return out
    if kind == "token":
        q, s = st["w"]
        N, K = q.shape
        inv = torch.exp2(s.double() - 127.0)
        n, k = torch.arange(N, device="cuda") // BLOCK, torch.arange(K, device="cuda") // BLOCK
        return {"Y": _cast64(st["x"], E4M3, 1, BLOCK)[2] @ (q.double() * inv[n][:, k]).t()}
    if kind == "linear":
        W = _cast64(st["W"], E4M3, BLOCK, BLOCK)[2]
        out = {"Y": _cast64(st["X"], E4M3, 1, BLOCK)[2] @ W.t()}
        if case["backward"]:
            out["dX"] = _cast64(st["dY"], E5M2, 1, BLOCK)[2] @ W
            out["dW"] = _cast64(st["dY"], E5M2, BLOCK, 1)[2].t() @ _cast64(st["X"], E4M3, BLOCK, 1)[2]
        return out
    if kind == "embed":
        t = st["tokens"]
        x = torch.zeros((case["T"], case["H"]), dtype=torch.float64, device="cuda")
        x[t >= 0] = st["table"][t[t >= 0]].double() * st["factor"]
        # what is cast, and the abs-max, are of the stored bf16 row
        kept = x.to(torch.bfloat16).double()
        out = {"x": x, "amax": kept.abs().max().reshape(1)}
        if case["cast"]:
            out["q"] = _grid64(kept * st["scale"].double(), E4M3)
        return out
    if kind == "embed_grad":
        t = st["tokens"]
        order = torch.argsort(t, stable=True)
        order = order[t[order] >= 0]
        dE = torch.zeros((case["V"], case["H"]), dtype=torch.float64, device="cuda")
        if order.numel():
            ids, counts = torch.unique_consecutive(t[order], return_counts=True)
            ends = torch.cumsum(counts, 0)
            dx = st["dx"].double()
            wide = max(1, (1 << 27) // max(1, order.numel()))
            for c in range(0, case["H"], wide):
                run_sum = torch.cumsum(dx[order, c:c + wide], 0)[ends - 1]
                dE[ids, c:c + wide] = torch.diff(run_sum, dim=0, prepend=torch.zeros_like(run_sum[:1])) * st["factor"]
        return {"dE": dE}
    total = sum(float((t.double() ** 2).sum()) for t in st["grads"])
    norm = math.sqrt(total)
    c = MAX_NORM / norm if norm > MAX_NORM else 1.0
    return {"norm": torch.tensor([norm], dtype=torch.float64, device="cuda"), "grads": [t.double() * c for t in st["grads"]]}
