"""What a training step of a block does between its products: rotary positions with the QK norm and the FP8 cast, and their backward; the backward
of the post-norm with its residual connection and of the activation; the AdamW update.

`run` computes them in elementary torch operations where `own` is false, and through paper_2505_20524_amd.fog where it is true.
"""
import math

import torch

own = False

E4M3, E5M2 = 0, 1
FP8_MAX = {E4M3: 448.0, E5M2: 57344.0}
FP8_DTYPE = {E4M3: torch.float8_e4m3fn, E5M2: torch.float8_e5m2}
HALF, INTERLEAVED = 0, 1
BLOCK = 128
GRAD_STD = 1e-3          # a gradient on its way back through the block
MAX_NORM = 1.0
LR, BETA1, BETA2, EPS, DECAY = 3e-4, 0.9, 0.95, 1e-8, 0.1
PARTS = (12288 * 4096, 4096 * 4096, 3 * 14336 * 4096)

# the costliest listed cases bound the drawn ones
MAX_HEADS = 8192 * 48 * 128
MAX_NORMED = 8192 * 4096
MAX_ACT = 8192 * 14336
MAX_UPDATE = 2 * sum(PARTS)


def listed():
    return [
        # a decoding step of 24 sequences, each at a position of its own, on grouped heads
        {"name": "rope 24 tokens 32/8", "kind": "rope", "B": 24, "S": 1, "H": 32, "Hkv": 8, "D": 128, "rot": 128, "layout": HALF, "norm": True,
         "positions": 131072, "given": True},
        # three sequences of a length that fits no tile; a quarter of a narrow head turned, pairs side by side, no norm
        {"name": "rope 3x777 5 heads", "kind": "rope", "B": 3, "S": 777, "H": 5, "Hkv": 5, "D": 80, "rot": 20, "layout": INTERLEAVED, "norm": False,
         "positions": 4096, "given": False},
        # two training sequences of 4096 tokens at an 8B-scale block's width
        {"name": "rope 2x4096 32/8", "kind": "rope", "B": 2, "S": 4096, "H": 32, "Hkv": 8, "D": 128, "rot": 128, "layout": HALF, "norm": True,
         "positions": 4096, "given": False},
        # a short packed batch: positions start again inside the row, padding behind
        {"name": "rope grad 1x333 16/4", "kind": "rope_grad", "B": 1, "S": 333, "H": 16, "Hkv": 4, "D": 128, "rot": 64, "layout": INTERLEAVED, "norm": True,
         "positions": 512, "given": True, "keep": True},
        {"name": "rope grad 2x4096 32/8", "kind": "rope_grad", "B": 2, "S": 4096, "H": 32, "Hkv": 8, "D": 128, "rot": 128, "layout": HALF, "norm": True,
         "positions": 4096, "given": False, "keep": False},
        # the end of a sub-layer on the way back, where sizes fit no tile
        {"name": "post-norm grad 777x2064", "kind": "postnorm_grad", "rows": 777, "cols": 2064, "branch": True, "keep": True},
        {"name": "post-norm grad 8192x4096", "kind": "postnorm_grad", "rows": 8192, "cols": 4096, "branch": True, "keep": False},
        # between the two products of the feed-forward half
        {"name": "GeLU grad 333x2736", "kind": "act_grad", "act": "gelu", "rows": 333, "cols": 2736, "keep": True},
        {"name": "xIELU grad 8192x14336", "kind": "act_grad", "act": "xielu", "rows": 8192, "cols": 14336, "keep": False},
        # a small model: many parameters, most of them gains of a few hundred numbers
        {"name": "AdamW 49 small", "kind": "adamw", "layers": 6, "hidden": 256, "inner": 704, "states": "f32", "master": True, "grad": "bf16"},
        # two blocks at 8B scale, what one of many ranks may hold
        {"name": "AdamW 2 blocks", "kind": "adamw", "layers": 2, "hidden": 4096, "inner": 14336, "states": "f32", "master": True, "grad": "bf16"},
        {"name": "AdamW 2 blocks, states in 8 bits", "kind": "adamw", "layers": 2, "hidden": 4096, "inner": 14336, "states": "fp8", "master": True, "grad": "bf16"},
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["rope", "rope", "rope_grad", "rope_grad", "postnorm_grad", "act_grad", "adamw", "adamw"])
    if kind in ("rope", "rope_grad"):
        while True:
            B, S = round(_log(rng, 1, 64)), round(_log(rng, 1, 8192))
            Hkv = round(_log(rng, 1, 16))
            H, D = Hkv * rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 96, 128, 128, 128, 192, 256])
            rot = rng.choice([D, D, D // 2, 2 * round(D / 8)])
            if B * S * (H + 2 * Hkv) * D <= MAX_HEADS:
                break
        case = {"kind": kind, "B": B, "S": S, "H": H, "Hkv": Hkv, "D": D, "rot": rot, "layout": rng.choice([HALF, INTERLEAVED]), "norm": rng.random() < 0.6,
                "positions": max(S, round(_log(rng, 1024, 131072))), "given": rng.random() < 0.4}
        if kind == "rope_grad":
            case["keep"] = rng.random() < 0.4
        return case
    if kind == "postnorm_grad":
        while True:
            rows, cols = round(_log(rng, 1, 65536)), round(_log(rng, 256, 16384))
            if rng.random() < 0.7:
                cols = 16 * max(1, round(cols / 16))
            if rows * cols <= MAX_NORMED:
                return {"kind": kind, "rows": rows, "cols": cols, "branch": rng.random() < 0.7, "keep": rng.random() < 0.4}
    if kind == "act_grad":
        while True:
            rows, cols = round(_log(rng, 1, 65536)), round(_log(rng, 256, 16384))
            if rng.random() < 0.7:
                cols = 16 * max(1, round(cols / 16))
            if rows * cols <= MAX_ACT:
                return {"kind": kind, "act": rng.choice(["xielu", "xielu", "gelu", "tanh"]), "rows": rows, "cols": cols, "keep": rng.random() < 0.4}
    while True:
        layers, hidden, inner = rng.randint(1, 6), 8 * round(_log(rng, 256, 4096) / 8), 8 * round(_log(rng, 512, 14336) / 8)
        if layers * sum(math.prod(s) for s in _layer(hidden, inner)) <= MAX_UPDATE:
            return {"kind": kind, "layers": layers, "hidden": hidden, "inner": inner, "states": rng.choice(["f32", "fp8"]), "master": rng.random() < 0.8,
                    "grad": rng.choice(["bf16", "bf16", "f32"])}


# ---------------------------------------------------------------------------------------------- inputs
def _normal(g, shape, std=1.0, dtype=torch.bfloat16):
    return torch.randn(shape, device="cuda", generator=g).mul_(std).to(dtype)


def _layer(hidden, inner):
    """Parameters of a block: projections of attention and of the gated feed-forward half, two gains of the post-norms, two scalars' vector."""
    return [(3 * hidden, hidden), (hidden, hidden), (inner, hidden), (inner, hidden), (hidden, inner), (hidden,), (hidden,), (2,)]


def _angles(case):
    """cos and sin of every position and pair, [positions, rot / 2] each, from 64-bit angles."""
    half = case["rot"] // 2
    f = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    a = torch.arange(case["positions"], device="cuda", dtype=torch.float64)[:, None] * f
    return torch.cos(a), torch.sin(a)


def _positions(case, g):
    """Positions as a program hands them over: a cache length each, or documents that start again inside a row with padding behind."""
    B, S = case["B"], case["S"]
    if S == 1:
        return torch.randint(0, case["positions"], (B, 1), device="cuda", generator=g, dtype=torch.int32)
    s = torch.arange(S, device="cuda", dtype=torch.int32).expand(B, S)
    cut = torch.randint(1, S, (B, 1), device="cuda", generator=g, dtype=torch.int32)
    p = torch.where(s < cut, s, s - cut)
    return torch.where(s >= S - S // 16, torch.full_like(p, -1), p).contiguous()


def _scalar(v):
    return torch.full((1,), float(v), device="cuda")


def _empty(*shape, dtype=torch.uint8):
    return torch.empty(shape, dtype=dtype, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    st, kind = {"case": case, "kept": {}}, case["kind"]
    if kind in ("rope", "rope_grad"):
        B, S, H, Hkv, D = case["B"], case["S"], case["H"], case["Hkv"], case["D"]
        st["x"] = _normal(g, (B, S, H + 2 * Hkv, D))
        st["table"] = torch.cat(_angles(case), dim=1).float()
        st["pos"] = _positions(case, g) if case["given"] else None
        st["amax"] = [torch.zeros(1, device="cuda") for _ in range(3)]
        if kind == "rope":
            # |y| <= sqrt(D) behind the norm; without it the range that a history of such rows gives
            st["scale"] = [_scalar(448.0 / (math.sqrt(D) if case["norm"] and i < 2 else 6.5)) for i in range(3)]
            st["q"] = [_empty(B, h, S, D) for h in (H, Hkv, Hkv)]
        else:
            st["dy"] = [_normal(g, (B, h, S, D), GRAD_STD) for h in (H, Hkv, Hkv)]
            st["scale"] = _scalar(57344.0 / (8 * GRAD_STD))
            st["q"] = _empty(B, S, H + 2 * Hkv, D)
            st["dx"] = _empty(B, S, H + 2 * Hkv, D, dtype=torch.bfloat16) if case["keep"] else None
    elif kind == "postnorm_grad":
        rows, cols = case["rows"], case["cols"]
        st["y"], st["dres"] = _normal(g, (rows, cols)), _normal(g, (rows, cols), GRAD_STD)
        st["dbranch"] = _normal(g, (rows, cols), GRAD_STD) if case["branch"] else None
        st["gamma"] = torch.rand(cols, device="cuda", generator=g) * 0.2 + 0.1
        st["scale"], st["amax"], st["dgamma"] = _scalar(57344.0 / (4 * GRAD_STD)), torch.zeros(1, device="cuda"), torch.empty(cols, device="cuda")
        st["dstream"] = torch.empty_like(st["dres"]) if case["branch"] else None
        st["dy"], st["q"] = torch.empty_like(st["y"]) if case["keep"] else None, _empty(rows, cols)
    elif kind == "act_grad":
        rows, cols = case["rows"], case["cols"]
        st["x"], st["dy"] = _normal(g, (rows, cols), 1.5), _normal(g, (rows, cols), GRAD_STD)
        st["alpha"] = {"xielu": (0.8, 0.6), "gelu": (), "tanh": (0.5,)}[case["act"]]
        st["dalpha"] = torch.empty(len(st["alpha"]), device="cuda") if st["alpha"] else None
        st["scale"], st["amax"] = _scalar(57344.0 / (60 * GRAD_STD)), torch.zeros(1, device="cuda")
        st["dx"], st["q"] = torch.empty_like(st["x"]) if case["keep"] else None, _empty(rows, cols)
    else:
        shapes = _layer(case["hidden"], case["inner"]) * case["layers"] + [(case["hidden"],)]
        # a program's buckets: every tensor begins at a multiple of 128 elements
        st["n"] = [math.prod(s) for s in shapes]
        st["at"] = [0]
        for n in st["n"]:
            st["at"].append(st["at"][-1] + (n + BLOCK - 1) // BLOCK * BLOCK)
        N = st["at"][-1]
        st["decay"] = [DECAY if len(s) == 2 else 0.0 for s in shapes]
        st["g"] = _normal(g, (N,), 1e-2, torch.bfloat16 if case["grad"] == "bf16" else torch.float32)
        master = torch.randn(N, device="cuda", generator=g).mul_(0.02)
        st["p"] = master.to(torch.bfloat16)
        st["master"] = master if case["master"] else None
        st["sumsq"] = torch.zeros(1, dtype=torch.float64, device="cuda")
        for n, a in zip(st["n"], st["at"]):
            st["sumsq"] += st["g"][a:a + n].double().square().sum()
        st["step"], st["seed"] = 1000, 12345 + seed % 1000
        m, v = torch.randn(N, device="cuda", generator=g).mul_(1e-4), torch.randn(N, device="cuda", generator=g).mul_(2e-4).square_()
        if case["states"] == "f32":
            st["m"], st["v"], st["ms"], st["vs"] = m, v, None, None
        else:
            st["m"], st["ms"] = _block_cast(m, E4M3)
            st["v"], st["vs"] = _block_cast(v, E5M2)
    return st


# ---------------------------------------------------------------------------------------------- plain form
def _cast(x32, scale, fmt):
    return (x32 * scale).clamp(-FP8_MAX[fmt], FP8_MAX[fmt]).to(FP8_DTYPE[fmt])


def _rows(st):
    """cos and sin for every token, [B, S, 1, rot / 2], and which tokens have a position of the table."""
    case, half = st["case"], st["case"]["rot"] // 2
    pos = torch.arange(case["S"], device="cuda").expand(case["B"], case["S"]) if st["pos"] is None else st["pos"].long()
    there = ((pos >= 0) & (pos < case["positions"]))[:, :, None, None]
    t = st["table"][pos.clamp(0, case["positions"] - 1)].unsqueeze(2)
    return t[..., :half], t[..., half:], there


def _turn(x, cos, sin, layout):
    half = cos.shape[-1]
    if layout == HALF:
        a, b = x[..., :half], x[..., half:2 * half]
        return torch.cat((a * cos - b * sin, b * cos + a * sin, x[..., 2 * half:]), dim=-1)
    a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
    return torch.cat((torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2), x[..., 2 * half:]), dim=-1)


def _heads(case):
    """First head, number of heads, whether turned: Q, K, V in the projection's result."""
    H, Hkv = case["H"], case["Hkv"]
    return ((0, H, True), (H, Hkv, True), (H + Hkv, Hkv, False))


def _rope_plain(st):
    case = st["case"]
    cos, sin, there = _rows(st)
    q, amax = [], []
    for i, (first, n, turned) in enumerate(_heads(case)):
        x = st["x"][:, :, first:first + n].float()
        if turned:
            if case["norm"]:
                x = x / x.square().mean(dim=-1, keepdim=True).sqrt()
            x = torch.where(there, _turn(x, cos, sin, case["layout"]), torch.zeros_like(x))
        amax.append(x.abs().amax().reshape(1))
        q.append(_cast(x, st["scale"][i], E4M3).transpose(1, 2).contiguous())
    return {"q": q, "amax": amax}


def _rope_grad_plain(st):
    case = st["case"]
    cos, sin, there = _rows(st)
    parts = []
    for (first, n, turned), dy in zip(_heads(case), st["dy"]):
        d = dy.float().transpose(1, 2)
        if turned:
            d = torch.where(there, _turn(d, cos, -sin, case["layout"]), torch.zeros_like(d))
            if case["norm"]:
                x = st["x"][:, :, first:first + n].float()
                xx = x.square().sum(dim=-1, keepdim=True)
                d = (d - x * ((x * d).sum(dim=-1, keepdim=True) / xx)) / (xx / case["D"]).sqrt()
        parts.append(d)
    dx = torch.cat(parts, dim=2).to(torch.bfloat16)
    out = {"q": _cast(dx.float(), st["scale"], E5M2), "amax": dx.abs().amax().float().reshape(1)}
    if case["keep"]:
        out["dx"] = dx
    return out


def _postnorm_grad_plain(st):
    case, y = st["case"], st["y"].float()
    G = st["dres"]
    if case["branch"]:
        G = (G.float() + st["dbranch"].float()).to(torch.bfloat16)
    inv = 1.0 / y.square().mean(dim=1, keepdim=True).sqrt()
    yh, t = y * inv, G.float() * st["gamma"]
    dy = (inv * (t - yh * (t * yh).mean(dim=1, keepdim=True))).to(torch.bfloat16)
    out = {"q": _cast(dy.float(), st["scale"], E5M2), "amax": dy.abs().amax().float().reshape(1), "dgamma": (G.float() * yh).sum(dim=0, dtype=torch.float64).float()}
    if case["branch"]:
        out["dstream"] = G
    if case["keep"]:
        out["dy"] = dy
    return out


def _act_grad_plain(st):
    case, x, dy = st["case"], st["x"].float(), st["dy"].float()
    dalpha = None
    if case["act"] == "xielu":
        ap, an = st["alpha"]
        e = torch.expm1(x.clamp(max=0.0))
        slope = torch.where(x > 0, 2 * ap * x + 0.5, an * e + 0.5)
        zero = torch.zeros((), device="cuda")
        dalpha = torch.stack([torch.where(x > 0, dy * x * x, zero).sum(dtype=torch.float64),
                              torch.where(x > 0, zero, dy * (e.double() - x).float()).sum(dtype=torch.float64)]).float()
    elif case["act"] == "gelu":
        slope = 0.5 * torch.erfc(x * -math.sqrt(0.5)) + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2 * math.pi))
    else:
        t = torch.tanh(st["alpha"][0] * x)
        slope = st["alpha"][0] * (1 - t * t)
        dalpha = (dy * x * (1 - t * t)).sum(dtype=torch.float64).float().reshape(1)
    dx = (dy * slope).to(torch.bfloat16)
    out = {"q": _cast(dx.float(), st["scale"], E5M2), "amax": dx.abs().amax().float().reshape(1)}
    if dalpha is not None:
        out["dalpha"] = dalpha
    if case["keep"]:
        out["dx"] = dx
    return out


def _exponent(amax, fmt):
    """k of the block's scale 2^k: the largest with amax 2^k <= FP8MAX (= 0.875 * 2^9 or 0.875 * 2^16)."""
    m, e = torch.frexp(amax)
    k = (9 if fmt == E4M3 else 16) - e - (m > 0.875).int()
    return torch.where((amax > 0) & torch.isfinite(amax), k.clamp(-126, 126), torch.zeros_like(k))


def _pow2(k):
    """2^k in 32 bits from its exponent field (-127 < k < 128)."""
    return ((k.int() + 127) << 23).view(torch.float32)


def _blocks(x):
    return torch.nn.functional.pad(x, (0, -x.numel() % BLOCK)).view(-1, BLOCK)


def _block_cast(x, fmt):
    """Codes and scale bytes of blocks of 128, to the nearest; a second moment that is not zero stays above zero."""
    b = _blocks(x)
    k = _exponent(b.abs().amax(dim=1, keepdim=True), fmt)
    y = b * _pow2(k)
    if fmt == E5M2:
        y = torch.where(b > 0, y.clamp(min=2.0 ** -16), y)
    return y.to(FP8_DTYPE[fmt]).view(torch.uint8).reshape(-1)[:x.numel()].contiguous(), (127 - k).to(torch.uint8).reshape(-1)


M32 = 0xFFFFFFFF


def _mix(h):
    """Three rounds of shift and multiplication on 32-bit numbers, kept in 64."""
    h = ((h ^ (h >> 16)) * 0x9E3779B1) & M32
    h = ((h ^ (h >> 15)) * 0x6A09E667) & M32
    h = ((h ^ (h >> 13)) * 0xBB67AE85) & M32
    return h ^ (h >> 16)


def _random(seed, step, tensor, n):
    """A 32-bit random number for each element of a tensor: a hash of the seed, the step, the tensor's number and the element's."""
    key = 0
    for w in (seed & M32, seed >> 32, step & M32, step >> 32, tensor):
        key = _mix((key + 0x9E3779B9 + w) & M32)
    i = torch.arange(n, device="cuda")
    return _mix((i & M32) ^ _mix(((i >> 32) + key) & M32))


def _round_by(y, r, fmt):
    """Magnitudes to one of the two codes beside them: up where the places dropped, plus the random number of as many bits, carry."""
    drop, low = (20, 2.0 ** -6) if fmt == E4M3 else (21, 2.0 ** -14)
    r = (r & 0xFFFFF if fmt == E4M3 else r >> 11).int()
    a = y.abs()
    small = a < low
    a = torch.where(small, a + low, a)
    a = ((a.view(torch.int32) + r) & -(1 << drop)).view(torch.float32)
    return torch.copysign(torch.where(small, a - low, a), y)


def _states_cast(x, r, fmt):
    b, n = _blocks(x), x.numel()
    k = _exponent(b.abs().amax(dim=1, keepdim=True), fmt)
    y = _round_by(b * _pow2(k), _blocks(r), fmt)
    if fmt == E5M2:
        y = torch.where(b > 0, y.clamp(min=2.0 ** -16), y)
    return y.to(FP8_DTYPE[fmt]).view(torch.uint8).reshape(-1)[:n], (127 - k).to(torch.uint8).reshape(-1)


def _states_values(q, s, fmt):
    return (_blocks(q).view(FP8_DTYPE[fmt]).float() * _pow2(s.int() - 127)[:, None]).reshape(-1)[:q.numel()]


def _span(st, i):
    a, n = st["at"][i], st["n"][i]
    return slice(a, a + n), slice(a // BLOCK, (a + n + BLOCK - 1) // BLOCK)


def _adamw_out(st):
    out = {"p": st["p"], "master": st["master"], "m": st["m"], "v": st["v"], "ms": st["ms"], "vs": st["vs"]}
    if st["case"]["states"] == "fp8":
        out["m"], out["v"] = st["m"].view(FP8_DTYPE[E4M3]), st["v"].view(FP8_DTYPE[E5M2])
    return {k: v for k, v in out.items() if v is not None}


def _adamw_plain(st):
    case, t, fp8 = st["case"], st["step"], st["case"]["states"] == "fp8"
    norm = st["sumsq"].sqrt()
    c = torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm)).float()
    rate, root = LR / (1 - BETA1 ** t), 1 / math.sqrt(1 - BETA2 ** t)
    for i in range(len(st["n"])):
        e, b = _span(st, i)
        g = st["g"][e].float() * c
        m, v = (_states_values(st["m"][e], st["ms"][b], E4M3), _states_values(st["v"][e], st["vs"][b], E5M2)) if fp8 else (st["m"][e], st["v"][e])
        m, v = m * BETA1 + g * (1 - BETA1), v * BETA2 + g * g * (1 - BETA2)
        p = st["master"][e] if case["master"] else st["p"][e].float()
        p = p * (1 - LR * st["decay"][i]) - m * rate / (v.sqrt() * root + EPS)
        if fp8 or not case["master"]:
            r = _random(st["seed"], t, i, st["n"][i])
        if case["master"]:
            st["master"][e] = p
            st["p"][e] = p.to(torch.bfloat16)
        else:       # up where the sixteen places dropped and as many random bits carry
            st["p"][e] = ((p.view(torch.int32) + (((r * 0x9E3779B1) & M32) >> 16).int()) & -65536).view(torch.float32).to(torch.bfloat16)
        if fp8:
            st["m"][e], st["ms"][b] = _states_cast(m, r, E4M3)
            st["v"][e], st["vs"][b] = _states_cast(v, r, E5M2)
        else:
            st["m"][e], st["v"][e] = m, v
    return _adamw_out(st)


PLAIN = {"rope": _rope_plain, "rope_grad": _rope_grad_plain, "postnorm_grad": _postnorm_grad_plain, "act_grad": _act_grad_plain, "adamw": _adamw_plain}


# ---------------------------------------------------------------------------------------------- the framework's calls
def _kept(st, name, make):
    """What the program keeps between its calls: a workspace, the array of descriptions of tensors that stay in place."""
    if name not in st["kept"]:
        st["kept"][name] = make()
    return st["kept"][name]


def _room(size):
    return torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")


def _run_own(st):
    from paper_2505_20524_amd import fog
    case, kind = st["case"], st["case"]["kind"]
    if kind == "rope":
        def jobs():
            return fog.make_rope_jobs([dict(x=st["x"][:, :, first:first + n], q=st["q"][i].transpose(1, 2), scale=st["scale"][i], amax=st["amax"][i],
                                            rotate=turned, gain=1.0 if turned and case["norm"] else 0.0) for i, (first, n, turned) in enumerate(_heads(case))])
        fog.rope_quantize(_kept(st, "jobs", jobs), st["table"], _kept(st, "ws", lambda: _room(fog.rope_workspace())), layout=case["layout"], positions=st["pos"])
        return {"q": [q.view(FP8_DTYPE[E4M3]) for q in st["q"]], "amax": st["amax"]}
    if kind == "rope_grad":
        def jobs():
            cut = lambda t, first, n: None if t is None else t[:, :, first:first + n]  # noqa: E731
            return fog.make_rope_grad_jobs([dict(dy=dy.transpose(1, 2), x=cut(st["x"], first, n) if turned and case["norm"] else None, dx=cut(st["dx"], first, n),
                                                 q=cut(st["q"], first, n), scale=st["scale"], amax=st["amax"][0], rotate=turned,
                                                 gain=1.0 if turned and case["norm"] else 0.0) for (first, n, turned), dy in zip(_heads(case), st["dy"])])
        fog.rope_grad(_kept(st, "jobs", jobs), st["table"], _kept(st, "ws", lambda: _room(fog.rope_workspace())), layout=case["layout"], positions=st["pos"])
        out = {"q": st["q"].view(FP8_DTYPE[E5M2]), "amax": st["amax"][0]}
        if case["keep"]:
            out["dx"] = st["dx"]
        return out
    if kind == "postnorm_grad":
        ws = _kept(st, "ws", lambda: _room(fog.postnorm_residual_grad_workspace(case["rows"], case["cols"])))
        fog.postnorm_residual_grad(st["dres"], st["y"], st["gamma"], E5M2, st["scale"], st["dgamma"], ws, dbranch=st["dbranch"], dstream=st["dstream"],
                                   dy=st["dy"], q=st["q"], amax_out=st["amax"])
        out = {"q": st["q"].view(FP8_DTYPE[E5M2]), "amax": st["amax"], "dgamma": st["dgamma"], "dstream": st["dstream"], "dy": st["dy"]}
        return {k: v for k, v in out.items() if v is not None}
    if kind == "act_grad":
        ws, more = _kept(st, "ws", lambda: _room(fog.act_grad_workspace())), {"dx": st["dx"], "q": st["q"], "amax_out": st["amax"]}
        if case["act"] == "xielu":
            fog.xielu_grad(st["x"], st["dy"], *st["alpha"], E5M2, st["scale"], ws, dalpha=st["dalpha"], **more)
        elif case["act"] == "tanh":
            fog.tanh_grad(st["x"], st["dy"], *st["alpha"], E5M2, st["scale"], ws, dalpha=st["dalpha"], **more)
        else:
            fog.gelu_grad(st["x"], st["dy"], E5M2, st["scale"], ws, **more)
        out = {"q": st["q"].view(FP8_DTYPE[E5M2]), "amax": st["amax"], "dalpha": st["dalpha"], "dx": st["dx"]}
        return {k: v for k, v in out.items() if v is not None}

    def jobs():
        items = []
        for i in range(len(st["n"])):
            e, b = _span(st, i)
            items.append(dict(p=st["p"][e], g=st["g"][e], m=st["m"][e], v=st["v"][e], master=st["master"][e] if case["master"] else None,
                              m_scale=st["ms"][b] if st["ms"] is not None else None, v_scale=st["vs"][b] if st["vs"] is not None else None,
                              weight_decay=st["decay"][i]))
        return fog.make_adamw_jobs(items)
    fog.adamw(_kept(st, "jobs", jobs), LR, st["step"], beta1=BETA1, beta2=BETA2, eps=EPS, seed=st["seed"], sumsq=st["sumsq"], max_norm=MAX_NORM)
    return _adamw_out(st)


def run(state):
    return _run_own(state) if own else PLAIN[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------------------------- work
def work(case):
    kind = case["kind"]
    if kind in ("rope", "rope_grad"):
        tokens, D, turned = case["B"] * case["S"], case["D"], case["H"] + case["Hkv"]
        n = tokens * (turned + case["Hkv"]) * D
        table = 4 * case["rot"] * (tokens if case["given"] else case["S"]) + (4 * tokens if case["given"] else 0)
        if kind == "rope":
            return {"bytes": 3 * n + table, "flops": tokens * turned * (3 * case["rot"] + (3 * D if case["norm"] else 0))}
        return {"bytes": n * (5 if case["keep"] else 3) + (2 * tokens * turned * D if case["norm"] else 0) + table,
                "flops": tokens * turned * (3 * case["rot"] + (7 * D if case["norm"] else 0))}
    n = case["rows"] * case["cols"] if "rows" in case else 0
    if kind == "postnorm_grad":
        return {"bytes": n * (5 + (4 if case["branch"] else 0) + (2 if case["keep"] else 0)) + 8 * case["cols"], "flops": 10 * n}
    if kind == "act_grad":
        return {"bytes": n * (7 if case["keep"] else 5), "flops": 10 * n}
    n = case["layers"] * sum(math.prod(s) for s in _layer(case["hidden"], case["inner"])) + case["hidden"]
    each = (2 if case["grad"] == "bf16" else 4) + (10 if case["master"] else 4) + (16 if case["states"] == "f32" else 4)
    return {"bytes": n * each, "flops": 14 * n}


# ---------------------------------------------------------------------------------------------- the same in 64 bits
def _grid64(v, fmt):
    """64-bit values rounded to the FP8 grid, ties to even, saturating: 3 or 2 places behind the leading bit, fewer below the smallest normal."""
    places, low = (3, -6) if fmt == E4M3 else (2, -14)
    step = torch.exp2((torch.frexp(v).exponent - 1).clamp(min=low).double() - places)
    return (torch.round(v / step) * step).clamp(-FP8_MAX[fmt], FP8_MAX[fmt])


def _kept64(v):
    """The bfloat16 that a 64-bit gradient is stored and cast as."""
    return v.to(torch.bfloat16).double()


def _pairs64(case):
    """For every dimension of a head its partner and the sign with which the partner's sine enters, and its pair; unturned ones are their own partner."""
    D, rot, half = case["D"], case["rot"], case["rot"] // 2
    d = torch.arange(D, device="cuda")
    if case["layout"] == HALF:
        first, pair = d < half, d % max(half, 1)
        partner = torch.where(first, d + half, d - half)
    else:
        first, pair = d % 2 == 0, d // 2
        partner = torch.where(first, d + 1, d - 1)
    on = d < rot
    return torch.where(on, partner, d), torch.where(on, torch.where(first, -1.0, 1.0), 0.0).double(), torch.where(on, pair, torch.zeros_like(d)), on


def _turn64(st, z, back):
    case = st["case"]
    B, S, half = case["B"], case["S"], case["rot"] // 2
    pos = torch.arange(S, device="cuda").repeat(B).view(B, S) if st["pos"] is None else st["pos"].long()
    partner, sign, pair, on = _pairs64(case)
    row = st["table"].double()[pos.clamp(0, case["positions"] - 1)]
    c = torch.where(on, row[:, :, :half][:, :, pair], torch.ones((), dtype=torch.float64, device="cuda"))
    s = row[:, :, half:][:, :, pair] * (-sign if back else sign)
    there = (pos >= 0) & (pos < case["positions"])
    return (z * c[:, :, None] + z[..., partner] * s[:, :, None]) * there[:, :, None, None]


def exact(case, seed):
    kind = case["kind"]
    if kind == "adamw":
        return _adamw64(prepare(case, seed))
    st = prepare(case, seed)
    if kind == "rope":
        q, amax = [], []
        for i, (first, n, turned) in enumerate(_heads(case)):
            y = st["x"][:, :, first:first + n].double()
            if turned:
                if case["norm"]:
                    y = y * (case["D"] / (y * y).sum(-1, keepdim=True)).sqrt()
                y = _turn64(st, y, False)
            amax.append(y.abs().max().reshape(1))
            q.append(_grid64(y * st["scale"][i].double(), E4M3).permute(0, 2, 1, 3).contiguous())
        return {"q": q, "amax": amax}
    if kind == "rope_grad":
        dx = torch.empty(st["x"].shape, dtype=torch.float64, device="cuda")
        for (first, n, turned), dy in zip(_heads(case), st["dy"]):
            d = dy.double().permute(0, 2, 1, 3)
            if turned:
                d = _turn64(st, d, True)
                if case["norm"]:
                    x = st["x"][:, :, first:first + n].double()
                    r = (x * x).mean(-1, keepdim=True).sqrt()
                    d = d / r - x * (x * d).mean(-1, keepdim=True) / r ** 3
            dx[:, :, first:first + n] = d
        kept = _kept64(dx)
        return {"q": _grid64(kept * st["scale"].double(), E5M2), "amax": kept.abs().max().reshape(1), **({"dx": dx} if case["keep"] else {})}
    if kind == "postnorm_grad":
        y, G = st["y"].double(), st["dres"].double()
        if case["branch"]:
            G = G + st["dbranch"].double()
        stream, G = G, _kept64(G)
        r = (y * y).mean(1, keepdim=True).sqrt()
        t = G * st["gamma"].double()
        dy = t / r - y * (t * y).mean(1, keepdim=True) / r ** 3
        kept = _kept64(dy)
        out = {"q": _grid64(kept * st["scale"].double(), E5M2), "amax": kept.abs().max().reshape(1), "dgamma": (G * y / r).sum(0)}
        if case["branch"]:
            out["dstream"] = stream
        if case["keep"]:
            out["dy"] = dy
        return out
    x, dy = st["x"].double(), st["dy"].double()
    out = {}
    if case["act"] == "xielu":
        ap, an = st["alpha"]
        e = torch.expm1(x)
        slope = torch.where(x > 0, 2 * ap * x, an * e) + 0.5
        out["dalpha"] = torch.stack([(dy * x * x)[x > 0].sum(), (dy * (e - x))[x <= 0].sum()])
    elif case["act"] == "gelu":
        slope = torch.special.ndtr(x) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    else:
        a = st["alpha"][0]
        slope = a / torch.cosh(a * x) ** 2
        out["dalpha"] = (dy * x / torch.cosh(a * x) ** 2).sum().reshape(1)
    dx = dy * slope
    kept = _kept64(dx)
    out.update(q=_grid64(kept * st["scale"].double(), E5M2), amax=kept.abs().max().reshape(1))
    if case["keep"]:
        out["dx"] = dx
    return out


def _values64(q, s, fmt):
    at = torch.arange(q.numel(), device="cuda") // BLOCK
    return q.view(FP8_DTYPE[fmt]).double() * torch.exp2(s.double() - 127.0)[at]


def _adamw64(st):
    """Parameters before they are rounded to bfloat16, and 32-bit states; a state in 8 bits is one of two codes by a random number, which has no value of its own."""
    case, t = st["case"], st["step"]
    norm = math.sqrt(st["sumsq"].item())
    c = MAX_NORM / norm if norm > MAX_NORM else 1.0
    out = {"p": st["p"].double(), "master": st["master"].double() if case["master"] else None,
           "m": None, "v": None, "ms": None, "vs": None}
    if case["states"] == "f32":
        out["m"], out["v"] = st["m"].double(), st["v"].double()
    for i in range(len(st["n"])):
        e, b = _span(st, i)
        g = st["g"][e].double() * c
        if case["states"] == "f32":
            m, v = st["m"][e].double(), st["v"][e].double()
        else:
            m, v = _values64(st["m"][e], st["ms"][b], E4M3), _values64(st["v"][e], st["vs"][b], E5M2)
        m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g * g
        if case["states"] == "f32":
            out["m"][e], out["v"][e] = m, v
        p = st["master" if case["master"] else "p"][e].double()
        p = p - LR * st["decay"][i] * p - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
        out["p"][e] = p
        if case["master"]:
            out["master"][e] = p
    return {k: v for k, v in out.items() if v is not None or (k in ("ms", "vs") and case["states"] == "fp8")}
