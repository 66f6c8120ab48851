"""GPU parity: rotary positions with QK norm and cast, their backward, and the table, against float64."""
import math

import numpy as np
import pytest
import torch

from oracle import bf16, fp8, rope
from paper_2505_20524_amd import fog

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
LAYOUTS = [fog.HALF, fog.INTERLEAVED]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(seed, *shape, std=1.0):
    return (torch.randn(shape, device="cuda", generator=gen(seed)) * std).bfloat16()


def one(v):
    return torch.full((1,), float(v), device="cuda")


def u8(*shape, fill=0xA5):
    return torch.full(shape, fill, dtype=torch.uint8, device="cuda")


def room():
    return u8(fog.rope_workspace(), fill=0xFF)


def h64(t):
    return t.double().cpu().numpy()


def make_table(positions, rot, **more):
    t = torch.empty((positions, rot), device="cuda")
    fog.rope_table(t, **more)
    return t


def pos_of(B, S, positions, offset=0):
    return np.arange(S)[None].repeat(B, 0) + offset if positions is None else positions.cpu().numpy().reshape(B, S)


def check_forward(x, q, amax, scale, table, pos, layout, gain, fmt, rotate=True):
    """Codes of a binary32 number within the tolerance of the float64 one: between the codes of its two ends."""
    y, size = rope.forward(h64(x), h64(table) if rotate and table is not None and table.shape[1] else None, pos, layout, gain)
    # norm: 16 sums in a lane and 6 between lanes (half of it behind the root), the mean, the root, the quotient, the product: 15; turn: 2; scaling: 1
    e = ((15 if gain else 0) + 4) * 1.01 * U * size
    if not gain:
        e = np.where(y == h64(x), 0.0, e)          # not turned, or by an angle of 0: nothing is rounded before the scaling
    s = float(scale.item())
    lo, hi = (fp8.decode(fp8.encode_sat(((y + d) * s).astype(np.float32), fmt), fmt) for d in (-e, e))
    got = fp8.decode(q.cpu().numpy(), fmt)
    assert np.all(got >= lo) and np.all(got <= hi), np.argwhere((got < lo) | (got > hi))[:5]
    if e.size:
        assert (lo != hi).mean() <= 1e-3 + 2.0 / e.size
    if amax is not None:
        top = np.abs(y).max() if y.size else 0.0
        assert abs(amax.item() - top) <= (e.max() if y.size else 0.0)


def check_backward(dy, x, dx, q, amax, scale, table, pos, layout, gain, fmt, rotate=True):
    want, size, along = rope.backward(h64(dy), None if x is None else h64(x), h64(table) if rotate and table is not None and table.shape[1] else None, pos, layout, gain)
    # turn 2; sums of 22, twice, and their quotient in `along` (47 with the turn's own), the difference 1, the norm's factor 15, the product 1
    e = U * 1.01 * (2 * size if not gain else 19 * size + 64 * along) + 2.0 ** -140
    got = h64(dx)
    lo, hi = bf16.f64_round(want - e), bf16.f64_round(want + e)
    assert np.all(got >= lo) and np.all(got <= hi), np.argwhere((got < lo) | (got > hi))[:5]
    if q is not None:
        assert np.array_equal(q.cpu().numpy(), fp8.encode_sat(np.float32(got) * np.float32(scale.item()), fmt))
    if amax is not None:
        assert amax.item() == (np.abs(got).max() if got.size else 0.0)


SHAPES = [  # B, S, heads, D, rot
    (1, 1, 1, 128, 128), (2, 3, 4, 128, 128), (1, 70, 5, 128, 64), (3, 33, 2, 64, 64), (2, 17, 3, 80, 20), (1, 9, 3, 96, 96), (2, 5, 2, 192, 96), (1, 40, 3, 256, 256),
    (2, 7, 1, 512, 512), (1, 3, 2, 1008, 18), (1, 6, 2, 1008, 1008), (2, 4, 3, 7, 6), (1, 5, 1, 1, 0), (2, 3, 2, 2, 2), (1, 130, 1, 32, 30), (1, 11, 17, 130, 2), (2, 5, 2, 288, 32)]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("B,S,H,D,rot", SHAPES)
@pytest.mark.parametrize("gain,fmt", [(0.0, fog.E4M3), (1.0, fog.E4M3), (2.5, fog.E5M2)])
def test_forward(B, S, H, D, rot, layout, gain, fmt):
    x, q = normal(B + S + D, B, S, H, D), u8(B, H, S, D)
    scale, amax = one(448.0 / 8 if fmt == fog.E4M3 else 1000.0), one(-1)
    table = make_table(S + 3, rot)
    fog.rope_quantize(fog.make_rope_jobs([dict(x=x, q=q.transpose(1, 2), scale=scale, amax=amax, gain=gain, fmt=fmt)]), table, room(), layout=layout, offset=2)
    check_forward(x, q.transpose(1, 2), amax, scale, table, pos_of(B, S, None, 2), layout, gain, fmt)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("B,S,H,D,rot", SHAPES)
@pytest.mark.parametrize("gain,fmt", [(0.0, fog.E5M2), (1.0, fog.E5M2), (2.5, fog.E4M3)])
def test_backward(B, S, H, D, rot, layout, gain, fmt):
    dy, x = normal(B + S + D, B, H, S, D, std=1e-3).transpose(1, 2), normal(B + S + D + 1, B, S, H, D)
    dx, q = normal(0, B, S, H, D), u8(B, S, H, D)
    scale, amax = one(57344.0 / 8e-3 if fmt == fog.E5M2 else 1e4), one(-1)
    table = make_table(S + 3, rot)
    item = dict(dy=dy, x=x if gain else None, dx=dx, q=q, scale=scale, amax=amax, gain=gain, fmt=fmt)
    fog.rope_grad(fog.make_rope_grad_jobs([item]), table, room(), layout=layout, offset=1)
    check_backward(dy, x, dx, q, amax, scale, table, pos_of(B, S, None, 1), layout, gain, fmt)
    # without dx the same codes and abs-max, without codes the same dx
    q2, amax2, dx2 = u8(B, S, H, D), one(-1), torch.zeros_like(dx)
    fog.rope_grad(fog.make_rope_grad_jobs([{**item, "dx": None, "q": q2, "amax": amax2}]), table, room(), layout=layout, offset=1)
    fog.rope_grad(fog.make_rope_grad_jobs([{**item, "dx": dx2, "q": None, "scale": None, "amax": None}]), table, layout=layout, offset=1)
    assert torch.equal(q2, q) and amax2.item() == amax.item() and torch.equal(dx2, dx)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("B,S,H,D,rot", [(2, 9, 3, 96, 32), (1, 355, 9, 128, 96), (3, 5, 2, 320, 96), (2, 45, 5, 992, 512), (5, 67, 7, 64, 64), (1, 300, 3, 32, 0)])
def test_stretches_of_whole_thirty_twos(B, S, H, D, rot, layout):
    """Runs half a stretch apart, turned or not; groups of tokens that eight does not divide, and jobs of one and of several segments of heads; codes at odd addresses."""
    x, y = normal(B + S + D, B, S, H, D), normal(B + S + D + 1, B, S, H, D)
    table, scale, amaxs = make_table(S, rot), one(448.0 / 8), [one(-1) for _ in range(4)]
    outs = [u8(B * H * S * D + 16) for _ in range(2)]
    q, v = (o[3:3 + B * H * S * D].view(B, H, S, D).transpose(1, 2) for o in outs)
    fog.rope_quantize(fog.make_rope_jobs([dict(x=x, q=q, scale=scale, amax=amaxs[0], gain=1.0), dict(x=y, q=v, scale=scale, amax=amaxs[1], rotate=False)]), table, room(),
                      layout=layout)
    check_forward(x, q, amaxs[0], scale, table, pos_of(B, S, None), layout, 1.0, fog.E4M3)
    check_forward(y, v, amaxs[1], scale, table, pos_of(B, S, None), layout, 0.0, fog.E4M3, rotate=False)
    for o in outs:
        assert bool((o[:3] == 0xA5).all()) and bool((o[3 + B * H * S * D:] == 0xA5).all())
    dy, dx, dq, sg = normal(B + S + D + 2, B, H, S, D, std=1e-3).transpose(1, 2), normal(0, B, S, H, D), u8(B, S, H, D), one(57344.0 / 8e-3)
    fog.rope_grad(fog.make_rope_grad_jobs([dict(dy=dy, x=x, dx=dx, q=dq, scale=sg, amax=amaxs[2], gain=1.0)]), table, room(), layout=layout)
    check_backward(dy, x, dx, dq, amaxs[2], sg, table, pos_of(B, S, None), layout, 1.0, fog.E5M2)


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_positions_of_every_kind(dtype, layout):
    """Positions in any order, some outside the table, in a table of far positions with an amplitude."""
    B, S, H, D, rot = 2, 50, 3, 128, 96
    table = make_table(300, rot, first=1_000_000, amplitude=1.2, factor=8.0, low=1.0, high=32.0, original=4096)
    pos = torch.randint(0, 300, (B, S), device="cuda", generator=gen(1), dtype=dtype)
    pos[0, 3], pos[0, 9], pos[1, 0], pos[1, 49], pos[1, 7], pos[0, 49] = -1, 300, 299, 0, -2 ** 31, 2 ** 31 - 1
    if dtype == torch.int64:
        pos[0, 4], pos[0, 5] = 1 << 32, -(1 << 40)          # no row either, though their low words are
    x, q, scale, amax = normal(2, B, S, H, D), u8(B, S, H, D), one(30.0), one(-1)
    fog.rope_quantize(fog.make_rope_jobs([dict(x=x, q=q, scale=scale, amax=amax, gain=1.0)]), table, room(), layout=layout, positions=pos)
    check_forward(x, q, amax, scale, table, pos_of(B, S, pos), layout, 1.0, fog.E4M3)
    away = (pos < 0) | (pos >= 300)
    assert bool((q[away] == 0).all()) and bool((q[~away] != 0).any(-1).all())
    dy, dx, g = normal(3, B, S, H, D), normal(0, B, S, H, D), u8(B, S, H, D)
    fog.rope_grad(fog.make_rope_grad_jobs([dict(dy=dy, x=x, dx=dx, q=g, scale=scale, amax=amax, gain=1.0)]), table, room(), layout=layout, positions=pos)
    check_backward(dy, x, dx, g, amax, scale, table, pos_of(B, S, pos), layout, 1.0, fog.E5M2)
    assert bool((dx[away] == 0).all()) and bool((g[away] == 0).all())


def test_offsets_beyond_the_table():
    x, q, table = normal(4, 1, 8, 2, 64), u8(1, 8, 2, 64), make_table(6, 64)
    for offset, rows in ((-3, slice(3, 8)), (2, slice(0, 4)), (100, slice(0, 0)), (-(1 << 40), slice(0, 0)), (1 << 40, slice(0, 0))):
        q.fill_(0xA5)
        fog.rope_quantize(fog.make_rope_jobs([dict(x=x, q=q, scale=one(40.0))]), table, offset=offset)
        check_forward(x, q, None, one(40.0), table, pos_of(1, 8, None, offset), fog.HALF, 0.0, fog.E4M3)
        assert bool((q[:, rows] != 0).any(-1).all()) or rows == slice(0, 0)


def fused(seed, B, S, H, Hkv, D, skew=0, pad=0):
    """Q, K, V as ranges of a projection's result with `pad` columns between tokens, `skew` elements off its alignment."""
    W = (H + 2 * Hkv) * D + pad
    flat = normal(seed, B * S * W + skew)[skew:]
    x = flat.view(B, S, W)
    cut = lambda a, n: x[:, :, a * D:(a + n) * D].unflatten(2, (n, D))  # noqa: E731
    return flat, (cut(0, H), cut(H, Hkv), cut(H + Hkv, Hkv))


@pytest.mark.parametrize("skew,pad", [(0, 0), (1, 0), (3, 5), (8, 8)])
@pytest.mark.parametrize("D,rot", [(128, 128), (80, 20), (64, 32)])
def test_fused_projection_to_heads_and_back(skew, pad, D, rot):
    B, S, H, Hkv = 2, 37, 4, 2
    flat, xs = fused(5, B, S, H, Hkv, D, skew, pad)
    table = make_table(S, rot)
    scales, amaxs = [one(50.0), one(40.0), one(30.0)], [one(-1) for _ in range(3)]
    outs = [u8(B * h * S * D + 40) for h in (H, Hkv, Hkv)]
    qs = [o[8 + skew:8 + skew + B * h * S * D].view(B, h, S, D).transpose(1, 2) for o, h in zip(outs, (H, Hkv, Hkv))]
    gains = [1.0, 1.0, 0.0]
    fog.rope_quantize(fog.make_rope_jobs([dict(x=x, q=q, scale=s, amax=a, gain=g, rotate=g > 0) for x, q, s, a, g in zip(xs, qs, scales, amaxs, gains)]), table, room())
    for x, q, s, a, g, o in zip(xs, qs, scales, amaxs, gains, outs):
        check_forward(x, q, a, s, table, pos_of(B, S, None), fog.HALF, g, fog.E4M3, rotate=g > 0)
        assert bool((o[:8 + skew] == 0xA5).all()) and bool((o[8 + skew + q.numel():] == 0xA5).all())
    # V: the plain cast's codes
    v, want = xs[2].contiguous().view(-1, D), u8(B * S * Hkv, D)
    fog.quantize(v, fog.E4M3, scales[2], q=want)
    assert torch.equal(qs[2].reshape(-1, D), want)
    # back into the columns of one matrix with one scale and one abs-max
    W = (H + 2 * Hkv) * D + pad
    dys = [normal(6 + i, B, h, S, D, std=1e-3).transpose(1, 2) for i, h in enumerate((H, Hkv, Hkv))]
    dflat, gflat = torch.full((B * S * W + skew + 16,), 9.0, dtype=torch.bfloat16, device="cuda"), u8(B * S * W + skew + 16)
    cut = lambda t, a, n: t[skew:skew + B * S * W].view(B, S, W)[:, :, a * D:(a + n) * D].unflatten(2, (n, D))  # noqa: E731
    scale, amax = one(57344.0 / 8e-3), one(-1)
    parts = [(0, H), (H, Hkv), (H + Hkv, Hkv)]
    items = [dict(dy=dy, x=x if g else None, dx=cut(dflat, *p), q=cut(gflat, *p), scale=scale, amax=amax, gain=g, rotate=g > 0)
             for dy, x, p, g in zip(dys, xs, parts, gains)]
    fog.rope_grad(fog.make_rope_grad_jobs(items), table, room())
    tops = []
    for item, x, g in zip(items, xs, gains):
        check_backward(item["dy"], x, item["dx"], item["q"], None, scale, table, pos_of(B, S, None), fog.HALF, g, fog.E5M2, rotate=g > 0)
        tops.append(item["dx"].abs().max().item())
    assert amax.item() == max(tops)
    for t, left in ((dflat, 9.0), (gflat, 0xA5)):
        assert bool((t[:skew] == left).all()) and bool((t[skew + B * S * W:] == left).all())
        if pad:
            assert bool((t[skew:skew + B * S * W].view(B, S, W)[:, :, W - pad:] == left).all())


def test_single_tokens_are_the_rows_of_a_batch():
    """A decoding step: every sequence at a position of its own, written into its row of a cache; the bits of the whole sequence's call."""
    B, S, H, D = 5, 40, 3, 128
    x, table = normal(7, B, S, H, D), make_table(S, D)
    whole, cache = u8(B, H, S, D), u8(B, H, S, D, fill=0)
    fog.rope_quantize(fog.make_rope_jobs([dict(x=x, q=whole.transpose(1, 2), scale=one(40.0), gain=1.0)]), table)
    for s in range(S):
        item = dict(x=x[:, s:s + 1], q=cache[:, :, s:s + 1].transpose(1, 2), scale=one(40.0), gain=1.0)
        if s % 2:
            fog.rope_quantize(fog.make_rope_jobs([item]), table, offset=s)
        else:
            fog.rope_quantize(fog.make_rope_jobs([item]), table, positions=torch.full((B, 1), s, device="cuda"))
    assert torch.equal(cache, whole)


def test_inputs_that_repeat():
    """A head that is given to several (strides of 0), and a whole batch of one token."""
    x = normal(8, 1, 6, 1, 64).expand(3, 6, 4, 64)
    q, table = u8(3, 6, 4, 64), make_table(6, 64)
    fog.rope_quantize(fog.make_rope_jobs([dict(x=x, q=q, scale=one(40.0), gain=1.0)]), table)
    check_forward(x, q, None, one(40.0), table, pos_of(3, 6, None), fog.HALF, 1.0, fog.E4M3)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("gain", [0.0, 1.0])
def test_zeros_infinities_and_nan_stay_in_their_vectors(layout, gain):
    B, S, H, D, rot = 1, 12, 2, 64, 32
    x, table = normal(9, B, S, H, D), make_table(S, rot)
    clean, q, amax = u8(B, S, H, D), u8(B, S, H, D), one(-1)
    call = lambda t, o: fog.rope_quantize(fog.make_rope_jobs([dict(x=t, q=o, scale=one(40.0), gain=gain, amax=amax)]), table, room(), layout=layout)  # noqa: E731
    call(x, clean)
    bad = x.clone()
    bad[0, 2, 1] = 0.0
    bad[0, 4, 0, 5] = float("nan")
    bad[0, 6, 1, 60] = float("inf")          # behind the turned part
    call(bad, q)
    assert math.isnan(amax.item())
    same = torch.ones((S, H), dtype=torch.bool)
    same[2, 1] = same[4, 0] = same[6, 1] = False
    assert torch.equal(q[0][same], clean[0][same])
    assert bool((q[0, 2, 1] & 0x7F == 0).all())
    v = fp8.decode(q[0, 4, 0].cpu().numpy(), fog.E4M3)
    if gain:
        assert np.isnan(v).all()
        w = fp8.decode(q[0, 6, 1].cpu().numpy(), fog.E4M3)       # x / inf: zeros, and inf / inf
        assert np.isnan(w[60]) and not np.delete(w, 60).any()
    else:
        partner = {fog.HALF: 21, fog.INTERLEAVED: 4}[layout]
        assert set(np.flatnonzero(np.isnan(v))) == {5, partner}
        assert (q[0, 6, 1] != clean[0, 6, 1]).nonzero().tolist() == [[60]] and q[0, 6, 1, 60].item() == 0x7E
    bad[0, 4, 0, 5] = 1.0
    bad[0, 6, 1, 60] = 1.0
    call(bad, q)
    assert math.isfinite(amax.item())
    # backward: a vector of zeros has no direction; a NaN shows in the abs-max
    dy, dx = normal(10, B, S, H, D), normal(0, B, S, H, D)
    back = lambda g: fog.rope_grad(fog.make_rope_grad_jobs([dict(dy=g, x=bad if gain else None, dx=dx, amax=amax, gain=gain)]), table, room(), layout=layout)  # noqa: E731
    back(dy)
    assert math.isfinite(amax.item()) and bool(torch.isfinite(dx).all())
    if gain:
        assert bool((dx[0, 2, 1] == 0).all())
    keep = dx.clone()
    dy[0, 3, 1, 50] = float("nan")
    back(dy)
    assert math.isnan(amax.item())
    same = torch.ones((S, H), dtype=torch.bool)
    same[3, 1] = False
    assert torch.equal(dx[0][same], keep[0][same]) and math.isnan(dx[0, 3, 1, 50].item())


def test_empty_jobs_and_lengths():
    amax, table = one(5.0), make_table(4, 64)
    fog.rope_quantize(fog.make_rope_jobs([dict(x=normal(0, 2, 0, 3, 64), q=u8(2, 0, 3, 64), scale=one(1), amax=amax)]), table, room())
    assert amax.item() == 0.0
    x, q, a0, a1 = normal(11, 2, 4, 3, 64), u8(2, 4, 3, 64), one(5.0), one(5.0)
    jobs = fog.make_rope_jobs([dict(x=x[:, :, :0], q=q[:, :, :0], scale=one(1), amax=a0), dict(x=x, q=q, scale=one(40.0), amax=a1)])
    fog.rope_quantize(jobs, table, room())
    check_forward(x, q, a1, one(40.0), table, pos_of(2, 4, None), fog.HALF, 0.0, fog.E4M3)
    assert a0.item() == 0.0
    fog.rope_quantize(fog.make_rope_jobs([]), table)


def test_eight_jobs_with_common_maxima():
    B, S, D = 2, 9, 64
    table, a, b = make_table(S, D), one(-1), one(-1)
    xs = [normal(20 + i, B, S, 1 + i, D, std=1.0 + i) for i in range(8)]
    qs = [u8(B, S, 1 + i, D) for i in range(8)]
    fog.rope_quantize(fog.make_rope_jobs([dict(x=x, q=q, scale=one(20.0), amax=(a, b, None)[i % 3], rotate=i % 2 == 0) for i, (x, q) in enumerate(zip(xs, qs))]), table, room())
    tops = []
    for i, (x, q) in enumerate(zip(xs, qs)):
        check_forward(x, q, None, one(20.0), table, pos_of(B, S, None), fog.HALF, 0.0, fog.E4M3, rotate=i % 2 == 0)
        tops.append(np.abs(rope.forward(h64(x), h64(table) if i % 2 == 0 else None, pos_of(B, S, None), fog.HALF)[0]).max())
    for got, want in ((a, max(tops[0::3])), (b, max(tops[1::3]))):
        assert abs(got.item() - want) <= 8 * U * want


def test_more_tokens_than_workgroups_and_many_heads():
    """Two million tokens of one short vector; four tokens of 20000 heads.  On small whole numbers and quarter turns everything is exact."""
    quarter = torch.tensor([[1.0, 0.0], [0.0, 1.0], [-1.0, 0.0], [0.0, -1.0]], device="cuda").repeat_interleave(8, dim=1)        # rot 16
    for B, S, H in ((2, 1_000_003, 1), (1, 4, 20011)):
        x = torch.randint(-8, 9, (B, S, H, 16), device="cuda", generator=gen(12)).bfloat16()
        pos = torch.randint(0, 4, (B, S), device="cuda", generator=gen(13))
        q, amax = u8(B, S, H, 16), one(-1)
        fog.rope_quantize(fog.make_rope_jobs([dict(x=x, q=q, scale=one(1.0), amax=amax)]), quarter, room(), positions=pos)
        a, b, p = x[..., :8].float(), x[..., 8:].float(), pos[:, :, None, None]
        want = torch.zeros((B, S, H, 16), device="cuda")
        for k, y in enumerate(((a, b), (-b, a), (-a, -b), (b, -a))):
            want = torch.where(p == k, torch.cat(y, -1), want)
        assert torch.equal(q.view(torch.float8_e4m3fn).float(), want) and amax.item() == 8.0
        dx = torch.empty_like(x)
        fog.rope_grad(fog.make_rope_grad_jobs([dict(dy=want.bfloat16(), dx=dx, amax=amax)]), quarter, room(), positions=pos)
        assert torch.equal(dx, x) and amax.item() == 8.0


def test_strides_beyond_2_to_the_32_elements():
    S, H, D = 3, 2, 128
    flat = torch.zeros((1 << 32) + 5000, dtype=torch.bfloat16, device="cuda")
    codes = torch.zeros((1 << 32) + 5000, dtype=torch.uint8, device="cuda")
    view = lambda t: t.as_strided((2, S, H, D), ((1 << 32) + 1, H * D, D, 1))  # noqa: E731
    x, q, table, amax = view(flat), view(codes), make_table(S, D), one(-1)
    x.copy_(normal(14, 2, S, H, D))
    fog.rope_quantize(fog.make_rope_jobs([dict(x=x, q=q, scale=one(40.0), amax=amax, gain=1.0)]), table, room())
    check_forward(x, q, amax, one(40.0), table, pos_of(2, S, None), fog.HALF, 1.0, fog.E4M3)
    assert int((codes != 0).sum()) <= 2 * S * H * D
    dy, g = normal(15, 2, S, H, D), torch.zeros((1 << 32) + 5000, dtype=torch.bfloat16, device="cuda")
    fog.rope_grad(fog.make_rope_grad_jobs([dict(dy=dy, x=x, dx=view(g), amax=amax, gain=1.0)]), table, room())
    check_backward(dy, x, view(g), None, amax, None, table, pos_of(2, S, None), fog.HALF, 1.0, fog.E5M2)


def test_a_step_in_a_graph_and_on_two_streams():
    B, S, H, Hkv, D = 2, 65, 4, 2, 128

    class Pass:
        def __init__(self, seed):
            _, self.x = fused(seed, B, S, H, Hkv, D)
            self.table, self.pos = make_table(200, D), torch.zeros((B, S), dtype=torch.int32, device="cuda")
            self.q = [u8(B, h, S, D) for h in (H, Hkv, Hkv)]
            self.amax, self.dx, self.ws, self.ws2 = [one(-1) for _ in range(4)], normal(0, B, S, H + 2 * Hkv, D), room(), room()
            self.dy = [normal(seed + i, B, h, S, D).transpose(1, 2) for i, h in enumerate((H, Hkv, Hkv))]
            cut = ((0, H), (H, Hkv), (H + Hkv, Hkv))
            self.fwd = fog.make_rope_jobs([dict(x=x, q=q.transpose(1, 2), scale=one(40.0), amax=a, gain=float(i < 2), rotate=i < 2)
                                           for i, (x, q, a) in enumerate(zip(self.x, self.q, self.amax))])
            self.bwd = fog.make_rope_grad_jobs([dict(dy=dy, x=x, dx=self.dx[:, :, a:a + n], amax=self.amax[3], gain=float(i < 2), rotate=i < 2)
                                                for i, (dy, x, (a, n)) in enumerate(zip(self.dy, self.x, cut))])

        def run(self, stream=None):
            fog.rope_quantize(self.fwd, self.table, self.ws, positions=self.pos, stream=stream)
            fog.rope_grad(self.bwd, self.table, self.ws2, positions=self.pos, stream=stream)

        def outputs(self):
            return [t.clone() for t in (*self.q, *self.amax, self.dx)]

    p = Pass(30)
    p.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run()
    for i in range(4):
        p.pos.copy_(torch.randint(-2, 202, (B, S), device="cuda", generator=gen(i)))
        for x in p.x:
            x.copy_(torch.randn(x.shape, device="cuda", generator=gen(100 + i)))
        p.run()
        want = p.outputs()
        torch.cuda.synchronize()
        for t in (*p.q, *p.amax, p.dx):
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(p.outputs(), want))
    ps, want = [Pass(40), Pass(50)], []
    for x in ps:
        x.run()
        want.append(x.outputs())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ps]
    for _ in range(5):
        for x, s in zip(ps, streams):
            x.run(stream=s)
    torch.cuda.synchronize()
    for x, w in zip(ps, want):
        assert all(torch.equal(a, b) for a, b in zip(x.outputs(), w))


@pytest.mark.parametrize("value", [1e-20, 1e-23, 1e-30, 3e17])
def test_very_short_and_long_vectors(value):
    """A norm whose squares still show, and vectors whose squares vanish: zeros in both directions, no infinity and no NaN beside them."""
    x, q, amax, dx = (normal(16, 2, 5, 2, 128).double() * value).bfloat16(), u8(2, 5, 2, 128), one(-1), normal(0, 2, 5, 2, 128)
    x[0, 0, 0, 3], x[0, 1] = 0.0, 0.0
    table = make_table(5, 128)
    fog.rope_quantize(fog.make_rope_jobs([dict(x=x, q=q, scale=one(1e9 if value == 1e-30 else 30.0), amax=amax, gain=1.0)]), table, room())
    assert math.isfinite(amax.item()) and not np.isnan(fp8.decode(q.cpu().numpy(), fog.E4M3)).any()
    dy = normal(17, 2, 5, 2, 128)
    fog.rope_grad(fog.make_rope_grad_jobs([dict(dy=dy, x=x, dx=dx, amax=amax, gain=1.0)]), table, room())
    assert bool(torch.isfinite(dx).all())
    if value in (3e17, 1e-30):
        y, _ = rope.forward(h64(x), h64(table), pos_of(2, 5, None), fog.HALF, 1.0)
        got = fp8.decode(q.cpu().numpy(), fog.E4M3)
        if value == 1e-30:
            assert not got.any() and bool((dx == 0).all())
        else:       # half a step of a code
            assert np.all(np.abs(got / 30.0 - y) <= 2.0 ** -4 * 1.01 * np.abs(y) + 2.0 ** -10 / 30)


@pytest.mark.parametrize("rot", [2, 20, 128, 600])
@pytest.mark.parametrize("first,positions", [(0, 1), (0, 130), (1_000_000, 65), (-40, 80), ((1 << 40), 3)])
@pytest.mark.parametrize("scaling", [{}, dict(base=5e5), dict(factor=4.0), dict(factor=8.0, low=1.0, high=32.0, original=4096.0, amplitude=1.25)])
def test_table(rot, first, positions, scaling):
    table = torch.full((positions + 1, rot), 7.0, device="cuda")
    fog.rope_table(table[:positions], first=first, **scaling)
    p = np.arange(first, first + positions)
    want = rope.table(p, rot, **scaling)
    angle = np.abs(p)[:, None] * np.tile(rope.frequencies(rot, **{k: v for k, v in scaling.items() if k != "amplitude"}), 2)
    # a power of up to 2^19 by its logarithm (two functions and three products of numbers up to 19) and the scaling: 2^-46 of the angle on either side
    tol = U * np.abs(want) + scaling.get("amplitude", 1.0) * (angle * 2.0 ** -45 + 2.0 ** -50)
    assert np.all(np.abs(h64(table[:positions]) - want) <= tol)
    assert bool((table[positions] == 7.0).all())


def test_a_table_of_many_positions():
    table = make_table(131072, 128)
    for p in (0, 1, 4095, 4096, 65535, 131071):
        assert np.abs(h64(table[p]) - rope.table([p], 128)[0]).max() <= U + p * 2.0 ** -45


def test_the_binding_refuses_tensors_of_other_devices():
    x, q, table = normal(1, 1, 4, 2, 64), u8(1, 4, 2, 64), make_table(4, 64)
    for bad in (dict(x=x.cpu()), dict(q=q.cpu()), dict(scale=torch.ones(1)), dict(amax=torch.ones(1))):
        with pytest.raises(ValueError):
            fog.rope_quantize(fog.make_rope_jobs([{**dict(x=x, q=q, scale=one(1.0)), **bad}]), table, room())
    jobs = fog.make_rope_jobs([dict(x=x, q=q, scale=one(1.0))])
    for call in (lambda: fog.rope_quantize(jobs, table.cpu()), lambda: fog.rope_quantize(jobs, table, positions=torch.zeros((1, 4), dtype=torch.int64)),
                 lambda: fog.rope_quantize(jobs, table, positions=torch.zeros((1, 3), dtype=torch.int64, device="cuda")),
                 lambda: fog.rope_quantize(jobs, table.double()), lambda: fog.rope_table(table.cpu())):
        with pytest.raises(ValueError):
            call()
