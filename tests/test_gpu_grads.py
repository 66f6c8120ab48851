"""GPU parity: the way back through the post-norm with its residual connection and through the activations, against float64."""
import math

import numpy as np
import pytest
import torch

from oracle import bf16, fp8, grads
from paper_2505_20524_amd import fog

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF = torch.bfloat16


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def matrix(rows, cols, ld=None, skew=0, dtype=BF, fill=7):
    """A [rows, cols] matrix with rows of `ld` elements, `skew` elements off its alignment, in a buffer full of `fill`."""
    ld = ld or cols
    base = torch.full((rows * ld + skew + 64,), fill, dtype=dtype, device="cuda")
    return base, base[skew:skew + rows * ld].view(rows, ld)[:, :cols]


def normal(seed, rows, cols, std=1.0, **more):
    m = matrix(rows, cols, **more)[1]
    m.copy_(torch.randn((rows, cols), device="cuda", generator=gen(seed)) * std)
    return m


def around(base, m, fill=7):
    """What lies around a matrix in its buffer is as it was."""
    other = torch.full_like(base, fill)
    other.as_strided(m.shape, m.stride(), m.storage_offset()).copy_(m)
    return torch.equal(base, other)


def one(v):
    return torch.full((1,), float(v), device="cuda")


def bytes_(n, fill=0xFF):
    return torch.full((max(n, 16),), fill, dtype=torch.uint8, device="cuda")


def h64(t):
    return t.double().cpu().numpy()


def check_rounded(got, want, e, what):
    """bf16 of a binary32 number within e of the float64 one."""
    g = h64(got)
    lo, hi = bf16.f64_round(want - e), bf16.f64_round(want + e)
    assert np.all((g >= lo) & (g <= hi)), (what, np.argwhere((g < lo) | (g > hi))[:5], g[(g < lo) | (g > hi)][:5])
    return g


def check_cast(q, amax, dx64, scale, fmt):
    if q is not None:
        assert np.array_equal(q.cpu().numpy(), fp8.encode_sat(np.float32(dx64) * np.float32(scale.item()), fmt))
    if amax is not None:
        assert amax.item() == (np.abs(dx64).max() if dx64.size else 0.0)


# ---------------------------------------------------------------------------------------------- post-norm
class Norm:
    def __init__(self, seed, rows, cols, branch=True, ld=0, skew=0):
        lay = dict(ld=cols + ld, skew=skew)
        self.rows, self.cols = rows, cols
        self.dres, self.y = normal(seed, rows, cols, 1e-3, **lay), normal(seed + 1, rows, cols, 1.0, **lay)
        self.dbranch = normal(seed + 2, rows, cols, 1e-3, **lay) if branch else None
        self.gamma = torch.rand(cols, device="cuda", generator=gen(seed + 3)) + 0.1
        (self.b_stream, self.dstream), (self.b_dy, self.dy) = matrix(rows, cols, **lay), matrix(rows, cols, **lay)
        self.b_q, self.q = matrix(rows, cols, dtype=torch.uint8, **lay)
        self.dgamma, self.amax, self.scale = torch.full((cols,), 3.0, device="cuda"), one(-1), one(57344.0 / 2e-2)
        self.ws = bytes_(fog.postnorm_residual_grad_workspace(rows, cols))

    def run(self, fmt=fog.E5M2, **change):
        a = dict(dbranch=self.dbranch, dstream=self.dstream, dy=self.dy, q=self.q, amax_out=self.amax)
        a.update(change)
        fog.postnorm_residual_grad(a.pop("dres", self.dres), self.y, self.gamma, fmt, self.scale, a.pop("dgamma", self.dgamma), self.ws, **a)

    def stream(self):
        """G, as one binary32 addition and one rounding give it."""
        g = h64(self.dres)
        if self.dbranch is not None:
            g = bf16.f64_round((g.astype(np.float32) + h64(self.dbranch).astype(np.float32)).astype(np.float64))
        return g

    def check(self, fmt=fog.E5M2, before=None):
        G = self.stream()
        assert np.array_equal(h64(self.dstream), G)
        want, dgamma, (size, along), terms = grads.postnorm(G, h64(self.y), h64(self.gamma))
        # chains of 64 in a lane, 6 between lanes and 8 between waves (80): the root's half and the mean, the quotient and the product (45), the sum along y and its quotient (162 and 45)
        dy = check_rounded(self.dy, want, 1.01 * U * (45 * size + 207 * along) + 2.0 ** -140, "dy")
        check_cast(self.q, self.amax, dy, self.scale, fmt)
        # a term: the norm's 42, two products; a wave's rows, 8 waves, 8 and 32 sums of the join
        n = -(-self.rows // 256) + 48 + 46
        base = 0.0 if before is None else before
        assert np.all(np.abs(h64(self.dgamma) - base - dgamma) <= 1.01 * U * (n * terms + np.abs(base)) + 2.0 ** -140)


SHAPES = [(1, 1), (1, 8), (3, 7), (5, 64), (9, 512), (17, 513), (300, 1000), (8, 1024), (2100, 260), (33, 2048), (777, 2064), (4, 4096), (2050, 4096), (13, 4097), (70, 8192),
          (5, 10001), (9, 16384), (3, 20000), (2, 32768), (600, 16400)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("branch", [True, False])
def test_postnorm(rows, cols, branch):
    n = Norm(rows + cols, rows, cols, branch)
    n.run()
    n.check()
    for b, m in ((n.b_stream, n.dstream), (n.b_dy, n.dy), (n.b_q, n.q)):
        assert around(b, m)


@pytest.mark.parametrize("ld,skew", [(0, 1), (8, 0), (3, 5), (1, 2)])
@pytest.mark.parametrize("rows,cols", [(40, 512), (23, 1001), (19, 4096), (6, 5000)])
def test_postnorm_rows_of_every_alignment(rows, cols, ld, skew):
    n = Norm(7, rows, cols, True, ld, skew)
    n.run(fog.E4M3)
    n.check(fog.E4M3)
    for b, m in ((n.b_stream, n.dstream), (n.b_dy, n.dy), (n.b_q, n.q)):
        assert around(b, m)


@pytest.mark.parametrize("rows,cols", [(50, 1000), (30, 4096), (12, 9000)])
def test_postnorm_without_some_results(rows, cols):
    n = Norm(11, rows, cols)
    n.run()
    want = [t.clone() for t in (n.dstream, n.dy, n.q, n.amax, n.dgamma)]
    for missing in ("dstream", "dy", "q", "amax_out", "dgamma"):
        for t in (n.dstream, n.dy, n.q, n.amax, n.dgamma):
            t.fill_(9)
        n.run(**{missing: None})
        for name, t, w in zip(("dstream", "dy", "q", "amax_out", "dgamma"), (n.dstream, n.dy, n.q, n.amax, n.dgamma), want):
            assert torch.equal(t, w) if name != missing else bool((t == 9).all()), (missing, name)


@pytest.mark.parametrize("rows,cols", [(50, 1000), (30, 4096), (12, 9000)])
def test_postnorm_in_place_and_added_to(rows, cols):
    n = Norm(12, rows, cols)
    n.run()
    want = [t.clone() for t in (n.dstream, n.dy, n.q, n.dgamma)]
    before = n.dgamma.clone()
    n.run(accumulate=True)
    n.check(before=h64(before))
    keep = [t.clone() for t in (n.dres, n.dbranch, n.y)]
    for into in ("dres", "dbranch"):
        for t, k in zip((n.dres, n.dbranch, n.y), keep):
            t.copy_(k)
        n.run(dstream=getattr(n, into), dy=n.y)
        assert torch.equal(getattr(n, into), want[0]) and torch.equal(n.y, want[1]) and torch.equal(n.q, want[2]) and torch.equal(n.dgamma, want[3])


def test_postnorm_rows_of_zeros_and_of_nan():
    n = Norm(13, 40, 600)
    n.y[3] = 0.0
    n.run()
    n.check()
    assert bool((n.dy[3] == 0).all())
    keep = n.dy.clone()
    n.y[5, 17] = float("nan")
    n.dres[7, 2] = float("inf")
    n.run()
    assert bool(torch.isnan(n.dy[5]).all()) and math.isnan(n.amax.item()) and bool((n.q[5] & 0x7F == 0x7F).all())
    same = [r for r in range(40) if r not in (5, 7)]
    assert torch.equal(n.dy[same], keep[same]) and math.isinf(n.dstream[7, 2].item())
    assert bool(torch.isnan(n.dgamma).all())            # x / NaN: every column of the row


@pytest.mark.parametrize("value", [1e-30, 1e-23, 3e17])
def test_postnorm_of_very_short_and_long_rows(value):
    n = Norm(16, 20, 700)
    n.y.mul_(value)
    n.y[3, 5], n.y[4] = 0.0, 0.0
    n.run()
    assert bool(torch.isfinite(n.dy).all()) and bool(torch.isfinite(n.dgamma).all()) and math.isfinite(n.amax.item())
    if value == 1e-30:
        assert bool((n.dy == 0).all()) and bool((n.dgamma == 0).all())
    if value == 3e17:
        n.check()


@pytest.mark.parametrize("rows,cols", [(0, 300), (5, 0), (0, 0)])
def test_postnorm_of_nothing(rows, cols):
    n = Norm(14, rows, cols)
    n.run()
    assert n.amax.item() == 0.0 and bool((n.dgamma == 0).all())
    n.dgamma.fill_(3.0)
    n.run(accumulate=True)
    assert bool((n.dgamma == 3.0).all())


def test_postnorm_is_the_same_on_every_run():
    n = Norm(15, 3000, 1111)
    n.run()
    first = [t.clone() for t in (n.dy, n.q, n.dgamma, n.amax)]
    for _ in range(3):
        n.ws.fill_(0x11)
        n.run()
        assert all(torch.equal(a, b) for a, b in zip((n.dy, n.q, n.dgamma, n.amax), first))


def test_postnorm_of_more_than_2_to_the_32_elements():
    """Rows far behind the first: on rows of equal numbers the norm is 1 and the gradients are whole numbers."""
    rows, cols = 131073, 32768
    one_row = torch.ones(cols, device="cuda")
    y, d = torch.ones((rows, cols), dtype=BF, device="cuda"), torch.zeros((rows, cols), dtype=BF, device="cuda")
    d[:, 0], d[-1, 5], d[-1, 6] = 1.0, 3.0, -3.0
    dgamma, amax = torch.zeros(cols, device="cuda"), one(-1)
    ws = bytes_(fog.postnorm_residual_grad_workspace(rows, cols))
    fog.postnorm_residual_grad(d, y, one_row, fog.E5M2, None, dgamma, ws, dy=d, amax_out=amax)
    # dy = G - sum(G) / 2^15: exact in binary32, then one rounding
    assert d[-1, 5].item() == 3.0 and d[-1, 6].item() == -3.0 and d[-1, 7].item() == -2.0 ** -15 and amax.item() == 3.0
    assert bool((d[:, 0] == torch.tensor(1 - 2.0 ** -15, device="cuda").to(BF)).all()) and dgamma[0].item() == rows
    assert dgamma[5].item() == 3.0 and dgamma[6].item() == -3.0 and float(dgamma[7:].abs().max()) == 0.0


# ---------------------------------------------------------------------------------------------- activations
ACTS = [("xielu", (0.8, 0.6)), ("xielu", (0.0, 2.5)), ("gelu", ()), ("tanh", (0.5,)), ("tanh", (-7.0,))]


class Act:
    def __init__(self, seed, act, alpha, rows, cols, ld=0, skew=0, std=1.5):
        lay = dict(ld=cols + ld, skew=skew)
        self.act, self.alpha, self.rows, self.cols = act, alpha, rows, cols
        self.x, self.d = normal(seed, rows, cols, std, **lay), normal(seed + 1, rows, cols, 1e-3, **lay)
        (self.b_dx, self.dx), (self.b_q, self.q) = matrix(rows, cols, **lay), matrix(rows, cols, dtype=torch.uint8, **lay)
        self.dalpha = torch.full((len(alpha),), 3.0, device="cuda") if alpha else None
        self.amax, self.scale, self.ws = one(-1), one(57344.0 / 3e-2), bytes_(fog.act_grad_workspace())

    def run(self, fmt=fog.E5M2, **change):
        a = dict(dx=self.dx, q=self.q, amax_out=self.amax)
        if self.alpha:
            a["dalpha"] = self.dalpha
        a.update(change)
        getattr(fog, self.act + "_grad")(self.x, self.d, *self.alpha, fmt, self.scale, self.ws, **a)

    def check(self, fmt=fog.E5M2, before=0.0):
        x, d = h64(self.x), h64(self.d)
        rel = 2.0 ** -19
        if self.act == "xielu":
            s, size, gs = grads.xielu(x, *[float(np.float32(a)) for a in self.alpha])
        elif self.act == "gelu":
            s, size, rest = grads.gelu_slope(x)
            size = size * (rel + x * x * 2.0 ** -23) / rel + rest * 2 * U / rel
            gs = []
        else:
            a = float(np.float32(self.alpha[0]))
            s, g = grads.tanh(x, a)
            grow = (rel + np.abs(a * x) * 2.0 ** -22) / rel
            size, gs = np.abs(s) * grow, [g]
        # (numbers below the smallest normal one, at the far ends, vanish or lose places)
        dx = check_rounded(self.dx, d * s, np.abs(d) * (1.01 * rel * size + 2.0 ** -120) + 2.0 ** -140, "dx")
        check_cast(self.q, self.amax, dx, self.scale, fmt)
        for i, g in enumerate(gs):
            # a term: 28 with the cancellation of e^x - 1 - x at -0.5 (tanh: 2^-19 and its growth), two products, a chain of 8, then binary64, one rounding
            each = np.abs(d * g) * (40 * U if self.act == "xielu" else 10 * U + rel * grow)
            assert abs(self.dalpha[i].item() - before - (d * g).sum()) <= 1.01 * each.sum() + 2 * U * (abs((d * g).sum()) + abs(before)) + 2.0 ** -120


@pytest.mark.parametrize("act,alpha", ACTS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (5, 33), (1, 4097), (333, 2736), (1000, 1024), (70, 14336), (40001, 17)])
def test_activation(act, alpha, rows, cols):
    a = Act(rows + cols, act, alpha, rows, cols)
    a.run()
    a.check()
    assert around(a.b_dx, a.dx) and around(a.b_q, a.q)


@pytest.mark.parametrize("act,alpha", ACTS)
@pytest.mark.parametrize("ld,skew", [(0, 1), (8, 0), (3, 5), (1, 2)])
@pytest.mark.parametrize("rows,cols", [(40, 512), (23, 1001), (600, 4096)])
def test_activation_rows_of_every_alignment(act, alpha, rows, cols, ld, skew):
    a = Act(21, act, alpha, rows, cols, ld, skew)
    a.run(fog.E4M3)
    a.check(fog.E4M3)
    assert around(a.b_dx, a.dx) and around(a.b_q, a.q)


@pytest.mark.parametrize("act,alpha", ACTS)
@pytest.mark.parametrize("rows,cols,ld,skew", [(1, 5_000_011, 0, 1), (2049, 2051, 0, 3), (1100, 4096, 16, 0), (1030, 4112, 3, 5), (1200, 4099, 1, 0)])
def test_activation_of_large_tensors(act, alpha, rows, cols, ld, skew):
    """From some four million elements on, end to end in a length that sixteen does not divide, in rows that it does, and in others."""
    a = Act(27, act, alpha, rows, cols, ld, skew)
    a.run()
    a.check()
    assert around(a.b_dx, a.dx) and around(a.b_q, a.q)


@pytest.mark.parametrize("rows", [3, 900])          # below and above the sizes that a table pays for
def test_xielu_sums_of_zeros_and_of_very_small_numbers(rows):
    """Exactly nothing from zeros; from numbers of at most 2^-24 their squares' half, or nothing."""
    a = Act(28, "xielu", (0.8, 0.6), rows, 8192)
    a.x[:, ::2], a.x[:, 1::2] = 0.0, -0.0
    a.run()
    assert a.dalpha.tolist() == [0.0, 0.0]
    a.x.fill_(-(2.0 ** -25))
    a.run()
    assert a.dalpha[0].item() == 0.0 and abs(a.dalpha[1].item()) <= 1.01 * 2.0 ** -51 * np.abs(h64(a.d)).sum()
    assert bool((a.dx == (a.d.float() * 0.5).to(BF)).all())


@pytest.mark.parametrize("act,alpha", ACTS)
@pytest.mark.parametrize("rows", [1, 96])          # 1, 96 times all 65536 - 512 finite numbers: below and above the sizes that a table pays for
def test_activation_at_every_number(act, alpha, rows):
    """Every finite bf16 number that is not beyond the binary32 range of its slope."""
    every = torch.arange(1 << 16, device="cuda", dtype=torch.int32).to(torch.int16).view(BF)
    every = every[torch.isfinite(every.float()) & (every.float().abs() <= 1e18)]
    a = Act(22, act, alpha, rows, every.numel())
    a.x.copy_(every.expand(rows, -1))
    a.d.fill_(2.0 ** -10)
    a.run(**({"dalpha": None} if alpha else {}))
    x, d = h64(a.x[0]), 2.0 ** -10
    if alpha:
        a.alpha, keep = alpha, a.dalpha
    rel = 2.0 ** -19
    if act == "xielu":
        s, size, _ = grads.xielu(x, *[float(np.float32(v)) for v in alpha])
    elif act == "gelu":
        s, size, rest = grads.gelu_slope(x)
        size = size * (1 + x * x * 2.0 ** -4) + rest * 2 * U / rel
    else:
        s, _ = grads.tanh(x, float(np.float32(alpha[0])))
        size = np.abs(s) * (1 + np.abs(alpha[0] * x) * 2.0 ** -3)
    for r in (0, rows - 1):
        check_rounded(a.dx[r], d * s, d * (1.01 * rel * size + 2.0 ** -120) + 2.0 ** -140, "dx")
    assert bool((a.dx == a.dx[0]).all())


@pytest.mark.parametrize("act,alpha", ACTS)
@pytest.mark.parametrize("rows,cols", [(40, 1000), (900, 8192)])
def test_activation_without_some_results_in_place_and_added_to(act, alpha, rows, cols):
    a = Act(23, act, alpha, rows, cols)
    a.run()
    names = ["dx", "q", "amax_out"] + (["dalpha"] if alpha else [])
    outs = [a.dx, a.q, a.amax] + ([a.dalpha] if alpha else [])
    want = [t.clone() for t in outs]
    for missing in names:
        for t in outs:
            t.fill_(9)
        a.run(**{missing: None})
        for name, t, w in zip(names, outs, want):
            assert torch.equal(t, w) if name != missing else bool((t == 9).all()), (missing, name)
    if alpha:
        a.dalpha.fill_(0.125)
        a.run(accumulate=True)
        for got, w in zip(a.dalpha.tolist(), want[3].tolist()):
            assert abs(got - (0.125 + w)) <= 2 * U * (0.125 + abs(w))
    keep = a.x.clone(), a.d.clone()
    a.run(dx=a.d)
    assert torch.equal(a.d, want[0]) and torch.equal(a.x, keep[0])
    a.d.copy_(keep[1])
    a.run(dx=a.x)
    assert torch.equal(a.x, want[0]) and torch.equal(a.d, keep[1])


@pytest.mark.parametrize("act,alpha", ACTS)
@pytest.mark.parametrize("rows", [3, 900])
def test_activation_of_numbers_that_are_not_finite(act, alpha, rows):
    a = Act(24, act, alpha, rows, 8192)
    a.run()
    keep = a.dx.clone()
    a.x[1, 5], a.d[2, 9] = float("nan"), float("nan")
    a.x[0, 3], a.x[0, 4] = float("inf"), float("-inf")
    a.run()
    assert math.isnan(a.dx[1, 5].item()) and math.isnan(a.dx[2, 9].item()) and math.isnan(a.amax.item())
    if alpha:
        assert bool(torch.isnan(a.dalpha).any())
    if act == "gelu":
        assert a.dx[0, 3].item() == a.d[0, 3].item() and a.dx[0, 4].item() == 0.0
    if act == "tanh":
        assert a.dx[0, 3].item() == 0.0 and a.dx[0, 4].item() == 0.0
    if act == "xielu":
        assert a.dx[0, 4].item() == (a.d[0, 4].float() * np.float32(0.5 - np.float32(alpha[1]))).to(BF).item()
    same = torch.ones_like(keep, dtype=torch.bool)
    same[1, 5] = same[2, 9] = same[0, 3] = same[0, 4] = False
    assert torch.equal(a.dx[same], keep[same])
    assert (a.q[1, 5].item() & 0x7F) == 0x7F and (a.q[2, 9].item() & 0x7F) == 0x7F


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("rows,cols,ld", [(3, 8192, 0), (900, 8192, 0), (1100, 4099, 1)])          # computed, from a table, and rows that no table takes
@pytest.mark.parametrize("x,d,which", [
    (INF, 1e-3, 0), (1.5, INF, 0), (1.5, -INF, 0), (1.5, NAN, 0), (INF, 0.0, 0), (INF, INF, 0), (3e38, INF, 0),
    (-INF, 1e-3, 1), (-1.5, INF, 1), (-1.5, -INF, 1), (-1.5, NAN, 1), (-INF, 0.0, 1), (0.0, INF, 1), (-0.0, NAN, 1), (-3e38, INF, 1), (NAN, 1e-3, 1)])
def test_what_is_not_finite_shows_in_its_own_sum(rows, cols, ld, x, d, which):
    """Numbers above zero belong to the first of the xIELU's sums, the others to the second: the one that they do not belong to is what it is without them."""
    a = Act(29, "xielu", (0.8, 0.6), rows, cols, ld)
    x64, d64 = h64(a.x), h64(a.d)
    for r, c in ((0, 0), (1, 513), (2, cols - 1), (rows - 1, 7)):
        a.x[r, c], a.d[r, c], x64[r, c], d64[r, c] = x, d, 0.0, 0.0
    a.run()
    assert not math.isfinite(a.dalpha[which].item())
    g = grads.xielu(x64, *[float(np.float32(v)) for v in a.alpha])[2][1 - which]
    terms = d64 * g
    assert abs(a.dalpha[1 - which].item() - terms.sum()) <= 1.01 * 40 * U * np.abs(terms).sum() + 2 * U * abs(terms.sum()) + 2.0 ** -120


@pytest.mark.parametrize("act,alpha", [ACTS[0], ACTS[2], ACTS[3]])
@pytest.mark.parametrize("rows,cols", [(0, 300), (5, 0)])
def test_activation_of_nothing(act, alpha, rows, cols):
    a = Act(25, act, alpha, rows, cols)
    a.run()
    assert a.amax.item() == 0.0
    if alpha:
        assert bool((a.dalpha == 0).all())
        a.dalpha.fill_(3.0)
        a.run(accumulate=True)
        assert bool((a.dalpha == 3.0).all())


@pytest.mark.parametrize("pad", [0, 8])
def test_activation_of_more_than_2_to_the_32_elements(pad):
    rows, cols = 65537, 65536
    x, d = matrix(rows, cols, cols + pad, fill=0)[1], matrix(rows, cols, cols + pad, fill=1)[1]
    x[-1, -1], x[-1, 0], x[0, 0] = 2.0, -1.0, 4.0
    dalpha, amax = torch.zeros(2, device="cuda"), one(-1)
    fog.xielu_grad(x, d, 1.0, 1.0, fog.E5M2, None, bytes_(fog.act_grad_workspace()), dx=d, amax_out=amax, dalpha=dalpha)
    assert d[-1, -1].item() == 4.5 and d[0, 0].item() == 8.5 and abs(d[-1, 0].item() - (math.exp(-1) - 0.5)) < 2.0 ** -8 and amax.item() == 8.5
    assert int((d != 0.5).sum()) == 3 and dalpha[0].item() == 20.0 and abs(dalpha[1].item() - math.exp(-1)) < 2.0 ** -20


# ---------------------------------------------------------------------------------------------- streams and graphs
def test_in_a_graph_and_on_two_streams():
    class Pass:
        def __init__(self, seed):
            self.norm, self.acts = Norm(seed, 500, 1300), [Act(seed + 10 * i, act, alpha, 200, 4096) for i, (act, alpha) in enumerate(ACTS)]

        def run(self, stream=None):
            self.norm.run(stream=stream)
            for a in self.acts:
                a.run(stream=stream)

        def new(self, seed):
            for i, t in enumerate([self.norm.dres, self.norm.dbranch, self.norm.y] + [m for a in self.acts for m in (a.x, a.d)]):
                t.copy_(torch.randn(t.shape, device="cuda", generator=gen(seed + i)))

        def outputs(self):
            n = self.norm
            return [t.clone() for t in [n.dstream, n.dy, n.q, n.amax, n.dgamma] + [m for a in self.acts for m in (a.dx, a.q, a.amax, a.dalpha) if m is not None]]

    p = Pass(60)
    p.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run()
    for i in range(4):
        p.new(100 * i)
        p.run()
        want = p.outputs()
        torch.cuda.synchronize()
        for t in (p.norm.dy, p.norm.dgamma, p.norm.amax, p.acts[0].dx, p.acts[0].dalpha, p.acts[2].amax):
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(p.outputs(), want))
    ps, want = [Pass(70), Pass(80)], []
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


def test_the_binding_refuses_what_the_calls_would_misread():
    n, a = Norm(90, 8, 64), Act(91, "xielu", (0.8, 0.6), 8, 64)
    for bad in (dict(dres=n.dres.cpu()), dict(dy=n.dy.float()), dict(q=n.q[:, :60]), dict(dgamma=torch.zeros(63, device="cuda")), dict(dgamma=n.dgamma.double()),
                dict(dbranch=n.dbranch.t()), dict(amax_out=torch.zeros(1))):
        with pytest.raises(ValueError):
            n.run(**bad)
    for bad in (dict(dx=a.dx.cpu()), dict(dx=a.dx[:4]), dict(q=a.q.float()), dict(dalpha=torch.zeros(1, device="cuda")), dict(amax_out=a.amax.half())):
        with pytest.raises(ValueError):
            a.run(**bad)
