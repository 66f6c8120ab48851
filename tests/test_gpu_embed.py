"""GPU parity: the embedding with its cast, and its gradient, against plain float64 evaluations."""
import numpy as np
import pytest
import torch

from oracle import bf16, fp8, scaling
from paper_2505_20524_amd import fog
from parity import dev, fscalar, host_u16

pytestmark = pytest.mark.gpu


def table_bits(seed, V, H, std=0.02):
    return bf16.f64_to_bits_rne(np.random.default_rng(seed).standard_normal((V, H)) * std)


def tokens_of(seed, T, V, invalid=0.1):
    """Ids with frequent ones among them, and some outside the table."""
    rng = np.random.default_rng(seed)
    t = (np.exp(rng.random(T) * np.log(V + 1)) - 1).astype(np.int64).clip(0, V - 1)
    out = rng.choice([-1, V, V + 5, -2 ** 31, 2 ** 31 - 1], T)
    return np.where(rng.random(T) < invalid, out, t)


def embed(tokens, table, factor, fmt, scale, with_q=True, pad=0, dtype=np.int32):
    T, H = tokens.size, table.shape[1]
    td = torch.zeros((table.shape[0], H + pad), dtype=torch.int16, device="cuda")
    td[:, :H] = dev(table)
    x = torch.full((T, H + pad), 0x1234, dtype=torch.int16, device="cuda")
    q = torch.full((T, H + pad), 0xA5, dtype=torch.uint8, device="cuda")
    amax = torch.full((1,), -1.0, device="cuda")
    fog.embed_quantize(dev(tokens.astype(dtype)), td[:, :H], factor, fmt, fscalar(scale) if with_q else None, x[:, :H],
                       q=q[:, :H] if with_q else None, amax_out=amax)
    torch.cuda.synchronize()
    if pad:
        assert bool((x[:, H:] == 0x1234).all()) and bool((q[:, H:] == 0xA5).all())
    return host_u16(x[:, :H]), q[:, :H].cpu().numpy(), amax.item()


@pytest.mark.parametrize("T,V,H,pad,dtype", [
    (1, 10, 8, 0, np.int32), (24, 300, 2048, 0, np.int64), (77, 50, 2064, 8, np.int64), (130, 1, 4096, 0, np.int32), (33, 40, 131, 0, np.int64),
    (9, 40, 264, 3, np.int32), (5000, 100, 64, 0, np.int64), (3, 20, 16384, 0, np.int32)])
def test_embedding(T, V, H, pad, dtype):
    table, tokens = table_bits(T, V, H), tokens_of(T, T, V)
    factor, scale = np.float32(np.sqrt(H)), np.float32(100.0)
    x, q, amax = embed(tokens, table, float(factor), fog.E4M3, scale, pad=pad, dtype=dtype)
    inside = (tokens >= 0) & (tokens < V)
    want = np.where(inside[:, None], bf16.bits_to_f32(table)[np.where(inside, tokens, 0)] * factor, np.float32(0))
    # one binary32 product, rounded once to bf16: the same bits; zeros of invalid rows are positive
    assert np.array_equal(x, bf16.f64_to_bits_rne(want.astype(np.float64)))
    assert np.array_equal(q, scaling.quantize(x, scale, fp8.E4M3))
    assert amax == scaling.amax(x)


@pytest.mark.parametrize("fmt", [fog.E4M3, fog.E5M2])
@pytest.mark.parametrize("H", [64, 65])
def test_embedding_of_values_that_are_not_finite(H, fmt):
    table = table_bits(1, 8, H)
    table[2, 5], table[3, 6], table[4, 7] = 0x7FC0, 0x7F80, 0xFF80
    tokens = np.array([1, 2, 3, 4, 0])
    x, q, amax = embed(tokens, table, 2.0, fmt, 4.0)
    assert np.array_equal(q, scaling.quantize(x, np.float32(4.0), fmt)) and np.isnan(amax)
    x, q, amax = embed(np.array([1, 3, 4]), table, 2.0, fmt, 4.0)
    assert amax == np.inf


def test_embedding_without_a_cast_and_without_tokens():
    table = table_bits(2, 30, 264)
    tokens = tokens_of(3, 50, 30)
    x, _, amax = embed(tokens, table, 1.0, fog.E4M3, 1.0, with_q=False)
    y, _, _ = embed(tokens, table, 1.0, fog.E4M3, 1.0)
    assert np.array_equal(x, y) and amax == scaling.amax(x)
    _, _, amax = embed(np.zeros(0, dtype=np.int64), table, 1.0, fog.E4M3, 1.0)
    assert amax == 0.0
    x, q, amax = embed(np.array([0, 5]), table[:0], 1.0, fog.E4M3, 1.0)      # a table without rows: every id is outside
    assert not x.any() and not q.any() and amax == 0.0


def gradient(tokens, dx, V, factor, dtype=torch.float32, accumulate=False, start=None, pad=0, token_type=np.int64, ws_fill=0xFF):
    T, H = dx.shape
    dxd = torch.zeros((T, H + pad), dtype=torch.int16, device="cuda")
    dxd[:, :H] = dev(dx)
    dE = torch.full((V, H + pad), 7.0, dtype=dtype, device="cuda")
    if start is not None:
        dE[:, :H] = torch.from_numpy(start).cuda().to(dtype)
    ws = torch.full((max(fog.embed_grad_workspace(T, V, H), 16),), ws_fill, dtype=torch.uint8, device="cuda")
    fog.embed_grad(dev(tokens.astype(token_type)), dxd[:, :H], factor, dE[:, :H], ws, accumulate=accumulate)
    torch.cuda.synchronize()
    if pad:
        assert bool((dE[:, H:] == 7.0).all())
    return dE[:, :H].cpu()


def exact_gradient(tokens, dx, V, factor):
    """(sum, sum of magnitudes, tokens of the id) in float64."""
    g, mag, n = np.zeros((V, dx.shape[1])), np.zeros((V, dx.shape[1])), np.zeros((V, 1))
    inside = (tokens >= 0) & (tokens < V)
    v = bf16.bits_to_f64(dx)[inside] * factor
    np.add.at(g, tokens[inside], v)
    np.add.at(mag, tokens[inside], np.abs(v))
    np.add.at(n, tokens[inside], 1.0)
    return g, mag, n


def check_gradient(got, want, mag, n, dtype, start=None):
    # binary32 sums of n terms in any order: n 2^-24 of the magnitudes; the factor and its product 2 more; one addition to what was there and one
    # rounding to the result's type: half a step, 2^-24 or 2^-8, of the result
    got = got.double().numpy()
    total = want if start is None else want + start
    tol = (n + 2) * 2.0 ** -24 * mag * 1.01 + (0 if start is None else 2.0 ** -24 * np.abs(total))
    half = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
    assert np.all(np.abs(got - total) <= tol + half * (np.abs(total) + tol)), np.abs(got - total).max()
    if start is None:
        assert not got[(n == 0)[:, 0]].any()
    else:
        assert np.array_equal(got[(n == 0)[:, 0]], start[(n == 0)[:, 0]])


GRADS = [(1, 5, 8), (2, 3, 264), (7, 100, 2064), (63, 1, 512), (64, 40, 520), (65, 33, 131), (777, 1000, 264), (1023, 17, 72), (1024, 5000, 64),
         (1025, 200, 1032), (2047, 300, 72), (2048, 5, 264), (2049, 4000, 24), (3000, 3, 1544), (20000, 900, 40), (40001, 50000, 16)]


@pytest.mark.parametrize("T,V,H", GRADS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient(T, V, H, dtype):
    tokens, dx = tokens_of(T + V, T, V), table_bits(T, T, H, 1e-3)
    factor = float(np.float32(np.sqrt(H)))
    want = exact_gradient(tokens, dx, V, factor)
    check_gradient(gradient(tokens, dx, V, factor, dtype), *want, dtype)
    start = bf16.f64_round(np.random.default_rng(V).standard_normal((V, H)) * 1e-2)
    check_gradient(gradient(tokens, dx, V, factor, dtype, accumulate=True, start=start), *want, dtype, start=start)


@pytest.mark.parametrize("H,pad,token_type", [(264, 8, np.int32), (264, 3, np.int64), (129, 2, np.int32)])
def test_gradient_strides_and_token_types(H, pad, token_type):
    tokens, dx = tokens_of(1, 700, 90), table_bits(2, 700, H, 1e-3)
    want = exact_gradient(tokens, dx, 90, 2.0)
    for dtype in (torch.float32, torch.bfloat16):
        check_gradient(gradient(tokens, dx, 90, 2.0, dtype, pad=pad, token_type=token_type), *want, dtype)


@pytest.mark.parametrize("T,H", [(5000, 40), (300, 1032), (70, 8), (20000, 264)])
def test_gradient_of_one_id_and_of_none(T, H):
    """A run over every chunk of the order; a batch of nothing but padding; both between ids that do not occur."""
    dx = table_bits(T, T, H, 1e-3)
    for tokens in (np.full(T, 3), np.full(T, -1), np.where(np.arange(T) % 2, 0, 6)):
        want = exact_gradient(tokens, dx, 7, 1.0)
        check_gradient(gradient(tokens, dx, 7, 1.0), *want, torch.float32)


def test_gradient_is_the_same_on_every_run_and_whatever_the_workspace_holds():
    tokens, dx = tokens_of(6, 9000, 70), table_bits(7, 9000, 264, 1e-3)
    first = gradient(tokens, dx, 70, 1.5)
    for fill in (0, 0x7F, 0xFF):
        assert torch.equal(gradient(tokens, dx, 70, 1.5, ws_fill=fill), first)


def test_gradient_without_tokens_clears_or_keeps():
    dx = np.zeros((0, 24), dtype=np.uint16)
    none = np.zeros(0, dtype=np.int64)
    assert not gradient(none, dx, 50, 1.0).any()
    assert bool((gradient(none, dx, 50, 1.0, accumulate=True) == 7.0).all())


def test_gradient_of_values_that_are_not_finite_stays_in_its_rows():
    tokens, dx = np.array([4, 1, 4, 2, -1, 9]), table_bits(8, 6, 40)
    dx[0, 3], dx[3, 5], dx[4], dx[5] = 0x7FC0, 0x7F80, 0x7FC0, 0x7FC0
    got = gradient(tokens, dx, 6, 1.0).numpy()
    assert np.isnan(got[4, 3]) and got[2, 5] == np.inf
    got[4, 3] = got[2, 5] = 0
    assert np.isfinite(got).all()


def test_a_table_beyond_32_bit_offsets():
    """The last rows of a gradient of more than 2^31 elements (5 GB in bf16)."""
    V, H = 40000, 65536
    tokens, dx = np.array([V - 1, 0, V - 1, 39000]), table_bits(3, 4, H, 1e-3)
    dE = torch.full((V, H), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(fog.embed_grad_workspace(4, V, H), dtype=torch.uint8, device="cuda")
    fog.embed_grad(dev(tokens), dev(dx), 1.0, dE, ws)
    x = torch.empty((4, H), dtype=torch.bfloat16, device="cuda")
    fog.embed_quantize(dev(tokens), dE, 1.0, fog.E4M3, None, x)
    torch.cuda.synchronize()
    d = bf16.bits_to_f64(dx)
    # two terms: one binary32 sum and half a bf16 step
    for row, want in ((V - 1, d[0] + d[2]), (0, d[1]), (39000, d[3])):
        assert np.all(np.abs(dE[row].double().cpu().numpy() - want) <= (2.0 ** -8 + 2.0 ** -23) * np.abs(want) + 2.0 ** -24 * (np.abs(d[0]) + np.abs(d[2])))
    assert int(torch.count_nonzero(dE[1:39000])) == 0 and int(torch.count_nonzero(dE[39001:V - 1])) == 0
    assert torch.equal(x[0], dE[V - 1]) and torch.equal(x[3], dE[39000])
