"""GPU: the block-scaled layer, the embedding and the gradients' norm as a training step and a decoding step use them together: against the
float64 oracle stage by stage, as exact derivatives of each other, in a captured graph, and on two streams at once."""
import math

import numpy as np
import pytest
import torch

from oracle import bf16, block, fp8, gemm
from paper_2505_20524_amd import fog
from parity import check_gemm_elementwise, dev, host_u16

pytestmark = pytest.mark.gpu


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8, device="cuda")


def blocks(n):
    return -(-n // 128)


class Step:
    """Embedding -> one linear layer -> gradients -> their norm -> clipping, with every buffer allocated once."""

    def __init__(self, T, V, H, N, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.T, self.V, self.H, self.N, self.gen = T, V, H, N, g
        normal = lambda std, *s: (torch.randn(s, device="cuda", generator=g) * std).bfloat16()  # noqa: E731
        self.table, self.W = normal(0.02, V, H), normal(0.02, N, H)
        self.tokens, self.dY = torch.empty(T, dtype=torch.int64, device="cuda"), torch.empty((T, N), dtype=torch.bfloat16, device="cuda")
        self.factor = math.sqrt(H)
        self.scale, self.amax = torch.full((1,), 64.0, device="cuda"), torch.zeros(1, device="cuda")
        half = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.x, self.q, self.Y, self.dX, self.dW = half(T, H), u8(T, H), half(T, N), half(T, H), half(N, H)
        self.dE = torch.empty((V, H), device="cuda")
        self.X = dict(q_row=u8(T, H), s_row=u8(blocks(H), T), q_col=u8(T, H), s_col=u8(blocks(T), H))
        self.G = dict(q_row=u8(T, N), s_row=u8(blocks(N), T), q_col=u8(T, N), s_col=u8(blocks(T), N))
        self.Wq, self.Ws = u8(N, H), u8(blocks(N), blocks(H))
        need = max(fog.fp8_gemm_block_workspace(fog.NT, T, N, H), fog.fp8_gemm_block_workspace(fog.NN, T, H, N),
                   fog.fp8_gemm_block_workspace(fog.TN, N, H, T), fog.embed_grad_workspace(T, V, H), 16)
        self.ws, self.ws_norm = u8(need), u8(fog.grad_sumsq_workspace(2))
        self.sumsq, self.norm = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
        self.clipped = [torch.empty_like(self.dW), torch.empty_like(self.dE)]
        self.jobs = fog.make_grad_jobs(list(zip((self.dW, self.dE), self.clipped)))
        self.new_batch()

    def new_batch(self):
        """Other tokens (a tenth of them padding) and another output gradient, in the same buffers."""
        t = torch.randint(0, self.V, (self.T,), device="cuda", generator=self.gen)
        self.tokens.copy_(torch.where(torch.rand(self.T, device="cuda", generator=self.gen) < 0.1, torch.full_like(t, -1), t))
        self.dY.copy_(torch.randn((self.T, self.N), device="cuda", generator=self.gen) * 1e-2)

    def run(self, max_norm=0.5, stream=None):
        T, V, H, N, X, G, k = self.T, self.V, self.H, self.N, self.X, self.G, dict(stream=stream)
        fog.embed_quantize(self.tokens, self.table, self.factor, fog.E4M3, self.scale, self.x, q=self.q, amax_out=self.amax, **k)
        fog.quantize_block(self.x, fog.E4M3, **X, **k)
        fog.quantize_tile(self.W, fog.E4M3, self.Wq, self.Ws, **k)
        fog.fp8_gemm_block(fog.NT, T, N, H, X["q_row"], fog.E4M3, fog.VECTOR, X["s_row"], self.Wq, fog.E4M3, fog.TILE, self.Ws, self.Y, workspace=self.ws, **k)
        fog.quantize_block(self.dY, fog.E5M2, **G, **k)
        fog.fp8_gemm_block(fog.NN, T, H, N, G["q_row"], fog.E5M2, fog.VECTOR, G["s_row"], self.Wq, fog.E4M3, fog.TILE, self.Ws, self.dX, workspace=self.ws, **k)
        fog.fp8_gemm_block(fog.TN, N, H, T, G["q_col"], fog.E5M2, fog.VECTOR, G["s_col"], X["q_col"], fog.E4M3, fog.VECTOR, X["s_col"], self.dW,
                           workspace=self.ws, **k)
        fog.embed_grad(self.tokens, self.dX, self.factor, self.dE, self.ws, **k)
        fog.grad_sumsq(self.jobs, self.sumsq, self.ws_norm, **k)
        fog.grad_clip(self.jobs, self.sumsq, max_norm, self.norm, **k)

    def outputs(self):
        return [t.clone() for t in (self.x, self.q, self.amax, self.Y, self.dX, self.dW, self.dE, self.sumsq, self.norm, *self.clipped)]


def check_product(layout, got, a, fa, sa, form_a, b, fb, sb, form_b, what):
    h = lambda t: t.cpu().numpy()  # noqa: E731
    want, mag = block.product(layout, block.decode(h(a), fa, h(sa), form_a), block.decode(h(b), fb, h(sb), form_b))
    check_gemm_elementwise(host_u16(got.view(torch.int16)), want, mag, what=what)


@pytest.mark.parametrize("T,V,H,N", [(77, 50, 272, 144), (300, 1000, 528, 400), (1040, 300, 256, 512)])
def test_a_training_step_stage_by_stage(T, V, H, N):
    """Every stage against the oracle on what the stage before it left on the device."""
    st = Step(T, V, H, N, seed=T)
    max_norm = 0.5
    st.run(max_norm)
    torch.cuda.synchronize()
    tok, inside = st.tokens.cpu().numpy(), st.tokens.cpu().numpy() >= 0
    x = np.where(inside[:, None], bf16.bits_to_f32(host_u16(st.table.view(torch.int16)))[np.where(inside, tok, 0)] * np.float32(st.factor), np.float32(0))
    xb = host_u16(st.x.view(torch.int16))
    assert np.array_equal(xb, bf16.f64_to_bits_rne(x.astype(np.float64)))
    for t, fmt, c in ((st.x, fp8.E4M3, st.X), (st.dY, fp8.E5M2, st.G)):
        for form, name in ((block.ROW, "row"), (block.COL, "col")):
            q, s = block.quantize(host_u16(t.view(torch.int16)), fmt, form)
            assert np.array_equal(c["q_" + name].cpu().numpy(), q) and np.array_equal(c["s_" + name].cpu().numpy(), s)
    q, s = block.quantize(host_u16(st.W.view(torch.int16)), fp8.E4M3, block.TILE)
    assert np.array_equal(st.Wq.cpu().numpy(), q) and np.array_equal(st.Ws.cpu().numpy(), s)
    check_product(gemm.NT, st.Y, st.X["q_row"], fp8.E4M3, st.X["s_row"], block.ROW, st.Wq, fp8.E4M3, st.Ws, block.TILE, "forward")
    check_product(gemm.NN, st.dX, st.G["q_row"], fp8.E5M2, st.G["s_row"], block.ROW, st.Wq, fp8.E4M3, st.Ws, block.TILE, "data gradient")
    check_product(gemm.TN, st.dW, st.G["q_col"], fp8.E5M2, st.G["s_col"], block.COL, st.X["q_col"], fp8.E4M3, st.X["s_col"], block.COL, "weight gradient")
    dE, mag = np.zeros((V, H)), np.zeros((V, H))
    rows = st.dX.double().cpu().numpy()[inside] * st.factor
    np.add.at(dE, tok[inside], rows)
    np.add.at(mag, tok[inside], np.abs(rows))
    # a run of T binary32 additions at most, the factor and its product, one rounding
    assert np.all(np.abs(st.dE.double().cpu().numpy() - dE) <= (T + 3) * 2.0 ** -24 * mag)
    total = float((st.dW.double() ** 2).sum() + (st.dE.double() ** 2).sum())
    n = st.dW.numel() + st.dE.numel()
    assert abs(st.sumsq.item() - total) <= 2 * n * 2.0 ** -53 * total
    assert math.sqrt(total) > max_norm
    for g, out in zip((st.dW, st.dE), st.clipped):
        want = g.double() * (max_norm / math.sqrt(total))
        # factor and product in binary32, half a step of the type
        assert bool(((out.double() - want).abs() <= (2.0 ** -22 + torch.finfo(g.dtype).eps / 2) * want.abs()).all())
    # the norm after clipping is the limit, up to the roundings of the clipped values
    after = math.sqrt(float((st.clipped[0].double() ** 2).sum() + (st.clipped[1].double() ** 2).sum()))
    assert abs(after - max_norm) <= 2.0 ** -8 * max_norm


def ints(rng, lo, hi, *shape):
    return rng.integers(lo, hi + 1, shape).astype(np.float64)


def half(a):
    return dev(bf16.f64_to_bits_rne(a))


def test_products_are_each_others_derivatives():
    """On small whole numbers everything is exact, so that <dY, Y(X + e) - Y(X)> = <dX, e> and <dY, Y(W + e) - Y(W)> = <dW, e> hold exactly."""
    rng = np.random.default_rng(1)
    T, N, H = 48, 32, 160
    sparse = lambda lo, hi, p, *s: ints(rng, lo, hi, *s) * (rng.random(s) < p)  # noqa: E731
    X, W, dY = sparse(-3, 3, 0.1, T, H), sparse(-3, 3, 0.1, N, H), sparse(-2, 2, 0.1, T, N)

    def forward(x, w):
        X_, W_, s_w = dict(q_row=u8(T, H), s_row=u8(blocks(H), T)), u8(N, H), u8(blocks(N), blocks(H))
        Y = torch.empty((T, N), dtype=torch.bfloat16, device="cuda")
        fog.quantize_block(half(x), fog.E4M3, **X_)
        fog.quantize_tile(half(w), fog.E4M3, W_, s_w)
        fog.fp8_gemm_block(fog.NT, T, N, H, X_["q_row"], fog.E4M3, fog.VECTOR, X_["s_row"], W_, fog.E4M3, fog.TILE, s_w, Y)
        return Y.double().cpu().numpy()

    G, C = (dict(q_row=u8(T, n), s_row=u8(blocks(n), T), q_col=u8(T, n), s_col=u8(1, n)) for n in (N, H))
    W_, s_w = u8(N, H), u8(1, 2)
    fog.quantize_block(half(dY), fog.E5M2, **G)
    fog.quantize_block(half(X), fog.E4M3, **C)
    fog.quantize_tile(half(W), fog.E4M3, W_, s_w)
    dX, dW = (torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in ((T, H), (N, H)))
    fog.fp8_gemm_block(fog.NN, T, H, N, G["q_row"], fog.E5M2, fog.VECTOR, G["s_row"], W_, fog.E4M3, fog.TILE, s_w, dX)
    fog.fp8_gemm_block(fog.TN, N, H, T, G["q_col"], fog.E5M2, fog.VECTOR, G["s_col"], C["q_col"], fog.E4M3, fog.VECTOR, C["s_col"], dW)
    base = forward(X, W)
    assert np.array_equal(base, X @ W.T) and np.abs(base).max() > 0
    for _ in range(3):
        e, f = sparse(-2, 2, 0.1, T, H), sparse(-2, 2, 0.1, N, H)
        assert (dY * (forward(X + e, W) - base)).sum() == (dX.double().cpu().numpy() * e).sum()
        assert (dY * (forward(X, W + f) - base)).sum() == (dW.double().cpu().numpy() * f).sum()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_embeddings_gradient_is_its_derivative(dtype):
    """<dx, x(E + e) - x(E)> = <dE, e>, exactly on small whole numbers and a factor of 2."""
    rng = np.random.default_rng(2)
    T, V, H = 90, 20, 24
    tokens = rng.integers(-1, V + 1, T)
    E, dx = ints(rng, -9, 9, V, H), ints(rng, -1, 1, T, H)

    def forward(table):
        x = torch.empty((T, H), dtype=torch.bfloat16, device="cuda")
        fog.embed_quantize(dev(tokens), half(table), 2.0, fog.E4M3, None, x)
        return x.double().cpu().numpy()

    dE = torch.empty((V, H), dtype=dtype, device="cuda")
    fog.embed_grad(dev(tokens), half(dx), 2.0, dE, u8(fog.embed_grad_workspace(T, V, H)))
    for _ in range(3):
        e = ints(rng, -5, 5, V, H)
        assert (dx * (forward(E + e) - forward(E))).sum() == (dE.double().cpu().numpy() * e).sum()


@pytest.mark.parametrize("T,V,H,N", [(300, 1000, 528, 400), (3000, 700, 256, 272)])
def test_a_step_in_a_graph(T, V, H, N):
    """Captured once, replayed on other batches with eager work and synchronizations between: the eager step's bits every time."""
    st = Step(T, V, H, N, seed=5)
    st.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.run()
    for _ in range(4):
        st.new_batch()
        st.run()
        want = st.outputs()
        torch.cuda.synchronize()
        for t in (st.x, st.Y, st.dX, st.dW, st.dE, *st.clipped):
            t.fill_(3.0)
        st.sumsq.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip(st.outputs(), want):
            assert torch.equal(got, w)


def test_steps_on_two_streams():
    """Two steps at once, each on a stream and with workspaces of its own: what each does by itself."""
    steps = [Step(300, 1000, 528, 400, seed=6), Step(2500, 90, 256, 144, seed=7)]
    want = []
    for st in steps:
        st.run()
        want.append(st.outputs())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(5):
        for st, s in zip(steps, streams):
            st.run(stream=s)
    torch.cuda.synchronize()
    for st, w in zip(steps, want):
        for got, ref in zip(st.outputs(), w):
            assert torch.equal(got, ref)


@pytest.mark.parametrize("M", [1, 3, 20])
def test_a_decoding_step(M):
    """Rows of single tokens through lookup, cast and a resident weight, as one batch and token by token: the same bits, because a row's sums do not
    depend on the rows beside it."""
    rng = np.random.default_rng(M)
    V, H, N = 60, 1040, 336
    table = dev(bf16.f64_to_bits_rne(rng.standard_normal((V, H)) * 0.02))
    W, s_w = u8(N, H), u8(blocks(N), blocks(H))
    fog.quantize_tile(dev(bf16.f64_to_bits_rne(rng.standard_normal((N, H)) * 0.02)), fog.E4M3, W, s_w)
    tokens = dev(rng.integers(0, V, M))

    def rows(t):
        m = t.numel()
        x, Y = torch.empty((m, H), dtype=torch.bfloat16, device="cuda"), torch.empty((m, N), dtype=torch.bfloat16, device="cuda")
        q, s = u8(m, H), u8(blocks(H), m)
        fog.embed_quantize(t, table, math.sqrt(H), fog.E4M3, None, x)
        fog.quantize_block(x, fog.E4M3, q_row=q, s_row=s)
        fog.fp8_gemm_block(fog.NT, m, N, H, q, fog.E4M3, fog.VECTOR, s, W, fog.E4M3, fog.TILE, s_w, Y)
        want, mag = block.product(gemm.NT, block.decode(q.cpu().numpy(), fp8.E4M3, s.cpu().numpy(), block.ROW),
                                  block.decode(W.cpu().numpy(), fp8.E4M3, s_w.cpu().numpy(), block.TILE))
        check_gemm_elementwise(host_u16(Y.view(torch.int16)), want, mag, what="decoding %d rows" % m)
        return Y

    whole = rows(tokens)
    for i in range(M):
        assert torch.equal(rows(tokens[i:i + 1])[0], whole[i])


def test_the_binding_refuses_tensors_of_other_devices():
    x, q, s = torch.zeros((4, 256), dtype=torch.bfloat16, device="cuda"), u8(4, 256), u8(2, 4)
    with pytest.raises(ValueError):
        fog.quantize_block(x.cpu(), fog.E4M3, q_row=q, s_row=s)
    with pytest.raises(ValueError):
        fog.quantize_block(x, fog.E4M3, q_row=q, s_row=s.cpu())
    with pytest.raises(ValueError):
        fog.grad_sumsq(fog.make_grad_jobs([x.cpu()]), torch.zeros(1, dtype=torch.float64, device="cuda"), u8(1 << 16))
    with pytest.raises(ValueError):
        fog.quantize_block(x.half(), fog.E4M3, q_row=q, s_row=s)
