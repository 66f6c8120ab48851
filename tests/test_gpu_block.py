"""GPU parity: casts and products with a scale for each block of 128 against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import bf16, block, fp8, gemm
from paper_2505_20524_amd import fog, synth
from parity import check_gemm_elementwise, dev, host_u16

pytestmark = pytest.mark.gpu

FORMS = (block.ROW, block.COL, block.TILE)
KIND = {block.ROW: fog.VECTOR, block.COL: fog.VECTOR, block.TILE: fog.TILE}


def spread_values(seed, rows, cols):
    """Normal values over 60 binary orders of magnitude, and outlier columns."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-30, 30, (rows, 1))) * np.exp2(rng.integers(-3, 4, (1, cols)))
    return bf16.f64_to_bits_rne(x)


def shape_of_scales(form, rows, cols):
    b = lambda n: -(-n // 128)  # noqa: E731
    return {block.ROW: (b(cols), rows), block.COL: (b(rows), cols), block.TILE: (b(rows), b(cols))}[form]


def cast_on_gpu(x, fmt, margin=0, forms=FORMS, pad=0, skew=0):
    """form -> (codes, scale bytes) from one call for ROW and COL together and one for TILE.  pad: extra elements behind every row of every
    buffer, which have to stay as they are; skew: elements that every buffer starts behind its alignment."""
    rows, cols = x.shape

    def room(r, c, dtype, fill):
        flat = torch.full((r * (c + pad) + skew,), fill, dtype=dtype, device="cuda")
        return flat, flat[skew:].view(r, c + pad)

    flat, xd = room(rows, cols, torch.int16, 0x7FC0)
    xd[:, :cols] = dev(x)
    out, kept = {}, []
    for form in forms:
        pair = [room(rows, cols, torch.uint8, 0xA5), room(*shape_of_scales(form, rows, cols), torch.uint8, 0xA5)]
        kept += pair
        out[form] = (pair[0][1][:, :cols], pair[1][1][:, :shape_of_scales(form, rows, cols)[1]])
    args = {}
    for form, name in ((block.ROW, "row"), (block.COL, "col")):
        if form in forms:
            args["q_" + name], args["s_" + name] = out[form]
    if args:
        fog.quantize_block(xd[:, :cols], fmt, margin=margin, **args)
    if block.TILE in forms:
        fog.quantize_tile(xd[:, :cols], fmt, *out[block.TILE], margin=margin)
    torch.cuda.synchronize()
    if pad or skew:
        for (flat, view), used in zip(kept, [u for form in forms for u in out[form]]):
            assert bool((flat[:skew] == 0xA5).all()) and bool((view[:, used.shape[1]:] == 0xA5).all())
    return {form: tuple(t.cpu().numpy() for t in out[form]) for form in forms}


SHAPES = [(1, 1), (1, 128), (1, 4096), (3, 130), (127, 129), (128, 128), (129, 257), (200, 72), (260, 392), (513, 1000)]


@pytest.mark.parametrize("fmt", [fp8.E4M3, fp8.E5M2])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_casts_are_bit_exact(rows, cols, fmt):
    x = spread_values(rows * 7 + cols, rows, cols)
    for form, (q, s) in cast_on_gpu(x, fmt).items():
        want_q, want_s = block.quantize(x, fmt, form)
        assert np.array_equal(s, want_s), form
        assert np.array_equal(q, want_q), form


@pytest.mark.parametrize("forms", [(block.ROW,), (block.COL,), (block.ROW, block.COL), (block.TILE,)])
@pytest.mark.parametrize("rows,cols,pad,skew", [(130, 264, 8, 0), (130, 264, 3, 0), (65, 200, 0, 8), (65, 200, 8, 1), (3, 129, 16, 16)])
def test_casts_with_strides_and_every_alignment(rows, cols, pad, skew, forms):
    x = spread_values(rows + pad, rows, cols)
    for form, (q, s) in cast_on_gpu(x, fp8.E4M3, forms=forms, pad=pad, skew=skew).items():
        want_q, want_s = block.quantize(x, fp8.E4M3, form)
        assert np.array_equal(s, want_s) and np.array_equal(q, want_q), form


@pytest.mark.parametrize("margin", [-64, -3, 2, 64])
@pytest.mark.parametrize("fmt", [fp8.E4M3, fp8.E5M2])
def test_cast_margins(fmt, margin):
    """A margin below zero saturates; one of 64 leaves subnormal codes and zeros."""
    x = spread_values(11, 140, 264)
    for form, (q, s) in cast_on_gpu(x, fmt, margin=margin).items():
        want_q, want_s = block.quantize(x, fmt, form, margin)
        assert np.array_equal(s, want_s) and np.array_equal(q, want_q), form


@pytest.mark.parametrize("cols", [256, 257])
@pytest.mark.parametrize("fmt", [fp8.E4M3, fp8.E5M2])
def test_cast_special_values(fmt, cols):
    """Blocks of zeros, with NaN of both signs, with infinities, with the largest and the smallest bf16, with values at the format's border;
    the blocks beside them are untouched by it."""
    x = spread_values(5, 256, cols)
    x[:128, :128] = 0
    x[130, 7], x[131, 200] = 0x7FC1, 0xFFC0
    x[3, 200], x[4, 201] = 0x7F80, 0xFF80
    x[140] = 0x0001
    x[141] = 0x8003
    x[142] = 0x7F7F
    x[143, ::2], x[143, 1::2] = 0x43E0, 0x43E1          # 448 and the value above it
    x[144] = 0x43E0
    x[145] = 0x4760                                     # 57344
    for form, (q, s) in cast_on_gpu(x, fmt).items():
        want_q, want_s = block.quantize(x, fmt, form)
        assert np.array_equal(s, want_s) and np.array_equal(q, want_q), form


def operands(layout, M, N, K, fa, fb, form_a, form_b, seed):
    """Casts of an activation-like [M, K] and a weight-like [N, K], laid out for `layout`, with bytes of scales along the contraction.
    form: VECTOR or TILE."""
    xb, wb, _ = synth.small_linear(seed, M, N, K)
    a = xb if layout != gemm.TN else np.ascontiguousarray(xb.T)
    b = wb if layout == gemm.NT else np.ascontiguousarray(wb.T)
    along_a = block.ROW if layout != gemm.TN else block.COL
    along_b = block.ROW if layout == gemm.NT else block.COL
    fa_, fb_ = along_a if form_a == fog.VECTOR else block.TILE, along_b if form_b == fog.VECTOR else block.TILE
    qa, sa = block.quantize(a, fa, fa_)
    qb, sb = block.quantize(b, fb, fb_)
    return (qa, sa, block.decode(qa, fa, sa, fa_)), (qb, sb, block.decode(qb, fb, sb, fb_))


def padded(s, by=5, fill=0xFF):
    """Scale bytes with bytes behind every row that no result may depend on."""
    t = torch.full((s.shape[0], s.shape[1] + by), fill, dtype=torch.uint8, device="cuda")
    t[:, :s.shape[1]] = dev(s)
    return t[:, :s.shape[1]]


def product(layout, M, N, K, a, fa, kind_a, b, fb, kind_b, workspace=True, ldc_pad=0):
    C = torch.full((M, N + ldc_pad), 0x7FC0, dtype=torch.int16, device="cuda")
    need = fog.fp8_gemm_block_workspace(layout, M, N, K) if workspace else 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    fog.fp8_gemm_block(layout, M, N, K, dev(a[0]), fa, kind_a, padded(a[1]), dev(b[0]), fb, kind_b, padded(b[1]), C[:, :N], workspace=ws)
    torch.cuda.synchronize()
    if ldc_pad:
        assert bool((C[:, N:] == 0x7FC0).all())
    return host_u16(C[:, :N])


def check(layout, M, N, K, fa=fp8.E4M3, fb=fp8.E4M3, kind_a=fog.VECTOR, kind_b=fog.TILE, seed=1, **kw):
    a, b = operands(layout, M, N, K, fa, fb, kind_a, kind_b, seed)
    want, mag = block.product(layout, a[2], b[2])
    got = product(layout, M, N, K, a, fa, kind_a, b, fb, kind_b, **kw)
    # half a bf16 step plus 2^-12 of the accumulated magnitude: the bound of the per-tensor product, whose instruction this is
    check_gemm_elementwise(got, want, mag, what="block gemm %d %dx%dx%d" % (layout, M, N, K))


def check_any_codes(got, want, mag, what):
    """For codes drawn evenly, whose products spread over 2^28: the instruction aligns the eight products of a group to the largest and keeps
    at least 12 places below it (tests/test_gpu_mfma_model.py), so that each of the seven others loses less than 2^-12 of the
    largest, and a group less than 7 * 2^-12 of its magnitude.  (2^-12 in all holds for products of like size.)"""
    check_gemm_elementwise(got, want, 7 * mag, what=what)


LAYOUTS = [gemm.NT, gemm.NN, gemm.TN]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("kind_a,kind_b", [(fog.VECTOR, fog.TILE), (fog.VECTOR, fog.VECTOR), (fog.TILE, fog.VECTOR), (fog.TILE, fog.TILE)])
@pytest.mark.parametrize("M,N,K", [(304, 528, 384), (272, 144, 400), (16, 272, 16), (144, 80, 4112)])
def test_products(layout, M, N, K, kind_a, kind_b):
    check(layout, M, N, K, kind_a=kind_a, kind_b=kind_b, seed=M + K)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("fa,fb", [(fp8.E4M3, fp8.E5M2), (fp8.E5M2, fp8.E4M3), (fp8.E5M2, fp8.E5M2)])
def test_product_formats(layout, fa, fb):
    check(layout, 208, 176, 272, fa, fb, fog.VECTOR, fog.VECTOR, seed=fa + 2 * fb)


KERNELS = [
    # M, N, K, (tile, workgroups per CU, split)
    (8176, 8208, 2064, (256, 256, 1, False)),       # several tiles a workgroup
    (2048, 8192, 1040, (256, 256, 1, False)),
    (1744, 2480, 9296, (256, 256, 1, True)),
    (1776, 3088, 2064, (256, 128, 1, False)),
    (2560, 1024, 16384, (256, 128, 1, True)),
    (4112, 4064, 528, (128, 128, 2, False)),
    (1040, 2064, 784, (128, 128, 1, False)),
    (272, 272, 9232, (64, 64, 2, True)),
    (304, 272, 400, (64, 64, 2, False)),
]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("M,N,K,kernel", KERNELS)
def test_every_kernel_of_the_product(layout, M, N, K, kernel):
    """Each tile and each way to cut the contraction, on codes and scale bytes of every kind: selected rows, the last ones among them."""
    plan = fog.probe_gemm_plan(layout, M, N, K, with_workspace=True, compute_units=256)
    assert plan[:3] + (plan[3] > 1,) == kernel
    rng = np.random.default_rng(M + N + K + layout)
    blocks = -(-K // 128)
    # finite codes of both signs; scale bytes over 2^-20 .. 2^4
    qa, qb = ((rng.integers(0, 0x7F, s) | rng.integers(0, 2, s) << 7).astype(np.uint8)
              for s in ((K, M) if layout == gemm.TN else (M, K), (N, K) if layout == gemm.NT else (K, N)))
    sa, sb = rng.integers(107, 132, (blocks, M)).astype(np.uint8), rng.integers(107, 132, (blocks, N)).astype(np.uint8)
    got = product(layout, M, N, K, (qa, sa), fp8.E4M3, fog.VECTOR, (qb, sb), fp8.E4M3, fog.VECTOR)
    rows = np.r_[0:2, 127:130, 255:258, M // 2, M - 2:M]
    if layout == gemm.TN:
        a = block.decode(np.ascontiguousarray(qa[:, rows]), fp8.E4M3, np.ascontiguousarray(sa[:, rows]), block.COL)
    else:
        a = block.decode(qa[rows], fp8.E4M3, np.ascontiguousarray(sa[:, rows]), block.ROW)
    want, mag = block.product(layout, a, block.decode(qb, fp8.E4M3, sb, block.ROW if layout == gemm.NT else block.COL))
    check_any_codes(got[rows], want, mag, what="rows of %dx%dx%d" % (M, N, K))


@pytest.mark.parametrize("M", [1, 4, 5, 8, 9, 12, 13, 16, 17, 20, 21, 24, 25, 28, 29, 32, 33, 64])
@pytest.mark.parametrize("N,K", [(1, 16), (17, 144), (1000, 4112), (2064, 1168), (8208, 272)])
def test_few_rows(M, N, K):
    check(gemm.NT, M, N, K, seed=M + N)


@pytest.mark.parametrize("fa,fb,kind_a,kind_b", [(0, 1, 0, 0), (1, 0, 1, 0), (1, 1, 1, 1)])
def test_few_rows_formats_and_forms(fa, fb, kind_a, kind_b):
    check(gemm.NT, 5, 336, 2064, fa, fb, kind_a, kind_b, seed=9)


@pytest.mark.parametrize("M", [3, 80])
@pytest.mark.parametrize("ldc_pad", [1, 4, 8])
def test_result_strides(M, ldc_pad):
    check(gemm.NT, M, 200, 400, ldc_pad=ldc_pad)


@pytest.mark.parametrize("M", [2, 144])
def test_scales_span_their_range(M):
    """Bytes from 1 to 254 whose products stay in binary32: rows of A scaled up as far as rows of B are scaled down."""
    rng = np.random.default_rng(8)
    N, K = 64, 512
    qa, qb = (fp8.encode_sat(rng.standard_normal(s).astype(np.float32), fp8.E4M3) for s in ((M, K), (N, K)))
    e = rng.integers(-126, 127, (4, 1))
    sa, sb = np.broadcast_to(127 + e, (4, M)).astype(np.uint8), np.clip(127 - e + rng.integers(-2, 3, (4, N)), 1, 254).astype(np.uint8)
    a, b = (qa, sa, block.decode(qa, fp8.E4M3, sa, block.ROW)), (qb, sb, block.decode(qb, fp8.E4M3, sb, block.ROW))
    want, mag = block.product(gemm.NT, a[2], b[2])
    check_gemm_elementwise(product(gemm.NT, M, N, K, a, fp8.E4M3, fog.VECTOR, b, fp8.E4M3, fog.VECTOR), want, mag)


def test_empty_products():
    C = torch.full((5, 7), 0x7FC0, dtype=torch.int16, device="cuda")
    none = torch.empty((0, 16), dtype=torch.uint8, device="cuda")
    lib = fog.load()
    assert lib.fog_fp8_gemm_block(0, 5, 7, 0, None, 0, 0, 0, None, 0, None, 0, 0, 1, None, 0, C.data_ptr(), 7, None, 0, None) == 0
    torch.cuda.synchronize()
    assert bool((C == 0).all())
    fog.quantize_block(none.view(torch.int16), fog.E4M3, q_row=none[:, :8], s_row=torch.empty((1, 0), dtype=torch.uint8, device="cuda"))


def test_a_cast_beyond_32_bit_offsets():
    """The last rows of a tensor of more than 2^31 elements, against the same rows cast by themselves."""
    rows, cols, last = 65536 + 40, 33000, 40
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x[-last:] = torch.randn((last, cols), device="cuda", generator=g)
    q, s = torch.full((rows, cols), 0xA5, dtype=torch.uint8, device="cuda"), torch.empty((-(-cols // 128), rows), dtype=torch.uint8, device="cuda")
    fog.quantize_block(x, fog.E4M3, q_row=q, s_row=s)
    q1, s1 = torch.empty((last, cols), dtype=torch.uint8, device="cuda"), torch.empty((-(-cols // 128), last), dtype=torch.uint8, device="cuda")
    fog.quantize_block(x[-last:], fog.E4M3, q_row=q1, s_row=s1)
    assert torch.equal(q[-last:], q1) and torch.equal(s[:, -last:], s1)
    assert int(torch.count_nonzero(q[:-last])) == 0 and bool((s[:, :-last] == 127).all())
    fog.quantize_tile(x, fog.E4M3, q, torch.empty((-(-rows // 128), -(-cols // 128)), dtype=torch.uint8, device="cuda"))
    assert int(torch.count_nonzero(q[:-last])) == 0 and int(torch.count_nonzero(q[-last:])) > last * cols // 2
