"""Block scales of the oracle: exponents at the borders, layouts of the scale bytes, unscaling."""
import numpy as np
import pytest

from oracle import bf16, block, fp8, gemm, scaling


@pytest.mark.parametrize("fmt,top", [(fp8.E4M3, 448.0), (fp8.E5M2, 57344.0)])
def test_exponent_at_the_borders(fmt, top):
    assert block.exponent(top, fmt) == 0
    assert block.exponent(top * (1 + 2 ** -7), fmt) == -1
    assert block.exponent(top / 2, fmt) == 1
    assert block.exponent(top, fmt, margin=3) == -3
    assert block.exponent(0.0, fmt) == 0 and block.exponent(np.inf, fmt) == 0 and block.exponent(np.nan, fmt) == 0
    assert block.exponent(2.0 ** -133, fmt) == 126
    assert block.exponent(3.3e38, fmt, margin=64) == -126


@pytest.mark.parametrize("form,shape", [(block.ROW, (3, 200)), (block.COL, (2, 300)), (block.TILE, (3, 2))])
def test_scale_bytes_lie_as_documented_and_undo_the_scale(form, shape):
    rng = np.random.default_rng(3)
    rows, cols = (200, 300)
    x = bf16.f64_to_bits_rne(rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-20, 20, (rows, cols))))
    if form == block.TILE:
        shape = (2, 3)
    q, s = block.quantize(x, fp8.E4M3, form)
    assert s.shape == (shape if form != block.COL else (2, 300))
    v, want = block.decode(q, fp8.E4M3, s, form), bf16.bits_to_f64(x)
    inv = block.decode(np.full_like(q, 0x38), fp8.E4M3, s, form)      # code of 1: the reciprocal scales themselves
    # half a step of the format (2^-4 relative), or of its smallest subnormal under the scale
    assert np.all(np.abs(v - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * inv))


def test_a_block_of_one_tensor_scale_is_the_tensor_cast():
    rng = np.random.default_rng(4)
    x = bf16.f64_to_bits_rne(rng.standard_normal((128, 128)))
    q, s = block.quantize(x, fp8.E5M2, block.TILE)
    assert np.array_equal(q, scaling.quantize(x, np.float32(2.0) ** (127 - int(s[0, 0])), fp8.E5M2))


def test_product_layouts():
    rng = np.random.default_rng(5)
    a, b = rng.standard_normal((4, 6)), rng.standard_normal((5, 6))
    want = a @ b.T
    for layout, p, q in ((gemm.NT, a, b), (gemm.NN, a, b.T), (gemm.TN, a.T, b.T)):
        got, mag = block.product(layout, p, q)
        assert np.allclose(got, want, rtol=1e-14) and np.all(mag >= np.abs(got) - 1e-12)
