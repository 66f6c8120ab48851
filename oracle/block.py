"""Block scales: casts and products with a scale for each block of 128 elements.

Appendix E's cast takes rho = FP8MaxValue / (2^m max|X|) over a whole tensor.  Here the maximum is taken over blocks of
128 elements of a row (ROW), 128 elements of a column (COL) or tiles of 128 x 128 (TILE), and rho is rounded down to a power of
two, 2^k, so that scaling and unscaling are exact.  A block's scale is kept as the byte 127 - k of its reciprocal 2^(byte - 127).

Readings: k = 0 for blocks whose maximum is zero or not finite; -126 <= k <= 126.
"""
import numpy as np

from . import bf16, fp8, gemm

BLOCK = 128
ROW, COL, TILE = "row", "col", "tile"
_SHAPE = {ROW: (1, BLOCK), COL: (BLOCK, 1), TILE: (BLOCK, BLOCK)}


def exponent(amax, fmt, margin=0):
    """Largest k with 2^margin * amax * 2^k <= FP8MaxValue, by trial in exact rational arithmetic (amax: a float)."""
    from fractions import Fraction
    if not np.isfinite(amax) or amax == 0:
        return 0
    a, top = Fraction(float(amax)) * Fraction(2) ** margin, Fraction(fp8.fp8_max(fmt))
    k = int(np.floor(np.log2(fp8.fp8_max(fmt)) - np.log2(float(amax)) - margin))
    while a * Fraction(2) ** (k + 1) <= top:
        k += 1
    while a * Fraction(2) ** k > top:
        k -= 1
    return max(-126, min(126, k))


def _block_amax(x, form):
    br, bc = _SHAPE[form]
    rows, cols = x.shape
    out = np.zeros((-(-rows // br), -(-cols // bc)), dtype=np.float32)
    for i in range(out.shape[0]):
        part = np.abs(x[i * br:(i + 1) * br])
        for j in range(out.shape[1]):
            out[i, j] = part[:, j * bc:(j + 1) * bc].max()      # NaN if any is
    return out


def _spread(per_block, form, rows, cols):
    br, bc = _SHAPE[form]
    return np.repeat(np.repeat(per_block, br, axis=0)[:rows], bc, axis=1)[:, :cols]


def quantize(x_bits, fmt, form, margin=0):
    """(codes, scale bytes) of a bf16 matrix; the bytes lie as the casts lay them: ROW [blocks of columns][rows], COL [blocks of
    rows][columns], TILE [blocks of rows][blocks of columns]."""
    x = bf16.bits_to_f32(np.asarray(x_bits, dtype=np.uint16))
    with np.errstate(invalid="ignore"):
        k = np.vectorize(lambda a: exponent(a, fmt, margin), otypes=[np.int64])(_block_amax(x, form))
        # a bf16 value times a power of two is exact in binary64; the codes' rounding sees binary32, in which only values far
        # below half the smallest code differ
        t = (x.astype(np.float64) * np.exp2(_spread(k, form, *x.shape).astype(np.float64))).astype(np.float32)
    s = (127 - k).astype(np.uint8)
    return fp8.encode_sat(t, fmt), np.ascontiguousarray(s.T) if form == ROW else s


def decode(codes, fmt, s, form):
    """float64 values that codes and scale bytes stand for."""
    s = np.asarray(s, dtype=np.float64)
    inv = np.exp2((s.T if form == ROW else s) - 127.0)
    return fp8.decode(codes, fmt) * _spread(inv, form, *codes.shape)


def product(layout, a, b):
    """(product, sum of magnitudes) of decoded operands as they are stored."""
    def mul(p, q):
        return p @ q.T if layout == gemm.NT else p @ q if layout == gemm.NN else p.T @ q
    return mul(a, b), mul(np.abs(a), np.abs(b))
