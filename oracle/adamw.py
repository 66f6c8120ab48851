"""The AdamW step and its states in FP8, from the formulas: moments rounded as the library states them (binary32, operation by operation), the
parameters in float64, and the rounding to one of the two neighbouring codes by a table of all codes instead of by bits.

The random numbers are integers of 32 bits: a hash of seed, step, tensor and element, in whole-number arithmetic.
"""
import numpy as np

from . import block, fp8

MASK = (1 << 32) - 1
ODD = (0x9E3779B1, 0x6A09E667, 0xBB67AE85)        # fractions of the golden ratio, of sqrt 2 and of sqrt 3, made odd
BITS = {fp8.E4M3: 20, fp8.E5M2: 21}               # places of a binary32 number that the format drops


def mix(h):
    """Three rounds of shift and multiplication (python integer or uint64 array below 2^32)."""
    for shift, odd in zip((16, 15, 13), ODD):
        h = ((h ^ (h >> shift)) * odd) & MASK
    return h ^ (h >> 16)


def random_bits(seed, step, tensor, first, n):
    """32 random bits for elements first .. first + n - 1 of a tensor."""
    key = 0
    for word in (seed & MASK, seed >> 32, step & MASK, step >> 32, tensor):
        key = mix((key + 0x9E3779B9 + word) & MASK)
    i = np.arange(first, first + n, dtype=np.uint64)
    high = mix(((i >> np.uint64(32)) + np.uint64(key)) & np.uint64(MASK))
    return mix((i & np.uint64(MASK)) ^ high)


def clip_factor(sumsq, max_norm):
    norm = np.sqrt(np.float64(sumsq))
    return np.float32(np.float64(np.float32(max_norm)) / norm) if norm > np.float64(np.float32(max_norm)) else np.float32(1)


def moments(m, v, g, c, beta1, beta2):
    """New m and v in binary32, each operation rounded once."""
    f = np.float32
    gc = g.astype(f) * f(c)
    return m.astype(f) * f(beta1) + gc * f(1 - beta1), v.astype(f) * f(beta2) + gc * gc * f(1 - beta2)


def update(p, m, v, lr, beta1, beta2, eps, weight_decay, t):
    """The parameters after the step in float64, from the new moments, and the size of what is taken from them (for tolerances)."""
    p, m, v = (np.asarray(a, dtype=np.float64) for a in (p, m, v))
    u = lr * (m / (1 - beta1 ** t)) / (np.sqrt(v / (1 - beta2 ** t)) + np.float64(np.float32(eps)))
    return p - lr * weight_decay * p - u, np.abs(u)


def round_by(y, r, fmt):
    """Non-negative numbers within the format's range to the code below or above: above where the share of the step that lies below, in units of 2^-BITS,
    plus the random number is a whole step."""
    codes = np.arange(0, 0x7F if fmt == fp8.E4M3 else 0x7C)
    values = fp8.decode(codes, fmt)
    lo = np.searchsorted(values, y, side="right") - 1
    hi = np.minimum(lo + 1, len(codes) - 1)
    step = np.where(hi > lo, values[hi] - values[lo], 1.0)
    share = np.rint((y - values[lo]) / step * 2.0 ** BITS[fmt])       # whole but below the smallest normal number, where it is rounded to whole
    r = r & 0xFFFFF if fmt == fp8.E4M3 else r >> 11
    return np.where(share + r >= 2.0 ** BITS[fmt], hi, lo).astype(np.uint8)


def encode(x, r, fmt):
    """(codes, scale bytes) of a state in binary32."""
    x = np.asarray(x, dtype=np.float32)
    n = len(x)
    codes, scales = np.zeros(n, np.uint8), np.zeros(-(-n // block.BLOCK), np.uint8)
    for b in range(len(scales)):
        at = slice(b * block.BLOCK, min(n, (b + 1) * block.BLOCK))
        k = block.exponent(np.abs(x[at]).max(), fmt)
        scales[b] = 127 - k
        y = np.abs(x[at]).astype(np.float64) * 2.0 ** k
        q = round_by(y, r[at].astype(np.int64), fmt)
        if fmt == fp8.E5M2:
            q = np.where((x[at] > 0) & (q == 0), 1, q)
        codes[at] = q | np.where(np.signbit(x[at]), 0x80, 0).astype(np.uint8)
    return codes, scales


def decode(codes, scales, fmt):
    """binary32 values of a state's codes."""
    return (fp8.decode(codes, fmt) * np.repeat(np.exp2(scales.astype(np.float64) - 127.0), block.BLOCK)[:len(codes)]).astype(np.float32)
