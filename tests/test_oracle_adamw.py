"""The AdamW oracle against facts that do not come from it."""
import numpy as np
import pytest
import torch

from oracle import adamw, fp8


def test_update_equals_torch_in_float64():
    rng = np.random.default_rng(1)
    p0 = rng.standard_normal(50)
    p = torch.nn.Parameter(torch.from_numpy(p0.copy()))
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.9, 0.95), eps=2.0 ** -27, weight_decay=0.1)
    m, v, q = np.zeros(50), np.zeros(50), p0.copy()
    for t in range(1, 6):
        g = rng.standard_normal(50)
        p.grad = torch.from_numpy(g)
        opt.step()
        m, v = 0.9 * m + 0.1 * g, 0.95 * v + 0.05 * g * g
        q, _ = adamw.update(q, m, v, 1e-2, 0.9, 0.95, 2.0 ** -27, 0.1, t)
        assert np.abs(p.detach().numpy() - q).max() < 1e-14


@pytest.mark.parametrize("fmt", [fp8.E4M3, fp8.E5M2])
def test_codes_stay_and_values_between_split_by_their_share(fmt):
    values = fp8.decode(np.arange(0, 0x7F if fmt == fp8.E4M3 else 0x7C), fmt)
    full = np.full(len(values), MASK := (1 << 32) - 1)
    assert np.array_equal(adamw.round_by(values, full, fmt), np.arange(len(values)))       # a code's value stays under any random number
    assert np.array_equal(adamw.round_by(values, 0 * full, fmt), np.arange(len(values)))
    mid = (values[1:] + values[:-1]) / 2
    top = 1 << 31 if fmt == fp8.E5M2 else 1 << 19           # the share of a half: up from the random number of a half on
    half = np.full(len(mid), top)
    assert np.array_equal(adamw.round_by(mid, half, fmt), np.arange(1, len(values)))
    assert np.array_equal(adamw.round_by(mid, half - (1 << 11 if fmt == fp8.E5M2 else 1), fmt), np.arange(len(values) - 1))
    assert MASK == full[0]


def test_the_hash_is_even_and_without_visible_ties():
    """2^18 numbers: every bit as often 0 as 1, the low and the high part in 256 classes each as a chance draw fills them, neighbours and other tensors, steps and seeds
    unrelated.  Six standard deviations, one of 2^18 draws of a half being 2^-10."""
    n = 1 << 18
    base = adamw.random_bits(7, 3, 0, 0, n)
    runs = [base] + [adamw.random_bits(*a, 0, n) for a in ((8, 3, 0), (7 + (1 << 32), 3, 0), (7, 4, 0), (7, 3 + (1 << 32), 0), (7, 3, 1))]
    runs.append(adamw.random_bits(7, 3, 0, 1 << 32, n))
    bound = 6 * 0.5 / np.sqrt(n)
    for r in runs:
        for bit in range(32):
            assert abs(((r >> np.uint64(bit)) & np.uint64(1)).mean() - 0.5) < bound
        for part in ((r & np.uint64(0xFFFFF)) >> np.uint64(12), r >> np.uint64(24)):
            counts = np.bincount(part.astype(np.int64), minlength=256)
            assert abs(((counts - n / 256) ** 2 / (n / 256)).sum() - 255) < 6 * np.sqrt(2 * 255)
        u = r / 2.0 ** 32 - 0.5
        assert abs((u[1:] * u[:-1]).mean()) < 6 / 12 / np.sqrt(n)
        low = (r & np.uint64(0xFFFFF)) / 2.0 ** 20 - 0.5
        assert abs((u * low).mean()) < 6 / 12 / np.sqrt(n) + 2.0 ** -12 / 12      # the two parts share nine bits, the lowest of one of them
    for r in runs[1:]:
        assert abs((((r ^ base) & np.uint64(1 << 31)) > 0).mean() - 0.5) < bound


def test_scales_and_floor():
    x = np.array([0.0, 1e-30, 3.0, 448.0] + [0.0] * 124 + [0.0, 5e-9, 1.0], np.float32)
    q, s = adamw.encode(x, np.zeros(len(x), np.int64), fp8.E5M2)
    assert s.tolist() == [127 - 7, 127 - 15] and q[0] == 0 and q[1] == 1 and q[128] == 0
    assert q[129] == 9           # 5e-9 2^15 = 1.342 2^-13: code 8 is 2^-13, a step is a quarter of it
    assert np.array_equal(adamw.decode(q, s, fp8.E5M2)[[2, 3, 130]], np.float32([3.0, 448.0, 1.0]))
    assert adamw.decode(np.zeros(5, np.uint8), np.zeros(1, np.uint8), fp8.E4M3).tolist() == [0.0] * 5
