"""The rotary oracle against facts that do not come from it."""
import cmath
import math

import numpy as np
import pytest

from oracle import rope


@pytest.mark.parametrize("layout", [rope.HALF, rope.INTERLEAVED])
def test_turn_is_a_complex_multiplication(layout):
    rng = np.random.default_rng(1)
    D, rot, p = 12, 8, 37
    x = rng.standard_normal((1, 1, 1, D))
    y, _ = rope.forward(x, rope.table(range(50), rot), np.array([[p]]), layout)
    for i in range(rot // 2):
        a, b = (i, i + 4) if layout == rope.HALF else (2 * i, 2 * i + 1)
        z = complex(x[0, 0, 0, a], x[0, 0, 0, b]) * cmath.exp(1j * p * 10000.0 ** (-2 * i / rot))
        assert abs(z - complex(y[0, 0, 0, a], y[0, 0, 0, b])) < 1e-13
    assert np.array_equal(y[..., rot:], x[..., rot:])


@pytest.mark.parametrize("layout", [rope.HALF, rope.INTERLEAVED])
def test_scores_depend_on_the_distance_only(layout):
    rng = np.random.default_rng(2)
    q, k = rng.standard_normal((2, 1, 1, 1, 16))
    tab = rope.table(range(1000), 16)
    at = lambda v, p: rope.forward(v, tab, np.array([[p]]), layout)[0].ravel()  # noqa: E731
    want = at(q, 9) @ at(k, 4)
    for shift in (1, 100, 900):
        assert abs(at(q, 9 + shift) @ at(k, 4 + shift) - want) < 1e-11
    assert np.array_equal(at(q, 0), q.ravel())


def test_scaled_frequencies():
    f = rope.frequencies(64)
    assert f[0] == 1.0 and abs(f[32 // 2] - 1e-2) < 1e-15
    assert np.allclose(rope.frequencies(64, factor=4.0), f / 4)
    g = rope.frequencies(64, factor=8.0, low=1.0, high=32.0, original=4096)
    turns = 4096 * f / (2 * math.pi)
    assert np.array_equal(g[turns >= 32], f[turns >= 32]) and np.allclose(g[turns <= 1], f[turns <= 1] / 8, rtol=1e-15)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and np.all(g[mid] < f[mid]) and np.all(g[mid] > f[mid] / 8)
    assert np.allclose(rope.table([5], 8, amplitude=3.0)[0, :4] ** 2 + rope.table([5], 8, amplitude=3.0)[0, 4:] ** 2, 9.0)


@pytest.mark.parametrize("layout", [rope.HALF, rope.INTERLEAVED])
@pytest.mark.parametrize("gain", [0.0, 1.7])
def test_backward_by_differences(layout, gain):
    rng = np.random.default_rng(3)
    x, dy = rng.standard_normal((2, 2, 3, 2, 10))
    tab, pos = rope.table(range(20), 6, amplitude=1.3), np.array([[0, 5, -1], [19, 20, 7]])
    f = lambda v: (rope.forward(v, tab, pos, layout, gain)[0] * dy).sum()  # noqa: E731
    dx, _, _ = rope.backward(dy, x, tab, pos, layout, gain)
    for at in [(0, 0, 0, 0), (0, 1, 1, 3), (1, 0, 0, 5), (1, 2, 1, 8), (0, 2, 0, 1), (1, 1, 1, 9)]:
        e = np.zeros_like(x)
        e[at] = 1e-6
        assert abs((f(x + e) - f(x - e)) / 2e-6 - dx[at]) < 1e-7
    assert not dx[0, 2].any() and not dx[1, 1].any()         # padding


def test_a_vector_of_zeros():
    x = np.zeros((1, 1, 1, 4))
    tab = rope.table(range(3), 4)
    assert not rope.forward(x, tab, np.array([[1]]), rope.HALF, 1.0)[0].any()
    assert not rope.backward(x + 1, x, tab, np.array([[1]]), rope.HALF, 1.0)[0].any()
