"""The gradient oracles by differences of the forward oracles."""
import numpy as np
import pytest

from oracle import bf16, gelu, grads, postnorm, xielu


def test_postnorm_by_differences():
    rng = np.random.default_rng(1)
    y, G, gamma = rng.standard_normal((4, 11)), rng.standard_normal((4, 11)), rng.standard_normal(11).astype(np.float32).astype(np.float64)
    norm = lambda v, g: g * v / np.sqrt((v * v).mean(-1, keepdims=True))  # noqa: E731
    assert np.allclose(norm(bf16.f64_round(y), gamma), postnorm.normalize(bf16.f64_to_bits_rne(y), gamma), rtol=1e-12)
    dy, dgamma, _, _ = grads.postnorm(G, y, gamma)
    for at in ((0, 0), (1, 5), (3, 10)):
        e = np.zeros_like(y)
        e[at] = 1e-6
        assert abs(((norm(y + e, gamma) - norm(y - e, gamma)) * G).sum() / 2e-6 - dy[at]) < 1e-8
    for c in (0, 4):
        e = np.zeros(11)
        e[c] = 1e-6
        assert abs(((norm(y, gamma + e) - norm(y, gamma - e)) * G).sum() / 2e-6 - dgamma[c]) < 1e-8
    y[2] = 0.0
    assert not grads.postnorm(G, y, gamma)[0][2].any()


X = np.concatenate([np.linspace(-9, 9, 181), [-1e-4, 1e-4, -0.5, 1e-30]])


def slope(f, x, h=1e-5):
    return (f(x + h) - f(x - h)) / (2 * h)


def test_xielu_by_differences():
    x = X[np.abs(X) > 1e-4]
    s, size, (g0, g1) = grads.xielu(x, 0.8, 0.6)
    assert np.abs(slope(lambda v: xielu.xielu(v, 0.8, 0.6), x) - s).max() < 1e-7 and np.all(size >= np.abs(s) - 1e-15)
    for g, a in ((g0, (1e-5, 0)), (g1, (0, 1e-5))):
        diff = (xielu.xielu(x, 0.8 + a[0], 0.6 + a[1]) - xielu.xielu(x, 0.8 - a[0], 0.6 - a[1])) / 2e-5
        assert np.abs(diff - g).max() < 1e-7
    assert abs(grads.xielu(np.array([-1e-4]), 1, 1)[2][1][0] / (0.5e-8 - 1e-12 / 6) - 1) < 1e-8


def test_gelu_by_differences():
    s, size, one = grads.gelu_slope(X)
    assert np.abs(slope(gelu.gelu, X) - s).max() < 1e-8
    assert np.all(size + one >= np.abs(s) - 1e-15) and abs(grads.gelu_slope(np.array([0.0]))[0][0] - 0.5) < 1e-16
    assert grads.gelu_slope(np.array([-12.0]))[0][0] < 0


@pytest.mark.parametrize("alpha", [0.5, -3.0])
def test_tanh_by_differences(alpha):
    s, g = grads.tanh(X, alpha)
    assert np.abs(slope(lambda v: gelu.tanh_alpha(v, alpha), X) - s).max() < 1e-7
    assert np.abs(slope(lambda a: gelu.tanh_alpha(X, a), alpha) - g).max() < 1e-7
