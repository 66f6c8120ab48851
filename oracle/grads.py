"""The way back through the post-norm with its residual connection and through the activations, in float64, with the size of the terms whose roundings a binary32
evaluation makes (for tolerances)."""
import math

import numpy as np
from scipy import special


def postnorm(G, y, gamma):
    """(dy, dgamma, size of dy's two terms, size of dgamma's terms) from the gradient G of the stream behind the norm."""
    yy = (y * y).sum(-1, keepdims=True)
    inv = np.divide(1.0, np.sqrt(yy / y.shape[-1]), out=np.zeros_like(yy), where=yy > 0)
    safe = np.where(yy > 0, yy, 1.0)
    t = G * gamma
    along, most = (t * y).sum(-1, keepdims=True) / safe, np.abs(t * y).sum(-1, keepdims=True) / safe
    return inv * (t - y * along), (G * y * inv).sum(0), (inv * np.abs(t), inv * np.abs(y) * most), np.abs(G * y * inv).sum(0)


def xielu(x, ap, an):
    """f'(x), its terms' size, and the derivatives after alpha_p and alpha_n."""
    e = np.expm1(np.minimum(x, 0.0))
    s = np.where(x > 0, 2 * ap * x, an * e)
    near = np.abs(x) < 1e-3
    curve = np.where(near, x * x / 2 + x ** 3 / 6 + x ** 4 / 24 + x ** 5 / 120, e - x)      # e^x - 1 - x without cancellation
    return s + 0.5, np.abs(s) + 0.5, [np.where(x > 0, x * x, 0.0), np.where(x > 0, 0.0, curve)]


def gelu_slope(x):
    """Phi(x) + x phi(x), and the size of its terms: for x > 0 taken from 1."""
    t = np.abs(x)
    phi = np.exp(-0.5 * t * t) / math.sqrt(2 * math.pi)
    tail = 0.5 * special.erfc(t / math.sqrt(2))
    return np.where(x < 0, tail - t * phi, 1.0 - tail + t * phi), tail + t * phi, np.where(x < 0, 0.0, 1.0)


def tanh(x, alpha):
    """alpha sech^2(alpha x) and the derivative after alpha."""
    with np.errstate(over="ignore"):
        s = 1.0 / np.cosh(alpha * x) ** 2
    return alpha * s, x * s
