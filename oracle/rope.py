"""Rotary positions with the QK norm, forward and backward, in float64, written as a matrix of the turn per position.

Each function also returns how large the terms are whose roundings a binary32 evaluation makes (for tolerances).
"""
import numpy as np

HALF, INTERLEAVED = 0, 1


def frequencies(rot, base=10000.0, factor=1.0, low=1.0, high=4.0, original=0.0):
    """Angle per position of each pair; scaled for contexts beyond `original` tokens."""
    f = np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)])
    if factor == 1.0:
        return f
    keep = np.zeros_like(f) if original == 0 else np.clip((original * f / (2 * np.pi) - low) / (high - low), 0.0, 1.0)
    return f * ((1 - keep) / factor + keep)


def table(positions, rot, amplitude=1.0, **scaling):
    """[len(positions), rot]: cosines, then sines, of the pairs, in float64."""
    a = np.asarray(positions, dtype=np.float64)[:, None] * frequencies(rot, **scaling)
    return np.concatenate([np.cos(a), np.sin(a)], axis=1) * amplitude


def pairs(rot, layout):
    """(a, b) of every pair."""
    return [(i, i + rot // 2) if layout == HALF else (2 * i, 2 * i + 1) for i in range(rot // 2)]


def matrix(row, D, layout):
    """The D x D matrix that turns a vector: y = z M^T."""
    rot = len(row)
    M = np.eye(D)
    for i, (a, b) in enumerate(pairs(rot, layout)):
        c, s = row[i], row[rot // 2 + i]
        M[a, a], M[a, b], M[b, b], M[b, a] = c, -s, c, s
    return M


def _matrices(tab, pos, D, layout):
    """A matrix for every token; zeros for a position that is no row of the table."""
    known = {}
    out = np.zeros(pos.shape + (D, D))
    for at in np.ndindex(pos.shape):
        p = int(pos[at])
        if 0 <= p < len(tab):
            if p not in known:
                known[p] = matrix(tab[p], D, layout)
            out[at] = known[p]
    return out


def forward(x, tab, pos, layout, gain=0.0):
    """x [B, S, H, D], tab [positions, rot], pos [B, S] -> y, and sum |terms|.  tab None: no turn."""
    z = x
    if gain > 0:
        r = np.sqrt((x * x).mean(-1, keepdims=True))
        z = np.divide(gain * x, r, out=np.zeros_like(x), where=r > 0)
    if tab is None:
        return z, np.abs(z)
    M = _matrices(tab, pos, x.shape[-1], layout)
    return np.matmul(z, np.swapaxes(M, -1, -2)), np.matmul(np.abs(z), np.swapaxes(np.abs(M), -1, -2))


def backward(dy, x, tab, pos, layout, gain=0.0):
    """dx [B, S, H, D] from dy and the forward's x (None without a norm); also the size of the turned gradient's terms and of the norm's term."""
    if tab is None:
        d, size = dy, np.abs(dy)
    else:
        M = _matrices(tab, pos, dy.shape[-1], layout)
        d, size = np.matmul(dy, M), np.matmul(np.abs(dy), np.abs(M))
    if gain == 0:
        return d, size, np.zeros_like(size)
    xx = (x * x).sum(-1, keepdims=True)
    inv = np.divide(gain, np.sqrt(xx / x.shape[-1]), out=np.zeros_like(xx), where=xx > 0)
    safe = np.where(xx > 0, xx, 1.0)
    along, most = (x * d).sum(-1, keepdims=True) / safe, (np.abs(x) * size).sum(-1, keepdims=True) / safe
    return inv * (d - x * along), inv * size, inv * np.abs(x) * most
