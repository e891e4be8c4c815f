"""fp64 oracle of the per-head norm with position rotation and of its gradient (NumPy)."""
from __future__ import annotations

import numpy as np

D = 64


def _pairs(rot: int, interleaved: bool):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def turn(y, pos, freq, rot, interleaved, sign=1.0):
    """Rows y [T][H][64] turned by sign * pos * freq."""
    y = np.array(y, np.float64)
    a, b = _pairs(rot, interleaved)
    ang = sign * np.asarray(pos, np.float64)[:, None] * np.asarray(freq, np.float64)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    ya, yb = y[..., a].copy(), y[..., b].copy()
    y[..., a], y[..., b] = ya * c - yb * s, ya * s + yb * c
    return y


def norm_rotate(x, gain, pos, freq, rot, interleaved, eps):
    """x [T][H][64], gain [64] or [H][64] -> [T][H][64]."""
    x = np.asarray(x, np.float64)
    ms = (x * x).mean(-1, keepdims=True) + eps
    r = np.where(ms > 0, 1 / np.sqrt(np.where(ms > 0, ms, 1)), 0.0)
    return turn(x * r * gain, pos, freq, rot, interleaved)


def norm_rotate_bwd(x, gain, pos, freq, rot, interleaved, eps, dy):
    """(dx [T][H][64], dgain in gain's shape, and the sum of |terms| of dgain)."""
    x = np.asarray(x, np.float64)
    ms = (x * x).mean(-1, keepdims=True) + eps
    r = np.where(ms > 0, 1 / np.sqrt(np.where(ms > 0, ms, 1)), 0.0)
    u = turn(dy, pos, freq, rot, interleaved, -1.0)
    n = x * r
    terms = u * n
    axes = 0 if np.ndim(gain) == 2 else (0, 1)
    w = u * gain
    dx = r * (w - n * (w * n).mean(-1, keepdims=True))
    return dx, terms.sum(axes), np.abs(terms).sum(axes)


def heads_first(y, L):
    """[T][H][64] -> [T/L][H][L][64]."""
    T, H, _ = y.shape
    return np.ascontiguousarray(y.reshape(T // L, L, H, D).transpose(0, 2, 1, 3))


def tokens_first(y):
    """The inverse."""
    B, H, L, _ = y.shape
    return np.ascontiguousarray(y.transpose(0, 2, 1, 3).reshape(B * L, H, D))
