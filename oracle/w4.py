"""fp64 oracle of the products with 4-bit weights (NumPy): scales, zero points and codes by their definition, the values
they stand for, and the products."""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def bf16_values() -> np.ndarray:
    """Every finite bf16 value from zero on, ascending, as fp64 (its index is its bit pattern)."""
    return (np.arange(0x7F80, dtype=np.uint32) << 16).view(np.float32).astype(np.float64)


def quantize(w, type_, group, zeros):
    """(codes [N][K] uint8, scales [N][groups]: bf16 bits uint16 or bytes uint8, zero points [N][groups] uint8 or None)."""
    w = np.asarray(w, np.float64)
    N, K = w.shape
    groups = -(-K // group)
    codes = np.zeros((N, K), np.uint8)
    scales = np.zeros((N, groups), np.uint8 if type_ == "e2m1" else np.uint16)
    zps = np.zeros((N, groups), np.uint8) if zeros else None
    every = bf16_values()
    for n in range(N):
        for g in range(groups):
            x = w[n, g * group:(g + 1) * group]
            at = (n, slice(g * group, g * group + len(x)))
            finite = np.isfinite(x).all()
            x = np.where(np.isfinite(x), x, 0) if finite else np.zeros_like(x)
            if type_ == "e2m1":
                e = 0
                while 6 * 2.0 ** (e - 127) < np.abs(x).max():
                    e += 1
                y = np.abs(x) / 2.0 ** (e - 127)
                dist = np.abs(y[:, None] - E2M1)
                best = dist.min(1, keepdims=True)
                # of two as near, the even code
                c = np.array([min(np.flatnonzero(d == b), key=lambda i: i % 2) for d, b in zip(dist, best[:, 0])])
                codes[at] = c + 8 * np.signbit(x) if finite else 0
                scales[n, g] = e if finite else 255
                continue
            lo, hi = min(0.0, x.min()), max(0.0, x.max())
            steps, reach = (15, hi - lo) if zeros else (7, max(hi, -lo))
            i = int(np.searchsorted(steps * every, reach))
            s = every[i] or 1.0
            z = min(np.rint(-lo / s), 15) if zeros else 8
            codes[at] = np.clip(np.rint(x / s) + z, 0, 15) if finite else 0
            scales[n, g] = i if finite else 0x7FC0
            if zeros:
                zps[n, g] = z if finite else 0
    return codes, scales, zps


def values(codes, scales, zps, type_, group):
    """fp64 [N][K]."""
    K = codes.shape[1]
    at = np.arange(K) // group
    if type_ == "e2m1":
        f = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
        return np.where(codes & 8, -1.0, 1.0) * E2M1[codes & 7] * f[:, at]
    f = (scales.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    z = 8.0 if zps is None else zps.astype(np.float64)[:, at]
    return f[:, at] * (codes - z)


def pack_rows(codes):
    """uint8 [N][K/2], the even input in the low half."""
    return codes[:, 0::2] | (codes[:, 1::2] << 4)


def linear(a, codes, scales, zps, type_, group, bias=None):
    """(a W^T + bias, the sum of the magnitudes that its terms can reach on the way: the codes' own for int4)."""
    a = np.asarray(a, np.float64)
    w = values(codes, scales, zps, type_, group)
    out = a @ w.T
    if type_ == "e2m1":
        size = np.abs(a) @ np.abs(w).T
    else:
        at = np.arange(codes.shape[1]) // group
        f = (scales.astype(np.uint32) << 16).view(np.float32).astype(np.float64)[:, at]
        z = 8.0 if zps is None else zps.astype(np.float64)[:, at]
        size = np.abs(a) @ (f * (codes + z)).T
    if bias is not None:
        out, size = out + bias, size + np.abs(bias)
    return out, size
