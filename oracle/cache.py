"""fp64 oracle of the paged cache (NumPy): codes and scales, where rows are, and attention over them."""
from __future__ import annotations

import numpy as np

D, BLOCK = 64, 32
ROW_BYTES = {"bf16": 128, "e4m3": 64, "e2m1": 32}
LARGEST = {"e4m3": 448.0, "e2m1": 6.0}


def code_values(type_: str) -> np.ndarray:
    """The values of the non-negative codes, in code order (e4m3's last is NaN)."""
    man, low = (3, -6) if type_ == "e4m3" else (1, 0)
    out = []
    for c in range(128 if type_ == "e4m3" else 8):
        f, m = c >> man, c & ((1 << man) - 1)
        out.append(m * 2.0 ** (low - man) if f == 0 else (1 + m * 2.0 ** -man) * 2.0 ** (low + f - 1))
    if type_ == "e4m3":
        out[127] = np.nan
    return np.array(out)


def _bf16(x):
    """fp64 -> the nearest bf16 (ties to even) as fp64; x must be fp32 values."""
    b = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)
    nan = np.isnan(np.asarray(x, np.float32))
    return np.where(nan, np.uint16(0x7FC0), r).astype(np.uint16)


def encode(x, type_):
    """Bytes [..., ROW_BYTES] and scale bytes [..., 2] (None for bf16) of rows x [..., 64]."""
    x = np.asarray(x, np.float64)
    if type_ == "bf16":
        return _bf16(x).view(np.uint8).reshape(*x.shape[:-1], 128), None
    b = x.reshape(*x.shape[:-1], 2, BLOCK)
    finite = np.isfinite(b).all(-1)
    b = np.where(finite[..., None], b, 0.0)
    top = np.abs(b).max(-1)
    byte = np.zeros(top.shape, np.int64)
    for e in range(1, 255):  # the smallest exponent with which the largest magnitude fits
        byte = np.where(top > LARGEST[type_] * 2.0 ** (byte - 127), np.maximum(byte, e), byte)
    y = np.abs(b) * 2.0 ** (127.0 - byte)[..., None]
    vals = code_values(type_)
    vals = vals[:127] if type_ == "e4m3" else vals
    hi = np.clip(np.searchsorted(vals, y), 1, len(vals) - 1)
    lo = hi - 1
    dl, dh = y - vals[lo], vals[hi] - y
    code = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
    code = code | (np.signbit(b).astype(np.int64) << (7 if type_ == "e4m3" else 3))
    code = np.where(finite[..., None], code, 0).astype(np.uint8).reshape(x.shape)
    if type_ == "e2m1":
        code = code[..., 0::2] | (code[..., 1::2] << 4)
    return code, np.where(finite, byte, 255).astype(np.uint8)


def decode(codes, scale, type_):
    """fp64 rows [..., 64]."""
    codes = np.ascontiguousarray(codes)
    if type_ == "bf16":
        return (codes.view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    if type_ == "e2m1":
        codes = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], D)
    bits = 8 if type_ == "e4m3" else 4
    v = code_values(type_)
    v = np.concatenate([v, -v])[codes & ((1 << bits) - 1)]
    f = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return v * np.repeat(f, BLOCK, -1)


def inverse_length(rows):
    """1 / |row|, 0 for rows shorter than 2^-126; NaN for non-finite ones."""
    with np.errstate(all="ignore"):
        n = np.sqrt((rows * rows).sum(-1))
        inv = np.where(n < 2.0 ** -126, 0.0, 1 / np.where(n == 0, 1, n))
    return np.where(np.isfinite(rows).all(-1), inv, np.nan)


def tokens(first, length, T):
    """(row t, sequence, position) of every row that belongs to a sequence."""
    for s in range(len(length)):
        a, b = int(first[s]), int(first[s + 1])
        for t in range(max(a, 0), min(b, T)):
            yield t, s, int(length[s]) - b + t


def slot(table, s, pos, page, n_pages):
    """(page, place) or None."""
    if pos < 0 or pos // page >= table.shape[1]:
        return None
    p = int(table[s, pos // page])
    return (p, pos % page) if 0 <= p < n_pages else None


def sequence_slots(table, s, n, page, n_pages):
    """Pages, places and whether there is a slot, of positions 0 .. n-1."""
    pos = np.arange(max(0, n))
    p = pos // page
    here = p < table.shape[1]
    ids = np.where(here, table[s, np.minimum(p, table.shape[1] - 1)], -1)
    here &= (ids >= 0) & (ids < n_pages)
    return np.where(here, ids, 0), pos % page, here


def attend(q, rows_k, rows_v, k_inv, first, length, table, page, scale, shared, self_mask):
    """q [T][H][64]; rows_k, rows_v [n_pages][Hkv][page][64] as stored, k_inv [n_pages][Hkv][page] or None.
    (out [T][H][64], lse [T][H], spread [T][H][64]: the weighted sum of |v|, reach [T][H]: the largest
    |logit| but for the self mask); rows of no sequence are NaN."""
    T, H, _ = q.shape
    n_pages, Hkv = rows_k.shape[:2]
    out, spread = np.full((T, H, D), np.nan), np.full((T, H, D), np.nan)
    lse, reach = np.full((T, H), np.nan), np.zeros((T, H))
    last = -1
    for t, s, pos in tokens(first, length, T):
        if s != last:
            ids, place, here = sequence_slots(table, s, int(length[s]), page, n_pages)
            K, V = rows_k[ids, :, place], rows_v[ids, :, place]  # [n][Hkv][64]
            if shared:
                K = K * k_inv[ids, :, place][..., None]
            last = s
        seen = here[:max(0, pos + 1)].copy()
        n = len(seen)
        for h in range(H):
            hk = h // (H // Hkv)
            ok = seen.copy()
            if shared and n and ok[:-1].any():
                ok[-1] = False
            if not ok.any():
                out[t, h], spread[t, h], lse[t, h] = 0.0, 0.0, -np.inf
                continue
            z = scale * (K[:n, hk][ok] @ q[t, h])
            reach[t, h] = np.abs(z).max()
            if shared and not ok[:-1].any():
                z = z - self_mask
            m = z.max()
            w = np.exp(z - m)
            lse[t, h] = m + np.log(w.sum())
            w /= w.sum()
            out[t, h] = w @ V[:n, hk][ok]
            spread[t, h] = w @ np.abs(V[:n, hk][ok])
    return out, lse, spread, reach
