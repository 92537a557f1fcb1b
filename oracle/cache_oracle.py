"""fp64 oracle of the operators around the paged cache: head norms with the position rotation, the 8-bit format, attention of new tokens.

Written from the formulas, in numpy, without the library's code.  Functions return the result and, where it helps a test to derive how far an
fp32 evaluation may be off, the sizes of the terms it is made of.
"""
from __future__ import annotations

import numpy as np


def norm_rope(x, weight, positions, inv_freq, rotary_dim, interleaved, eps):
    """x [tokens, heads, 128] -> (y, sizes): y the result before rounding, sizes the sum of the absolute terms of each element."""
    y = np.array(x, dtype=np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    size = np.abs(y)
    if rotary_dim:
        half = rotary_dim // 2
        c = np.arange(half)
        first, second = (2 * c, 2 * c + 1) if interleaved else (c, c + half)
        angle = np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(inv_freq, dtype=np.float64)[None]
        cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
        a, b = y[..., first].copy(), y[..., second].copy()
        y[..., first], y[..., second] = a * cos - b * sin, b * cos + a * sin
        size[..., first] = size[..., second] = np.abs(a) + np.abs(b)
    return y, size


def _e4m3_grid():
    codes = np.arange(127, dtype=np.int64)                  # 0 .. 448; 127 is NaN
    e, m = codes >> 3, codes & 7
    return np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))


_GRID = _e4m3_grid()


def mx_scale(x):
    """Bytes e [..., 4]: 2^(e - 127) is the smallest power of two with max |x| <= 448 * 2^(e - 127) over the finite of 32 channels, 1 <= e <= 254."""
    a = np.abs(np.asarray(x, dtype=np.float64)).reshape(*x.shape[:-1], 4, 32)
    most = np.where(np.isfinite(a), a, 0.0).max(-1)
    e = np.full(most.shape, 1, dtype=np.int64)
    nz = most > 0
    k = np.floor(np.log2(most[nz])).astype(np.int64) - 10   # surely too small; then up until it fits
    for _ in range(6):
        k = np.where(most[nz] > 448.0 * 2.0 ** k, k + 1, k)
    e[nz] = np.clip(k + 127, 1, 254)
    return e.astype(np.uint8)


def mx_quantise(x):
    """Codes (uint8 [..., 128]) and scale bytes of x, ties to the even code."""
    x = np.asarray(x, dtype=np.float64)
    e = mx_scale(x)
    units = x.reshape(*e.shape, 32) * 2.0 ** (127.0 - e.astype(np.float64))[..., None]
    a = np.abs(units)
    finite = np.isfinite(a)
    a0 = np.where(finite, a, 0.0)
    hi = np.clip(np.searchsorted(_GRID, a0), 0, 126)        # the first code at or above
    lo = np.clip(hi - 1, 0, 126)
    up, down = _GRID[hi] - a0, a0 - _GRID[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)) | (_GRID[hi] == a0), hi, lo)
    code = np.where(finite, code, 127) | np.where(np.signbit(units) & finite, 128, 0)
    return code.astype(np.uint8).reshape(x.shape), e


def mx_values(codes, e):
    codes = np.asarray(codes)
    mag = np.where((codes & 127) == 127, np.nan, _GRID[np.minimum(codes & 127, 126)])
    v = np.where(codes & 128, -mag, mag)
    return (v.reshape(*e.shape, 32) * 2.0 ** (np.asarray(e, dtype=np.float64) - 127.0)[..., None]).reshape(codes.shape)


def paged_attention(q, held_k, held_v, page_size, table, q_start, kv_len, scale):
    """q [tokens, hq, 128], held_k / held_v [pages, hkv, page, 128]: out, lse, and for each output sum_u p_u |v_u|, for each row the largest
    sum_c |q_c k_c| * scale.  Hidden tokens take no part, whatever they hold; tokens of a page outside the pool are hidden."""
    q = np.asarray(q, dtype=np.float64)
    T, hq, d = q.shape
    pages, hkv = held_k.shape[:2]
    G = hq // hkv
    out, size = np.zeros((T, hq, d)), np.zeros((T, hq, d))
    lse, logit = np.full((T, hq), -np.inf), np.zeros((T, hq))
    for i in range(len(kv_len)):
        n, total = int(q_start[i + 1] - q_start[i]), int(kv_len[i])
        u = np.arange(total)
        page = np.asarray(table[i])[u // page_size] if total else np.zeros(0, dtype=np.int64)
        there = (page >= 0) & (page < pages)
        rows = slice(int(q_start[i]), int(q_start[i]) + n)
        see = there[None] & (u[None] <= (total - n + np.arange(n))[:, None])              # [n, total]
        some = see.any(1)
        for h in range(hkv):
            k = np.asarray(held_k[np.where(there, page, 0), h, u % page_size], dtype=np.float64)
            v = np.asarray(held_v[np.where(there, page, 0), h, u % page_size], dtype=np.float64)
            odd = np.nonzero((~np.isfinite(v)).any(1))[0]
            whole = np.where(np.isfinite(v), v, 0.0)
            for g in range(G if some.any() else 0):
                x = q[rows, h * G + g]
                z = np.where(see, x @ k.T * scale, -np.inf)
                m = np.where(some, z.max(1), 0.0)[:, None]
                p = np.exp(z - m)
                l = p.sum(1)
                p = p / np.where(some, l, 1.0)[:, None]
                y = p @ whole
                for key in odd:                                                           # only the rows that see it have part in it
                    for ch in np.nonzero(~np.isfinite(v[key]))[0]:
                        y[see[:, key], ch] += p[see[:, key], key] * v[key, ch]
                out[rows, h * G + g] = y
                size[rows, h * G + g] = p @ np.abs(whole)
                lse[rows, h * G + g] = np.where(some, m[:, 0] + np.log(np.where(some, l, 1.0)), -np.inf)
                logit[rows, h * G + g] = np.where(see, np.abs(x) @ np.abs(k).T * scale, 0.0).max(1)
    return out, lse, size, logit
