"""fp64 oracles of the norm of each head, of the 8-bit cache and of decode attention over it.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

from . import attention as oa
from . import serving as so


def e4m3_values():
    """The value of each byte: a sign, four exponent bits with bias 7, three fraction bits; 127 and 255 are NaN."""
    b = np.arange(128)
    e, m = b >> 3, b & 7
    x = np.where(e > 0, 2.0 ** (e - 7.0) * (1 + m / 8), m * 2.0 ** -9)
    x[127] = np.nan
    return np.concatenate([x, -x])


def encode(x):
    """x [..., d] -> (values over the scale as e4m3 values, exponent bytes [...]): the smallest power of two, at least 2^-126, with
    the largest finite magnitude at most 448 of it; nearest values, ties to the even byte; NaN for what is not finite."""
    x = np.asarray(x, dtype=np.float64)
    fin = np.isfinite(x)
    most = np.where(fin, np.abs(x), 0.0).max(-1)
    frac, exp = np.frexp(most / 448.0)  # most = 448 frac 2^exp, frac in [1/2, 1)
    e = np.where(most > 0, np.where(frac == 0.5, exp - 1, exp), -126)
    e = np.maximum(e, -126)
    y = np.where(fin, x, 0.0) * 2.0 ** -e[..., None].astype(np.float64)
    grid = e4m3_values()[:127]
    a = np.abs(y)
    hi = np.clip(np.searchsorted(grid, a), 0, 126)  # the first value not below
    lo = np.maximum(hi - 1, 0)
    up = (grid[hi] - a < a - grid[lo]) | ((grid[hi] - a == a - grid[lo]) & (hi % 2 == 0)) | (hi == 0)
    q = np.copysign(np.where(up, grid[hi], grid[lo]), y)
    return np.where(fin, q, np.nan), (e + 127).astype(np.uint8)


def decode(k, v, scales):
    """bf16 pages' values (as float64) of an 8-bit cache: k [P, h, 16, d], v [P, h, d, 16] and scales [P, h, 2, 16], all bytes."""
    val = e4m3_values()
    p = np.where(scales == 0, 0.0, 2.0 ** (scales.astype(np.float64) - 127))
    return val[k] * p[:, :, 0, :, None], val[v] * p[:, :, 1, None, :]


def normalised(qkv, h_q, h_kv, d, w_q, w_k, eps):
    """The projection with its query and key heads normalised."""
    x = np.array(qkv, dtype=np.float64).reshape(len(qkv), h_q + 2 * h_kv, d)
    y = x[:, :h_q + h_kv]
    y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps)
    y[:, :h_q] *= 1.0 if w_q is None else w_q
    y[:, h_q:] *= 1.0 if w_k is None else w_k
    x[:, :h_q + h_kv] = y
    return x.reshape(len(qkv), -1)


def norm_split(qkv, k_cache, v_cache, page_table, seq_meta, h_q, h_kv, d, norm, rope):
    """norm (w_q, w_k, eps) or None, rope (freq, adjacent, pair_axis, positions) or None."""
    x = qkv if norm is None else normalised(qkv, h_q, h_kv, d, *norm)
    return so.rope_split(x, k_cache, v_cache, page_table, seq_meta, h_q, h_kv, d, *(rope or ([0.0], False)))


def decode_attention(q, k_cache, v_cache, page_table, seq_meta):
    """(out, sum of p |v|, largest sum of |q k| / sqrt(d) of a head) in float64; tokens of pages outside the pool do not count."""
    R, hq, d = q.shape
    out, mag, most = (np.full(s, np.nan) for s in ((R, hq, d), (R, hq, d), (R, hq)))
    g = hq // k_cache.shape[1]
    for r, m in enumerate(seq_meta):
        n = m[3] + 1
        ids = np.asarray(page_table)[r, np.arange(n) // 16]
        ok = (ids >= 0) & (ids < len(k_cache))
        if not ok.any():
            continue
        row = np.where(np.asarray(page_table)[r] < 0, 0, page_table[r]) % len(k_cache)
        K = oa.gather_kv(k_cache, row, n, 16, False)[ok]
        V = oa.gather_kv(v_cache, row, n, 16, True)[ok]
        with np.errstate(over="ignore", invalid="ignore"):
            for h in range(hq):
                k, v = K[:, h // g], V[:, h // g]
                s = k @ q[r, h] / np.sqrt(d)
                p = np.exp(s - s.max())
                p /= p.sum()
                out[r, h], mag[r, h] = p @ v, p @ np.abs(v)
                most[r, h] = (np.abs(k) @ np.abs(q[r, h])).max() / np.sqrt(d)
    return out, mag, most
