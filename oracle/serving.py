"""fp64 oracles of the token-level operators of a served model: the QKV split with position rotation, low-rank
adapters, and sampling.  Test infrastructure only."""
from __future__ import annotations

import math

import numpy as np


def rotate(x, angles, adjacent):
    """x [..., d] with its first 2 n dimensions turned by angles [..., n]."""
    n = angles.shape[-1]
    y = np.array(x, dtype=np.float64)
    i = np.arange(n)
    a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + n)
    c, s = np.cos(angles), np.sin(angles)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def token_places(seq_meta):
    """(request, cache position) of every row."""
    req = np.concatenate([np.full(m[2], r) for r, m in enumerate(seq_meta)])
    pos = np.concatenate([m[3] + np.arange(m[2]) for m in seq_meta])
    return req, pos


def rope_split(qkv, k_cache, v_cache, page_table, seq_meta, h_q, h_kv, d, inv_freq, adjacent, pair_axis=None, positions=None):
    """(q, k_cache, v_cache) after the call; pages outside the pool are skipped."""
    req, pos = token_places(seq_meta)
    x = np.asarray(qkv, dtype=np.float64).reshape(len(pos), h_q + 2 * h_kv, d)
    axis = np.zeros(len(inv_freq), int) if pair_axis is None else np.asarray(pair_axis)
    p = np.broadcast_to(pos, (int(axis.max()) + 1, len(pos))) if positions is None else np.atleast_2d(positions)
    angles = p[axis].T.astype(np.float64) * np.asarray(inv_freq, dtype=np.float64)  # [T, pairs]
    y = rotate(x, angles[:, None], adjacent)
    kc, vc = np.array(k_cache, dtype=np.float64), np.array(v_cache, dtype=np.float64)
    for t in range(len(pos)):
        page = page_table[req[t], pos[t] // 16]
        if 0 <= page < len(kc):
            kc[page, :, pos[t] % 16] = y[t, h_q:h_q + h_kv]
            vc[page, :, :, pos[t] % 16] = x[t, h_q + h_kv:]
    return y[:, :h_q], kc, vc


def lora_add(x, base, a, b, scale, seq_meta, adapter_ids):
    """(out, magnitude): magnitude is the sum of the adapter's terms without their signs."""
    out, mag = np.array(base, dtype=np.float64), np.zeros(base.shape)
    for m, i in zip(seq_meta, adapter_ids):
        if i < 0:
            continue
        rows = slice(m[1], m[1] + m[2])
        s = 1.0 if scale is None else float(scale[i])
        out[rows] += s * (x[rows] @ a[i].T) @ b[i].T
        mag[rows] += abs(s) * (np.abs(x[rows]) @ np.abs(a[i]).T) @ np.abs(b[i]).T
    return out, mag


def sample_row(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """(token, probability) of one row of logits."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, dtype=np.float64))
    best = x.max()
    if best == -np.inf:
        return -1, 0.0
    if not temperature > 0:
        return int(np.argmax(x)), 1.0
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    y = x[order]
    with np.errstate(invalid="ignore"):
        gap = np.where(y == best, 0.0, best - y)
        w = np.exp(-(gap / float(temperature)))
    w = np.where(np.isfinite(gap), w, 0.0)
    if top_k > 0:
        w = w[:top_k]
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        need = max(0.0, float(top_p)) * math.fsum(w)
        w = w[:max(1, int(np.count_nonzero(before < need)))]
    if min_p > 0:
        w = w[w >= min(1.0, float(min_p))]
    cum = np.cumsum(w)
    u = min(float(u), 1 - 2.0 ** -24) if u > 0 else 0.0
    at = min(int(np.searchsorted(cum, u * cum[-1], side="right")), len(w) - 1)
    return int(order[at]), float(w[at] / cum[-1])


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    get = lambda v, i, off: off if v is None else v[i]  # noqa: E731
    rows = [sample_row(x, get(temperature, i, 1.0), get(top_k, i, 0), get(top_p, i, 1.0), get(min_p, i, 0.0), u[i])
            for i, x in enumerate(logits)]
    return np.array([r[0] for r in rows], dtype=np.int32), np.array([r[1] for r in rows])
