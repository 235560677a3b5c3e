"""Plain CPU implementation of attention over latent rows, in 64 bits: what is written, products of heads, absorbed and expanded attention.

Layout and rules are those that include/spm.h states; nothing here is shared with the GPU code.
"""
from __future__ import annotations

import numpy as np

from .ref_cache import page_of, places


def turn(x, positions, inv_freq, axis_of, neighbours):
    """x [rows, ..., rope] with the first 2 * len(inv_freq) elements turned; positions [axes, rows]."""
    x = np.asarray(x, np.float64)
    y = x.copy()
    n = len(inv_freq)
    for i, f in enumerate(np.asarray(inv_freq, np.float64)):
        angle = np.asarray(positions[axis_of[i]], np.float64) * f
        c, s = (v.reshape(-1, *[1] * (x.ndim - 2)) for v in (np.cos(angle), np.sin(angle)))
        a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + n)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def norm(x, gamma, eps):
    x = np.asarray(x, np.float64)
    return x if gamma is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(gamma, np.float64)


def context(pages, table, seq, length):
    """(rows [n, width] float64, which of the first `length` tokens exist)."""
    page_size = pages.shape[1]
    rows, there = [], []
    for t in range(max(0, min(length, table.shape[1] * page_size))):
        p = page_of(pages, table, seq, t, page_size)
        there.append(p is not None)
        rows.append(np.zeros(pages.shape[2]) if p is None else pages[p, t % page_size])
    return np.array(rows, np.float64).reshape(-1, pages.shape[2]), np.array(there, bool)


def _softmax(z):
    p = np.exp(z - z.max(-1, keepdims=True))
    return p / p.sum(-1, keepdims=True)


def attend(q, pages, table, lengths, row_start, scale, latent, w_k=None, w_v=None):
    """q [rows, heads, ...] float64 -> (out, sum of p |value|, largest |scale| sum |q key| of a seen token), rows of no sequence NaN. Without w_k
    and w_v the absorbed form: keys are whole rows, values their latent part. With them (float64 [heads, head, latent]) the expanded one, and then
    also the sum of p |w_v| |latent| and the largest |scale| |q| |w_k| |latent|: what sums made of latent vectors may be off by a part of."""
    n_rows, heads = q.shape[:2]
    size = latent if w_v is None else w_v.shape[1]
    out, spread, made = np.full((n_rows, heads, size), np.nan), np.zeros((n_rows, heads, size)), np.zeros((n_rows, heads, size))
    reach, reach_made = np.zeros((n_rows, heads, 1)), np.zeros((n_rows, heads, 1))
    kept = {}
    for i, at in enumerate(places(lengths, row_start, n_rows)):
        if at is None:
            continue
        seq, pos = at
        if seq not in kept:
            kept.clear()
            rows, there = context(pages, table, seq, lengths[seq])
            if w_k is None:
                kept[seq] = there, [(rows, rows[:, :latent])] * heads
            else:
                c, r = rows[:, :latent], rows[:, latent:]
                kept[seq] = there, [(np.concatenate((c @ w_k[h].T, r), 1), c @ w_v[h].T, np.abs(c) @ np.abs(w_k[h]).T, np.abs(c) @ np.abs(w_v[h]).T)
                                    for h in range(heads)]
        there, kv = kept[seq]
        see = np.flatnonzero(there & (np.arange(len(there)) <= pos))
        for h in range(heads):
            if not len(see):
                out[i, h] = 0
                continue
            k, v = kv[h][0][see], kv[h][1][see]
            p = _softmax(k @ q[i, h] * scale)
            out[i, h], spread[i, h] = p @ v, p @ np.abs(v)
            reach[i, h] = (np.abs(k) @ np.abs(q[i, h])).max() * abs(scale)
            if w_k is not None:
                made[i, h] = p @ kv[h][3][see]
                reach_made[i, h] = (kv[h][2][see] @ np.abs(q[i, h, :w_k.shape[1]])).max() * abs(scale)
    return (out, spread, reach) if w_k is None else (out, spread, reach, made, reach_made)
