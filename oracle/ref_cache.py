"""Plain CPU implementation of the attention block's cache side, in 64 bits: rotary positions, the 4-bit key/value cache, attention.

Layout and rules are those that include/spm.h states; nothing here is shared with the GPU code.
"""
from __future__ import annotations

import numpy as np


def rotate(x, positions, inv_freq, axis_of, gamma=None, eps=1e-6, neighbours=False):
    """x [rows, heads, hd]; positions [axes, rows]; returns float64."""
    x = np.asarray(x, np.float64)
    if gamma is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(gamma, np.float64)
    y = x.copy()
    for i, f in enumerate(np.asarray(inv_freq, np.float64)):
        angle = np.asarray(positions[axis_of[i]], np.float64) * f
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + len(inv_freq))
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def quantise(x):
    """Rows [..., hd] fp32 -> (codes [..., hd], scales fp16 [..., hd/32]); every operation is one fp32 operation."""
    x = np.asarray(x, np.float32)
    g = x.reshape(*x.shape[:-1], -1, 32)
    g = np.where(np.isnan(g), np.float32(0), g)
    at = np.abs(g).argmax(-1)                       # the lowest index of equals
    m = np.take_along_axis(g, at[..., None], -1)
    with np.errstate(over="ignore", divide="ignore", invalid="ignore"):
        d = np.clip(m * np.float32(-0.125), np.float32(-65504), np.float32(65504)).astype(np.float16)
        inv = np.where(d == 0, np.float32(0), np.float32(1) / d.astype(np.float32)).astype(np.float32)
        t = np.rint(g * inv)
    codes = np.clip(t, -8, 7).astype(np.int64) + 8
    return codes.reshape(x.shape).astype(np.uint8), d[..., 0]


def put(pages, page, head, offset, part, codes, scales):
    """One row of codes [hd] and scales [hd/32] of keys (part 0) or values (1) at token `offset` of a page, byte by byte."""
    hd = codes.size
    block = pages[page, head, offset // 16]
    tok = offset % 16
    for g in range(hd // 32):
        for b in range(16):
            block[part * 8 * hd + (g * 16 + tok) * 16 + b] = codes[32 * g + 2 * b] | codes[32 * g + 2 * b + 1] << 4
        at = 16 * hd + part * hd + (tok * (hd // 32) + g) * 2
        block[at:at + 2] = np.frombuffer(np.float16(scales[g]).tobytes(), np.uint8)


def get(pages, page, head, offset, part):
    """The row of `put`, as float64 values [hd]."""
    hd = pages.shape[3] // 18
    block = pages[page, head, offset // 16]
    tok = offset % 16
    code = np.empty(hd)
    for g in range(hd // 32):
        raw = block[part * 8 * hd + (g * 16 + tok) * 16:][:16]
        code[32 * g:32 * g + 32:2], code[32 * g + 1:32 * g + 32:2] = raw & 15, raw >> 4
    return (code - 8) * scales(pages, page, head, offset, part)


def scales(pages, page, head, offset, part):
    """The scale of each element of that row, as float64 values [hd]."""
    hd = pages.shape[3] // 18
    at = 16 * hd + part * hd + offset % 16 * (hd // 32) * 2
    return np.repeat(np.frombuffer(pages[page, head, offset // 16][at:at + hd // 16].tobytes(), np.float16).astype(np.float64), 32)


def places(lengths, row_start, n_rows):
    """(sequence, position) of each row, None for rows of no sequence."""
    out = [None] * n_rows
    for s, (a, b) in enumerate(zip(row_start[:-1], row_start[1:])):
        for i in range(a, min(b, n_rows)):
            out[i] = (s, lengths[s] - (b - i))
    return out


def page_of(pages, table, seq, pos, page_size):
    """Pool page that holds a token, None where there is none."""
    if pos < 0 or pos // page_size >= table.shape[1]:
        return None
    p = int(table[seq, pos // page_size])
    return p if 0 <= p < pages.shape[0] else None


def context(pages, table, seq, length, page_size, head):
    """(keys, values [n, hd], which of the first `length` tokens exist, 8 |scale| of the values' elements [n, hd])."""
    k, v, there, wide = [], [], [], []
    hd = pages.shape[3] // 18
    for t in range(max(0, length)):
        p = page_of(pages, table, seq, t, page_size)
        there.append(p is not None)
        for part, out in ((0, k), (1, v)):
            out.append(get(pages, p, head, t % page_size, part) if p is not None else np.zeros(hd))
        wide.append(np.zeros(hd) if p is None else 8 * np.abs(scales(pages, p, head, t % page_size, 1)))
    return np.array(k).reshape(-1, hd), np.array(v).reshape(-1, hd), np.array(there, bool), np.array(wide).reshape(-1, hd)


def attend(q, pages, table, lengths, row_start, scale):
    """q [rows, heads, hd] float64 -> (out, sum of p |v|, largest scale * sum |q k|, sum of p times what a value of its group can be), each
    [rows, heads, hd or 1]; rows of no sequence: NaN."""
    n_rows, heads, hd = q.shape
    kv_heads, page_size = pages.shape[1], pages.shape[2] * 16
    out = np.full(q.shape, np.nan)
    spread, reach, span = np.zeros(q.shape), np.zeros((n_rows, heads, 1)), np.zeros(q.shape)
    where = places(lengths, row_start, n_rows)
    kept = {}
    for i, at in enumerate(where):
        if at is None:
            continue
        seq, pos = at
        for h in range(heads):
            c = h // (heads // kv_heads)
            if (seq, c) not in kept:
                kept[seq, c] = context(pages, table, seq, min(lengths[seq], table.shape[1] * page_size), page_size, c)
            k, v, there, wide = kept[seq, c]
            see = there & (np.arange(len(there)) <= pos)
            if not see.any():
                out[i, h] = 0
                continue
            z = k[see] @ q[i, h] * scale
            p = np.exp(z - z.max())
            p /= p.sum()
            out[i, h] = p @ v[see]
            spread[i, h] = p @ np.abs(v[see])
            span[i, h] = p @ wide[see]
            reach[i, h] = (np.abs(k[see]) @ np.abs(q[i, h])).max() * abs(scale)
    return out, spread, reach, span
