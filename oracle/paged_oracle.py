"""fp64 oracle of the paged cache: rotation, append, and attention through a page table.

TEST INFRASTRUCTURE ONLY.  A page holds page_size consecutive positions of one KV
head; table[b, g, i] is the page of positions i * page_size .. of head g of
sequence b, and a number outside [0, num_pages) an absent page.  The mask of a
query at position p is that of the rest of the oracle: keys j <= p with j < s, or
within the band of w (or of blocks).  All work is float64 on the stored values.
"""
from __future__ import annotations

import math
from typing import Optional, Sequence

import numpy as np

from .moa_oracle import _as64, visible_set


def rotate_ref(x, positions, inv_freq, interleaved: bool = False) -> np.ndarray:
    """x [T, H, D] with dimensions 0 .. 2 len(inv_freq) - 1 turned by positions[t] * inv_freq[i]."""
    out = _as64(x).copy()
    f = _as64(inv_freq)
    for t, p in enumerate(positions):
        for i in range(len(f)):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + len(f))
            c, s = math.cos(float(p) * f[i]), math.sin(float(p) * f[i])
            u, v = out[t, :, a].copy(), out[t, :, b].copy()
            out[t, :, a], out[t, :, b] = u * c - v * s, v * c + u * s
    return out


def token_rows(positions: Sequence[int], seq_start: Optional[Sequence[int]]):
    """[(row, sequence, position)] of every token that a call handles."""
    out = []
    for b, p in enumerate(positions):
        if p < 0:
            continue
        if seq_start is None:
            out.append((b, b, int(p)))
        else:
            out += [(t, b, int(p) + t - int(seq_start[b])) for t in range(int(seq_start[b]), int(seq_start[b + 1]))]
    return out


def slot_ref(table, num_pages: int, page_size: int, b: int, g: int, pos: int) -> int:
    """Row of the pool that holds a position, -1 where its page is absent."""
    i = pos // page_size
    if i >= table.shape[2]:
        return -1
    page = int(table[b, g, i])
    return page * page_size + pos % page_size if 0 <= page < num_pages else -1


def paged_attention_ref(q, k_pages, v_pages, table, positions, seq_start, windows, num_sink: int,
                        scale: Optional[float] = None, block: int = 0, prefix_table=None, prefix_len: int = 0):
    """(o, a, s), fp64 [T, H_q, D], [T, H_q, D] and [T, H_q]: the outputs, the weighted
    mean of |v|, and the largest scale * sum |q_d k_d| of a row's keys (what rounding
    errors are relative to).  Rows of no sequence are NaN; a row that sees no key is 0."""
    q, kp, vp = _as64(q), _as64(k_pages), _as64(v_pages)
    table = np.asarray(table)
    n_pages, ps, d = kp.shape
    kp, vp = kp.reshape(-1, d), vp.reshape(-1, d)
    hq, hkv = q.shape[1], table.shape[1]
    group = hq // hkv
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    o, a, s = np.full(q.shape, np.nan), np.zeros(q.shape), np.zeros(q.shape[:2])
    for t, b, p in token_rows(positions, seq_start):
        for g, w in enumerate(windows):
            keys = visible_set(p, int(w), num_sink, block)
            pages = np.full(len(keys), -1, dtype=np.int64)
            inside = keys < table.shape[2] * ps
            pages[inside] = table[b, g, keys[inside] // ps]
            if prefix_len:
                early = keys < prefix_len
                pages[early] = np.asarray(prefix_table)[g, keys[early] // ps]
            held = (pages >= 0) & (pages < n_pages)
            slots = pages[held] * ps + keys[held] % ps
            heads = slice(g * group, (g + 1) * group)
            if len(slots) == 0:
                o[t, heads] = 0.0
                continue
            k, v = kp[slots], vp[slots]
            sc = scale * (q[t, heads] @ k.T)
            e = np.exp(sc - sc.max(axis=1, keepdims=True))
            e /= e.sum(axis=1, keepdims=True)
            o[t, heads], a[t, heads] = e @ v, e @ np.abs(v)
            s[t, heads] = scale * (np.abs(q[t, heads]) @ np.abs(k).T).max(axis=1)
    return o, a, s
