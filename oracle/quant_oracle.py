"""fp64 oracle of the 8-bit paged cache and of the page tables.

TEST INFRASTRUCTURE ONLY.  The numbers of an e4m3 byte are listed from their definition (sign,
4 exponent bits with bias 7, 3 mantissa bits, subnormals, all ones: no number), and a value is
stored as the nearest of them, found by search, a tie as the one with an even byte.
"""
from __future__ import annotations

import math
from typing import Optional, Sequence

import numpy as np

BLOCK, LOWEST, HIGHEST, MOST = 16, -117, 119, 448.0


def e4m3_values() -> np.ndarray:
    """The number of each of the 256 bytes."""
    out = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = math.nan if c & 0x7F == 0x7F else (-x if c & 0x80 else x)
    return out


_VALUES = e4m3_values()


def encode_ref(x) -> np.ndarray:
    """Bytes of the e4m3 numbers nearest to x (already divided by its scale); past 448: 448; not finite: 0x7F."""
    x = np.asarray(x, dtype=np.float64)
    up = _VALUES[:127]                                   # 0 .. 448
    a = np.minimum(np.where(np.isfinite(x), np.abs(x), 0.0), MOST)
    hi = np.searchsorted(up, a).clip(1, 126)
    lo = hi - 1
    left, right = a - up[lo], up[hi] - a
    code = np.where((left < right) | ((left == right) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.signbit(x), code | 0x80, code)
    return np.where(np.isfinite(x), code, 0x7F).astype(np.uint8)


def decode_ref(code) -> np.ndarray:
    return _VALUES[np.asarray(code, dtype=np.uint8)]


def exponent_ref(amax: float) -> int:
    """The smallest e >= -117, at most 119, with amax <= 448 * 2^e."""
    e = LOWEST
    while e < HIGHEST and amax > math.ldexp(MOST, e):
        e += 1
    return e


def store_ref(codes, scales, new, slots) -> None:
    """New rows [n, D] of one sequence and head, at the pool's rows slots[n] (negative: nowhere), which
    follow one another in their blocks; codes uint8 [rows, D], scales [rows / 16], in place."""
    new = np.asarray(new, dtype=np.float64)
    i = 0
    while i < len(slots):
        if slots[i] < 0:
            i += 1
            continue
        block, first = slots[i] // BLOCK, slots[i] % BLOCK
        n = 1
        while i + n < len(slots) and slots[i + n] == slots[i] + n and slots[i + n] // BLOCK == block:
            n += 1
        x = new[i:i + n]
        e = exponent_ref(np.abs(x[np.isfinite(x)]).max(initial=0.0))
        if first > 0:
            old = exponent_of(scales[block])
            if e > old:
                rows = slice(block * BLOCK, block * BLOCK + first)
                codes[rows] = encode_ref(decode_ref(codes[rows]) * 2.0 ** (old - e))
            e = max(e, old)
        scales[block] = 2.0 ** e
        codes[slots[i]:slots[i] + n] = encode_ref(x * 2.0 ** -e)
        i += n


def exponent_of(scale: float) -> int:
    """Of a stored scale; 0: nothing is stored yet."""
    return LOWEST if scale == 0 else int(min(max(math.frexp(float(scale))[1] - 1, LOWEST), HIGHEST))


def assign_ref(table, free_pages, counts, page_size: int, positions: Sequence[int], seq_start: Optional[Sequence[int]],
               fresh: Optional[Sequence[int]], n_tokens: int, windows: Sequence[int], num_sink: int, block_band: bool,
               lacked_by=None):
    """(table, free_pages, counts, slots): the page tables after a call, entry by entry, and the rows of
    its tokens {(row, head): slot}.  lacked_by (in place): sequences that lacked a page, which get none until fresh."""
    table, free = np.array(table, dtype=np.int64), [int(x) for x in free_pages]
    batch, hkv, width = table.shape
    n_pages, n = len(free), max(0, min(int(counts[0]), len(free)))
    there = lambda x: 0 <= x < n_pages
    tokens = []
    for b in range(batch):
        first, count = (b, 1) if seq_start is None else (int(seq_start[b]), int(seq_start[b + 1]) - int(seq_start[b]))
        if positions[b] < 0 or count < 0 or first < 0 or first + count > n_tokens:
            count = 0
        tokens.append((first, count))
    for b in range(batch):
        p = int(positions[b])
        for g, w in enumerate(windows):
            lo = p - int(w) + 1
            if block_band:
                lo = min(lo, (p // 64 - -(-int(w) // 64) + 1) * 64)
            for i in range(width):
                old = p >= 0 and i * page_size >= num_sink and (i + 1) * page_size <= lo
                if there(table[b, g, i]) and ((fresh is not None and fresh[b]) or old):
                    if n < n_pages:
                        free[n] = int(table[b, g, i])
                        n += 1
                    table[b, g, i] = -1
    held = [False] * batch
    for b in range(batch if lacked_by is not None else 0):
        if fresh is not None and fresh[b]:
            lacked_by[b] = 0
        held[b] = lacked_by[b] != 0
    lacked, slots = 0, {}
    for b in range(batch):
        first, count = tokens[b]
        for g in range(hkv):
            for i in range(width):
                p0, p1 = int(positions[b]), int(positions[b]) + count - 1
                if count and not held[b] and p0 // page_size <= i <= p1 // page_size and not there(table[b, g, i]):
                    if n > 0:
                        n -= 1
                        table[b, g, i] = free[n]
                    else:
                        lacked += 1
                        if lacked_by is not None:
                            lacked_by[b] = 1
    for b in range(batch):
        first, count = tokens[b]
        for t in range(count):
            p = int(positions[b]) + t
            for g in range(hkv):
                page = table[b, g, p // page_size] if p // page_size < width else -1
                slots[first + t, g] = int(page) * page_size + p % page_size if there(page) else -1
    return table, np.array(free), np.array([n, lacked]), slots
