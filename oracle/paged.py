"""Oracle for serving from a paged key/value cache -- TEST INFRASTRUCTURE ONLY: block tables and slots, rows in bf16 or 8 bits, the bounds of
pages and the scores they allow, attention over pages. One request, one page, one row at a time; computed numbers in float64 from the stored
bits, straight from the definitions.

A page holds P positions; position s of request b lies in row s % P of physical page table[b, s // P], and its slot is that page's
number times P plus the row.
"""
from __future__ import annotations

import numpy as np

from . import quantize_e4m3
from .sparse_attn import bf16_bits_to_f64


def ceil_div(a: int, b: int) -> int:
    return -(-a // b)


def page_tables(table, lens, new_tokens, free_pages, free_count: int, P: int, n_slots: int):
    """Returns (table, lens, free_count, token_begin, start, slots, seq) after the new tokens have their pages."""
    table, lens = np.array(table, dtype=np.int64), np.array(lens, dtype=np.int64)
    B, ld = table.shape
    slots, seq = np.full(n_slots, -1, dtype=np.int64), np.full(n_slots, -1, dtype=np.int64)
    begin, start = np.zeros(B + 1, dtype=np.int64), np.full(B, -1, dtype=np.int64)
    open_ = True
    for b in range(B):
        n = int(new_tokens[b])
        begin[b + 1] = begin[b] + n
        have, want = ceil_div(int(lens[b]), P), ceil_div(int(lens[b]) + n, P)
        open_ = open_ and want <= ld and want - have <= free_count and begin[b + 1] <= n_slots
        if open_:
            start[b] = lens[b]
            for p in range(have, want):
                free_count -= 1
                table[b, p] = free_pages[free_count]
            lens[b] += n
        for t in range(int(begin[b]), min(int(begin[b + 1]), n_slots)):
            seq[t] = b
            if open_:
                s = int(start[b]) + t - int(begin[b])
                page = int(table[b, s // P])
                slots[t] = page * P + s % P if page >= 0 else -1
    return table, lens, free_count, begin, start, slots, seq


def page_release(table, lens, keep, free_pages, free_count: int, P: int):
    """Returns (table, lens, free_pages, free_count) after every request has been cut to keep[b] positions; entries that are no page (below 0) stay off the stack."""
    table, lens, free_pages = np.array(table, dtype=np.int64), np.array(lens, dtype=np.int64), np.array(free_pages, dtype=np.int64)
    back = []
    for b in range(table.shape[0]):
        kept = min(int(lens[b]), max(int(keep[b]), 0))
        for p in range(ceil_div(kept, P), min(ceil_div(int(lens[b]), P), table.shape[1])):
            if table[b, p] >= 0:
                back.append(int(table[b, p]))
            table[b, p] = -1
        lens[b] = kept
    for page in reversed(back):
        if free_count < free_pages.shape[0]:
            free_pages[free_count] = page
            free_count += 1
    return table, lens, free_pages, free_count


def page_rows(table, positions, P: int, seq=None):
    out = np.full(positions.shape, -1, dtype=np.int64)
    B, ld = table.shape
    for r in range(positions.shape[0]):
        b = r if seq is None else int(seq[r])
        if not 0 <= b < B:
            continue
        for j, s in enumerate(positions[r]):
            if s >= 0 and s // P < ld and table[b, s // P] >= 0:
                out[r, j] = int(table[b, s // P]) * P + int(s) % P
    return out


_E4M3 = None


def e4m3_values(codes) -> np.ndarray:
    """float64 values of e4m3 codes (uint8), from the format: sign, 4 exponent bits of bias 7, 3 mantissa bits; 0x7F is no number."""
    global _E4M3
    if _E4M3 is None:
        c = np.arange(256)
        e, m = (c >> 3) & 15, c & 7
        v = np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7.0), m / 8.0 * 2.0 ** -6)
        v = np.where((c & 127) == 127, np.nan, v)
        _E4M3 = np.where(c & 128, -v, v)
    return _E4M3[np.asarray(codes)]


def quantize_row(bits):
    """One row of one head, bf16 bits [d] -> (codes, scale)."""
    codes, scale = quantize_e4m3(np.ascontiguousarray(bits).reshape(1, -1))
    return codes[0], scale[0]


def to_bf16(a) -> np.ndarray:
    """float64 -> the nearest bf16 (ties to even), as float64; for values within bf16's normal range."""
    a = np.asarray(a, dtype=np.float64)
    m, e = np.frexp(a)
    return np.ldexp(np.rint(m * 256.0), e - 8)


def bounds(rows) -> np.ndarray:
    """rows [n, d] as they read back in bf16 -> [2, d]: smallest and largest value of every column."""
    return np.stack([rows.min(axis=0), rows.max(axis=0)])


def page_score(q, edge, scale: float):
    """q [R, d], edge [2, d] -> (the largest score a key within the bounds could reach, the sum of magnitudes of the row where it is largest)."""
    terms = np.maximum(q * edge[0], q * edge[1])
    return scale * terms.sum(axis=1).max(), abs(scale) * np.abs(terms).sum(axis=1).max()


def page_score_any(q, edge, scale: float) -> float:
    """page_score for any bit patterns: a product of 0 and an infinity counts as 0, a row whose sum is no number as 3e38."""
    def product(x, y):
        with np.errstate(invalid="ignore"):
            return np.where(((x == 0) & np.isinf(y)) | ((y == 0) & np.isinf(x)), 0.0, x * y)
    best = -np.inf
    for row in q:
        with np.errstate(invalid="ignore"):
            total = scale * np.maximum(product(row, edge[0]), product(row, edge[1])).sum()
        best = max(best, float(np.float32(3e38)) if np.isnan(total) else total)
    return best


def attention(q, k, v, scale: float, mask):
    """q [R, d], k, v [n, d] float64, mask [R, n]. Returns out [R, d], lse [R], spread [R, d] = sum p |v|, reach [R] = scale * max_s sum |q||k|."""
    R, n = q.shape[0], k.shape[0]
    out, spread = np.zeros((R, v.shape[1])), np.zeros((R, v.shape[1]))
    lse, reach = np.full(R, -np.inf), np.zeros(R)
    if n == 0:
        return out, lse, spread, reach
    for r in range(R):
        use = mask[r]
        if not use.any():
            continue
        x = scale * (k[use] @ q[r])
        m = x.max()
        e = np.exp(x - m)
        lse[r] = m + np.log(e.sum())
        p = e / e.sum()
        out[r], spread[r] = p @ v[use], p @ np.abs(v[use])
        reach[r] = (abs(scale) * (np.abs(k[use]) @ np.abs(q[r]))).max()
    return out, lse, spread, reach


def bf16_rows(bits) -> np.ndarray:
    return bf16_bits_to_f64(bits)
