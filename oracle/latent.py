"""Oracle for the latent-cache operators -- TEST INFRASTRUCTURE ONLY: the 4-bit row format, dense attention over latent rows,
head-summed attention weights, and the eviction of positions by accumulated weight. Everything in float64 from the stored
bits, straight from the definitions; nothing is blocked, fused or reordered.

Row format (416 bytes): 512 four-bit codes (nibble = code + 8; the little-endian word of columns 8g..8g+7 holds, from the
lowest nibble, columns 0 2 4 6 1 3 5 7 of the eight), 16 bf16 scales (one per 32 columns), 64 bf16 positional columns.
A group's scale is the smallest number of 5 significant bits that is at least max|x| / 7, and at least 2^-100;
code = x / scale to the nearest integer, ties to even.
"""
from __future__ import annotations

from fractions import Fraction

import numpy as np

from .sparse_attn import bf16_bits_to_f64

COLS, VALUE_COLS, GROUP, ROW_BYTES = 576, 512, 32, 416
NIBBLE_COLUMN = (0, 2, 4, 6, 1, 3, 5, 7)


def five_bits_up(x: float) -> float:
    """The smallest number of 5 significant bits that is >= x > 0."""
    m, e = np.frexp(x)                                  # m in [1/2, 1)
    return float(np.ldexp(np.ceil(m * 32.0) / 32.0, e))


def group_scale(amax: float) -> float:
    """max|x| / 7 rounded up to 5 bits. The quotient is taken exactly, so that a maximum of exactly 7 steps is seen as such."""
    amax = max(float(amax), 7.0 * 2.0 ** -100)
    s = five_bits_up(amax / 7.0)
    down = s * (1.0 - 2.0 ** -30)
    prev = five_bits_up(down * (1 - 2.0 ** -5)) if down > 0 else s          # the 5-bit number below s, or s itself
    if prev < s and Fraction(prev) * 7 >= Fraction(amax):
        s = prev
    return s


def quantize_rows(x: np.ndarray) -> np.ndarray:
    """x [n, 576] float64 (bf16 values) -> rows [n, 416] uint8."""
    x = np.asarray(x, dtype=np.float64)
    n = x.shape[0]
    out = np.zeros((n, ROW_BYTES), dtype=np.uint8)
    for r in range(n):
        for g in range(VALUE_COLS // GROUP):
            v = x[r, g * GROUP:(g + 1) * GROUP]
            s = group_scale(np.abs(v).max())
            out[r, 256 + 2 * g:258 + 2 * g] = np.array([np.float32(s).view(np.uint32) >> 16], dtype=np.uint16).view(np.uint8)
            code = np.clip(np.rint(v / s), -7, 7).astype(np.int64) + 8      # bf16 over a 5-bit number: halves come out exact
            for j, u in enumerate(code):
                c = g * GROUP + j
                k = NIBBLE_COLUMN.index(c % 8)
                out[r, (c // 8) * 4 + k // 2] |= np.uint8(u << (4 * (k % 2)))
    rope = (x[:, VALUE_COLS:].astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
    out[:, 288:] = np.ascontiguousarray(rope).view(np.uint8)
    return out


def row_values(rows: np.ndarray) -> np.ndarray:
    """rows [n, 416] uint8 or [n, 576] uint16 (bf16 bits) -> [n, 576] float64."""
    rows = np.ascontiguousarray(rows)
    if rows.dtype == np.uint16:
        return bf16_bits_to_f64(rows)
    c = np.arange(VALUE_COLS)
    k = np.array([NIBBLE_COLUMN.index(i) for i in range(8)])[c % 8]
    code = ((rows[:, (c // 8) * 4 + k // 2] >> (4 * (k % 2))) & 15).astype(np.float64) - 8.0
    scale = bf16_bits_to_f64(np.ascontiguousarray(rows[:, 256:288]).view(np.uint16))
    rope = bf16_bits_to_f64(np.ascontiguousarray(rows[:, 288:]).view(np.uint16))
    return np.concatenate([code * scale[:, c // GROUP], rope], axis=1)


def attention(q_bits, kv, scale, keys):
    """One sequence: q_bits [R, 576] uint16, kv [n] rows, keys [R] = how many leading rows each query row sees, or a bool
    mask [R, n]. Returns (out [R, 512], lse [R], spread [R, 512] = sum p |v|, reach [R] = scale * max_s sum |q||k|, p [R, n])."""
    q, rows = bf16_bits_to_f64(q_bits), row_values(kv)
    R, n = q.shape[0], rows.shape[0]
    keys = np.asarray(keys)
    mask = keys if keys.ndim == 2 else np.arange(n)[None, :] < keys[:, None]
    out, spread = np.zeros((R, VALUE_COLS)), np.zeros((R, VALUE_COLS))
    lse, reach, p = np.full(R, -np.inf), np.zeros(R), np.zeros((R, n))
    if n:
        with np.errstate(invalid="ignore"):
            x = np.where(mask, scale * (q @ rows.T), -np.inf)
        size = np.where(mask, abs(scale) * (np.abs(q) @ np.abs(rows).T), 0.0)
        for r in range(R):
            if not mask[r].any():
                continue
            m = x[r].max()
            e = np.exp(x[r] - m)
            z = e.sum()
            lse[r] = m + np.log(z)
            p[r] = e / z
            used = rows[mask[r]]
            out[r] = p[r][mask[r]] @ used[:, :VALUE_COLS]
            spread[r] = p[r][mask[r]] @ np.abs(used[:, :VALUE_COLS])
            reach[r] = size[r].max()
    return out, lse, spread, reach, p


def evict(acc, n: int, budget: int, recent: int) -> np.ndarray:
    """Positions of a sequence that stay, ascending: the newest `recent`, and the largest acc among the others (ties: lowest)."""
    if n <= budget:
        return np.arange(n)
    old = n - recent
    order = np.argsort(-np.asarray(acc[:old], dtype=np.float64), kind="stable")[:budget - recent]
    return np.sort(np.concatenate([order, np.arange(old, n)]))
