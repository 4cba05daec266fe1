"""Pins of the latent-cache oracle (no GPU): the 4-bit format against closed forms and exact arithmetic, the attention against
the sparse-attention oracle and brute force, the eviction against a brute-force choice."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import latent
from oracle import sparse_attn as oracle_sa



def bf16(a):
    return (np.asarray(a, dtype=np.float32).view(np.uint32) + 0x8000 >> 16 << 16).astype(np.uint32).view(np.float32).astype(np.float64)


def bits(a):
    return (np.asarray(a, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)


def test_scale_is_the_smallest_of_five_bits():
    rng = np.random.default_rng(0)
    for amax in np.concatenate([bf16(np.exp(rng.uniform(-20, 20, 300))), bf16([7.0, 14.0, 7.0 * 1.0625, 0.4375, 1.0, 7.03125])]):
        s = latent.group_scale(amax)
        m, e = np.frexp(s)
        assert (m * 32) == int(m * 32) and Fraction(s) * 7 >= Fraction(amax)
        below = np.ldexp((m * 32 - 1) / 32, e) if m > 0.5 else np.ldexp(31 / 32, e - 1)
        assert Fraction(below) * 7 < Fraction(amax)
    assert latent.group_scale(0.0) == 2.0 ** -100


def test_product_of_code_and_scale_is_exact_in_bf16():
    for m in range(16, 32):
        for code in range(-8, 8):
            assert bf16(code * m / 16.0) == code * m / 16.0


def test_rows_round_trip_and_known_bytes():
    x = np.zeros((1, 576))
    x[0, :8] = [7, -7, 1, 2, 3, 4, 5, 6]            # scale 1 in the first group
    x[0, 512:] = np.arange(64) - 32.0
    row = latent.quantize_rows(x)
    assert row[0, :4].tolist() == [(9 << 4) | 15, (13 << 4) | 11, (10 << 4) | 1, (14 << 4) | 12]     # columns 0 2 | 4 6 | 1 3 | 5 7
    assert row[0, 4:256].tolist() == [0x88] * 252
    assert np.array_equal(latent.row_values(row), x)
    rng = np.random.default_rng(1)
    y = bf16(rng.standard_normal((5, 576)))
    back = latent.row_values(latent.quantize_rows(y))
    assert np.array_equal(back[:, 512:], y[:, 512:])
    step = np.repeat(np.abs(y[:, :512]).reshape(5, 16, 32).max(axis=2) / 7.0, 32, axis=1)
    assert np.all(np.abs(back - y)[:, :512] <= step * (1 + 1 / 16) / 2)      # half a step, a step at most 1/16 wider than the tightest
    again = latent.row_values(latent.quantize_rows(back))
    assert np.all(np.abs(again - back) <= np.abs(back) * 2.0 ** -3)          # values already on a grid stay near it


def test_ties_go_to_the_even_code():
    x = np.zeros((1, 576))
    x[0, :5] = [7.0, 0.5, 1.5, -2.5, 3.5]
    back = latent.row_values(latent.quantize_rows(x))[0, :5]
    assert back.tolist() == [7.0, 0.0, 2.0, -2.0, 4.0]


def test_attention_agrees_with_the_sparse_oracle_and_masks():
    rng = np.random.default_rng(2)
    q, kv = bits(bf16(rng.standard_normal((3, 576)))), bits(bf16(rng.standard_normal((11, 576))))
    out, lse, spread, reach, p = latent.attention(q, kv, 0.07, np.array([11, 4, 0]))
    for r, n in ((0, 11), (1, 4)):
        o, l = oracle_sa.sparse_attention(q[None, r:r + 1], kv, np.arange(n, dtype=np.int32)[None], 512, 0.07)
        assert np.allclose(out[r], o[0, 0], atol=1e-14) and np.allclose(lse[r], l[0, 0])
    assert np.all(out[2] == 0) and lse[2] == -np.inf and np.all(p[2] == 0)
    assert np.allclose(p.sum(axis=1), [1, 1, 0]) and np.all(p[1, 4:] == 0) and np.all(spread >= np.abs(out) - 1e-12)
    m = np.zeros((3, 11), dtype=bool)
    m[:, [2, 5]] = True
    o2, _, _, _, _ = latent.attention(q, kv, 0.07, m)
    o3, _ = oracle_sa.sparse_attention(q[None], kv, np.array([[5, -1, 2]], dtype=np.int32), 512, 0.07)
    assert np.allclose(o2, o3[0], atol=1e-14)


@pytest.mark.parametrize("n,budget,recent", [(5, 8, 3), (8, 8, 8), (9, 8, 8), (9, 8, 0), (20, 7, 3), (20, 1, 1), (20, 1, 0)])
def test_eviction_by_brute_force(n, budget, recent):
    rng = np.random.default_rng(n * 100 + budget * 10 + recent)
    acc = rng.integers(0, 4, n).astype(np.float32)         # many ties
    keep = latent.evict(acc, n, budget, recent)
    assert len(keep) == min(n, budget) and np.all(np.diff(keep) > 0)
    if n > budget:
        assert set(range(n - recent, n)) <= set(keep.tolist())
        gone = [s for s in range(n - recent) if s not in keep]
        stay = [s for s in keep if s < n - recent]
        for g in gone:
            assert all(acc[s] > acc[g] or (acc[s] == acc[g] and s < g) for s in stay)
