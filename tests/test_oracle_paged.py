"""Pins of the paged-cache oracle (no GPU): block tables against a brute-force allocator's invariants, rows and bounds against closed forms,
attention against the sparse-attention oracle."""
import numpy as np
import pytest
import torch

import oracle as orc
from oracle import paged
from oracle import sparse_attn
from tests.util import codes


@pytest.mark.parametrize("P", [16, 48])
def test_every_page_has_one_owner_and_release_undoes(P):
    rng = np.random.default_rng(P)
    B, ld, n_pages = 9, 12, 60
    free = rng.permutation(n_pages)
    table, lens, count = np.full((B, ld), -1), np.zeros(B, dtype=np.int64), n_pages
    for step in range(30):
        new = rng.integers(0, 40, B)
        before = (table.copy(), lens.copy(), free.copy(), count)
        table, lens, count, begin, start, slots, seq = paged.page_tables(table, lens, new, free, count, P, int(new.sum()))
        held = [int(p) for b in range(B) for p in table[b, :paged.ceil_div(int(lens[b]), P)]]
        assert sorted(held + [int(p) for p in free[:count]]) == list(range(n_pages))
        ok = start >= 0
        assert np.all(ok[:-1] | ~ok[1:])                                  # once one is refused, all behind it are
        good = slots[slots >= 0]
        assert len(set(good.tolist())) == good.size == new[ok].sum()
        undone = paged.page_release(table, lens, before[1], free, count, P)
        assert np.array_equal(undone[0], before[0]) and np.array_equal(undone[1], before[1])
        assert undone[3] == before[3] and np.array_equal(undone[2][:before[3]], before[2][:before[3]])
        keep = rng.integers(0, lens + 1)
        table, lens, free, count = paged.page_release(table, lens, keep, free, count, P)


def test_slots_and_rows_agree():
    t, lens, count, begin, start, slots, seq = paged.page_tables([[3, 7, -1, -1], [0, 2, 5, -1]], [30, 33], [20, 1], [9, 8, 4], 3, 16, 25)
    assert t.tolist() == [[3, 7, 4, 8], [0, 2, 5, -1]] and lens.tolist() == [50, 34] and count == 1
    assert begin.tolist() == [0, 20, 21] and start.tolist() == [30, 33]
    assert slots[:3].tolist() == [7 * 16 + 14, 7 * 16 + 15, 4 * 16] and slots[20] == 5 * 16 + 1
    assert np.array_equal(paged.page_rows(t, np.arange(30, 50)[None, :], 16, [0])[0], slots[:20])
    assert paged.page_rows(t, np.array([[-1, 64, 63, 0]]), 16, [1]).tolist() == [[-1, -1, -1, 0]]
    assert slots[21:].tolist() == [-1] * 4 and seq.tolist() == [0] * 20 + [1] + [-1] * 4


def test_a_request_that_does_not_fit_the_table_is_refused_with_all_behind_it():
    t, lens, count, begin, start, slots, seq = paged.page_tables([[1, -1], [2, -1], [3, -1]], [16, 16, 16], [16, 17, 1], [5, 6, 7, 8], 4, 16, 40)
    assert start.tolist() == [16, -1, -1] and lens.tolist() == [32, 16, 16] and count == 3 and t.tolist() == [[1, 8], [2, -1], [3, -1]]
    assert np.all(slots[16:] == -1) and np.all(slots[:16] == 8 * 16 + np.arange(16))


def test_e4m3_values_are_torchs():
    c = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    assert np.array_equal(paged.e4m3_values(c.numpy()), c.view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)


def test_rounding_to_bf16_is_torchs():
    g = torch.Generator().manual_seed(0)
    x = torch.randn(2000, generator=g, dtype=torch.float64) * torch.exp(8 * torch.randn(2000, generator=g, dtype=torch.float64))
    x = torch.cat([x, torch.tensor([1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, -1 - 2.0 ** -8, 0.0], dtype=torch.float64)])
    assert np.array_equal(paged.to_bf16(x.numpy()), x.to(torch.bfloat16).double().numpy())


def test_bounds_hold_every_score():
    rng = np.random.default_rng(3)
    rows, q = rng.standard_normal((16, 64)), rng.standard_normal((5, 64))
    u, _ = paged.page_score(q, paged.bounds(rows), 0.3)
    assert u >= 0.3 * (q @ rows.T).max()
    one, _ = paged.page_score(q, paged.bounds(rows[:1]), 0.3)
    assert one == pytest.approx(0.3 * (q @ rows[0]).max(), rel=1e-12)


def test_attention_is_the_sparse_oracles():
    g = torch.Generator().manual_seed(5)
    q, kv = torch.randn((6, 64), generator=g).to(torch.bfloat16), torch.randn((30, 64), generator=g).to(torch.bfloat16)
    out, lse, spread, reach = paged.attention(paged.bf16_rows(codes(q)), paged.bf16_rows(codes(kv)), paged.bf16_rows(codes(kv)), 0.2, np.ones((6, 30), dtype=bool))
    o, z = sparse_attn.sparse_attention(codes(q)[None], codes(kv), np.arange(30)[None], 64, 0.2)
    assert np.allclose(out, o[0], atol=1e-12) and np.allclose(lse, z[0], atol=1e-12)
    none = paged.attention(paged.bf16_rows(codes(q)), paged.bf16_rows(codes(kv)), paged.bf16_rows(codes(kv)), 0.2, np.zeros((6, 30), dtype=bool))
    assert np.all(none[0] == 0) and np.all(np.isneginf(none[1]))


def test_quantised_rows():
    x = torch.randn((3, 64), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    c, s = paged.quantize_row(codes(x)[1])
    full, scales = orc.quantize_e4m3(codes(x))
    assert np.array_equal(c, full[1]) and s == scales[1]
    assert np.abs(paged.e4m3_values(c) * s - paged.bf16_rows(codes(x))[1]).max() <= 448 * s * 2.0 ** -4
