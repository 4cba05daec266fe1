"""Scores of pages from their bounds, and the selection that follows from them, against the oracle."""
import numpy as np
import pytest
import torch

from oracle import paged as oracle
from paper_2603_12201_b200 import binding as idxc
from tests.paged_util import DEV, bf16, gen, int32, tables
from tests.util import codes

pytestmark = pytest.mark.gpu
FORCED = float(np.float32(3e38))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,P,H,H_kv,n_step,first,last", [
    ([1], 16, 1, 1, 1, 0, 0), ([777, 0, 16], 16, 32, 8, 1, 1, 1), ([3000], 48, 16, 1, 1, 0, 2), ([100, 2000, 17], 16, 34, 2, 1, 2, 0), ([900, 5], 32, 64, 1, 1, 0, 0),
    ([500], 16, 128, 1, 1, 1, 1), ([333, 1500], 64, 12, 4, 4, 1, 1), ([600], 16, 100, 1, 3, 5, 5), ([40000], 16, 8, 2, 1, 1, 1),
    ([900, 33], 16, 24, 12, 1, 1, 1), ([500], 32, 18, 6, 1, 0, 0), ([700], 16, 22, 11, 1, 1, 0), ([300], 16, 256, 2, 1, 1, 1), ([2000], 1024, 16, 16, 1, 0, 1)])
def test_against_the_oracle(d, lens, P, H, H_kv, n_step, first, last):
    g = gen(sum(lens) + H + d)
    table, n_pages = tables(lens, P, g)
    middle, half = bf16((n_pages, H_kv, 1, d), g).float(), bf16((n_pages, H_kv, 1, d), g).float().abs()
    bounds = torch.cat((middle - half, middle + half), dim=2).to(torch.bfloat16)
    B, ld = table.shape
    if sum(lens) < 5000:
        table[0, 0] = -3
    row = bf16((B, n_step, H + 3, d), g)
    q = row.to(DEV)[:, :, :H]
    scores = torch.full((B * H_kv, ld + 2), 0.5, device=DEV)
    n_out = torch.full((B * H_kv,), -1, dtype=torch.int32, device=DEV)
    idxc.page_scores(bounds.to(DEV), q, table.to(DEV), int32(lens), P, 0.07, scores, n_out, first, last)
    got, qv, ev = scores.cpu().numpy(), oracle.bf16_rows(codes(row[:, :, :H])), oracle.bf16_rows(codes(bounds))
    assert n_out.cpu().tolist() == [oracle.ceil_div(n, P) for n in lens for _ in range(H_kv)]
    group = H // H_kv
    for b, n in enumerate(lens):
        pages = oracle.ceil_div(n, P)
        for h in range(H_kv):
            r = got[b * H_kv + h]
            assert np.all(r[pages:] == 0.5)
            for p in range(pages):
                if p < first or p >= pages - last:
                    assert r[p] == np.float32(FORCED)
                elif table[b, p] < 0:
                    assert r[p] == -np.float32(FORCED)
                elif pages < 200 or p % 37 == 0:
                    u, size = oracle.page_score(qv[b, :, h * group:(h + 1) * group].reshape(-1, d), ev[int(table[b, p]), h], 0.07)
                    # 2 d exact products summed in 2 d / 16 <= 16 matrix steps of relative error at most 2^-21 each (every row's error counts: the
                    # largest may change places), then scaled
                    reach = 0.07 * np.abs(np.maximum(qv[b, :, h * group:(h + 1) * group].reshape(-1, d) * ev[int(table[b, p]), h, 0],
                                                     qv[b, :, h * group:(h + 1) * group].reshape(-1, d) * ev[int(table[b, p]), h, 1])).sum(axis=1).max()
                    assert abs(r[p] - u) <= 2.0 ** -17 * reach + 2.0 ** -23 * abs(u), (b, h, p)


def test_scores_bound_every_key_and_feed_the_selection():
    P, H, H_kv, d, lens = 16, 8, 2, 64, [700, 130]
    g = gen(9)
    table, n_pages = tables(lens, P, g)
    k = bf16((n_pages, P, H_kv, d), g)
    cache = idxc.PagedCache(torch.zeros_like(k).to(DEV), torch.zeros_like(k).to(DEV), bounds=torch.zeros((n_pages, H_kv, 2, d), dtype=torch.bfloat16, device=DEV))
    for b, n in enumerate(lens):
        pos = torch.arange(n)
        slots = table[b, pos // P].long() * P + pos % P
        rows = k[table[b, pos // P].long(), pos % P].to(DEV)
        idxc.paged_append(cache, rows, rows, slots.to(DEV))
    q = bf16((2, 1, H, d), g).to(DEV)
    ld = (table.shape[1] + 3) // 4 * 4
    scores, n_out = torch.zeros((2 * H_kv, ld), device=DEV), torch.zeros(2 * H_kv, dtype=torch.int32, device=DEV)
    idxc.page_scores(cache.bounds, q, table.to(DEV), int32(lens), P, 1.0, scores, n_out, 0, 0)
    for b, n in enumerate(lens):
        for h in range(H_kv):
            x = torch.einsum("hd,ptd->hpt", q[b, 0, h * 4:h * 4 + 4].float(), cache.k[:, :, h].float())
            for p in range(n // P):
                assert scores[b * H_kv + h, p] >= x[:, table[b, p]].max() - 1e-3
    sel = torch.empty((2 * H_kv, 6), dtype=torch.int32, device=DEV)
    idxc.topk_rows(scores, 6, sel, lens=n_out)
    want = torch.topk(scores[0, :int(n_out[0])], 6).indices.sort().values
    assert torch.equal(sel[0].long(), want)
    out, lse = idxc.paged_attention(cache, q, table.to(DEV), int32(lens), 700, 0.1, pages=sel)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
