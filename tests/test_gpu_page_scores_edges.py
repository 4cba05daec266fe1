"""Scores of pages whose bounds are infinite, and of new tokens that hold zeros, infinities or no numbers, against the definition."""
import numpy as np
import pytest
import torch

from oracle import paged as oracle
from paper_2603_12201_b200 import binding as idxc
from tests.paged_util import DEV, bf16, gen, int32, tables
from tests.util import codes

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,H_kv,n_step", [(1, 1, 1), (8, 8, 1), (24, 3, 2), (32, 8, 4), (20, 2, 2), (100, 2, 3)])
@pytest.mark.parametrize("tokens", ["ordinary", "zeros", "no_numbers", "infinite"])
def test_against_the_definition(tokens, H, H_kv, n_step, d):
    """Up to 16 rows of a key head stay in registers; 20 lie in shared memory; 150 take three passes."""
    g = gen(H + d + n_step)
    P, lens, scale = 16, [16 * 75, 700], 0.07
    table, n_pages = tables(lens, P, g)
    middle, half = bf16((n_pages, H_kv, 1, d), g).float(), bf16((n_pages, H_kv, 1, d), g).float().abs()
    bounds = torch.cat((middle - half, middle + half), dim=2).to(torch.bfloat16)
    # by physical page: what one key column does there (both columns where two are given)
    kinds = [(-INF, None), (None, INF), (-INF, INF), (INF, -INF), (INF, INF), (-INF, -INF), (0.0, INF), (-INF, 0.0)]
    for p in range(n_pages):
        for h in range(H_kv):
            if p % 3 == 2:
                continue                                    # finite
            for n in range(1 + p % 2):
                lo, hi = kinds[(p // 3 + 3 * n + h) % len(kinds)]
                col = int(torch.randint(0, d, (1,), generator=g))
                if lo is not None:
                    bounds[p, h, 0, col] = lo
                if hi is not None:
                    bounds[p, h, 1, col] = hi
    q = bf16((2, n_step, H, d), g)
    q[:, :, :, torch.randperm(d, generator=g)[:d // 4]] = 0.0
    if tokens == "zeros":
        q[0] = 0.0
        q[1, :, ::2] = -0.0
    elif tokens == "no_numbers":
        q[0, 0, 0, 5] = NAN
        q[1, n_step - 1, H - 1] = NAN
    elif tokens == "infinite":
        q[0, 0, 0, 7] = INF
        q[1, n_step - 1, H - 1, d - 1] = -INF
    ld, group = table.shape[1], H // H_kv
    scores, n_out = torch.full((2 * H_kv, ld), 0.5, device=DEV), torch.empty(2 * H_kv, dtype=torch.int32, device=DEV)
    idxc.page_scores(bounds.to(DEV), q.to(DEV), table.to(DEV), int32(lens), P, scale, scores, n_out, 0, 0)
    got, qv, ev = scores.double().cpu().numpy(), oracle.bf16_rows(codes(q)), oracle.bf16_rows(codes(bounds))
    seen = set()
    for b, n in enumerate(lens):
        for h in range(H_kv):
            rows = qv[b, :, h * group:(h + 1) * group].reshape(-1, d)
            for p in range(oracle.ceil_div(n, P)):
                edge = ev[int(table[b, p]), h]
                want, have = oracle.page_score_any(rows, edge, float(np.float32(scale))), got[b * H_kv + h, p]
                seen.add("inf" if want == INF else "-inf" if want == -INF else "kept" if want > 1e38 else "finite")
                if abs(want) > 1e38:
                    assert have == want, (b, h, p, have, want)
                    continue
                # as for finite bounds: 2 d exact products (of a lane's columns or of 16 at a time) summed in steps of relative error at most
                # 2^-21, 16 of them or fewer, then scaled; columns of infinite magnitude are not among the terms of a finite sum
                with np.errstate(invalid="ignore"):
                    terms = np.maximum(rows * edge[0], rows * edge[1])
                reach = scale * np.where(np.isfinite(terms), np.abs(terms), 0.0).sum(axis=1).max()
                assert abs(have - want) <= 2.0 ** -17 * reach + 2.0 ** -23 * abs(want), (b, h, p, have, want)
    assert tokens != "ordinary" or {"inf", "finite"} <= seen      # (the inputs reach both; of zeros alone every score is 0)


def test_one_key_of_minus_infinity_hides_no_page():
    """A page with one key element of -inf is chosen for its other keys, and the attention over it takes them."""
    P, H, d, n = 16, 4, 64, 64
    g = gen(2)
    cache = idxc.PagedCache(*[torch.zeros((4, P, 1, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)],
                            bounds=torch.zeros((4, 1, 2, d), dtype=torch.bfloat16, device=DEV))
    q = (bf16((1, 1, H, d), g).abs() + 0.5).to(torch.bfloat16)
    k = bf16((n, 1, d), g) * 0.01
    k[20:24] = 2.0 * q[0, 0, 0] / q[0, 0, 0].norm()         # page 1 holds the keys that matter,
    k[25, 0, 3] = -INF                                      # and one that no token wants
    table = torch.arange(4, dtype=torch.int32, device=DEV)[None].contiguous()
    idxc.paged_append(cache, k.to(DEV), bf16((n, 1, d), g).to(DEV), torch.arange(n, device=DEV))
    scores, n_out = torch.zeros((1, 4), device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    idxc.page_scores(cache.bounds, q.to(DEV), table, int32([n]), P, 1.0, scores, n_out, 0, 0)
    sel = torch.empty((1, 1), dtype=torch.int32, device=DEV)
    idxc.topk_rows(scores, 1, sel, lens=n_out)
    assert sel.item() == 1 and torch.isfinite(scores).all()
    out, lse = idxc.paged_attention(cache, q.to(DEV), table, int32([n]), n, 1.0, pages=sel)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
