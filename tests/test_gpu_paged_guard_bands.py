"""Out-of-bounds writes and run-to-run determinism of the paged-cache calls, as tests/test_gpu_guard_bands.py has them for the others: every output,
workspace and updated buffer between sentinel bands, which have to hold after the call; what a call must leave alone is compared with its first
fill; every call runs twice and has to give the same bits."""
import ctypes

import pytest
import torch

from paper_2603_12201_b200 import binding as idxc
from tests.paged_util import DEV, bf16, gen, int32, tables
from tests.test_gpu_guard_bands import Guarded, _twice

pytestmark = pytest.mark.gpu


def guarded_cache(n_pages, P, H_kv, d, eight, g, bounds=True):
    kind = torch.float8_e4m3fn if eight else torch.bfloat16
    kv = [Guarded((n_pages, P, H_kv, d), kind) for _ in range(2)]
    for x in kv:
        x.t.copy_((torch.randn(x.t.shape, generator=g) * 20).clamp_(-400, 400).to(DEV))
    scales = [Guarded((n_pages, H_kv, P), torch.float32, 0.01) for _ in range(2)] if eight else []
    edge = [Guarded((n_pages, H_kv, 2, d), torch.bfloat16, 0.5)] if bounds else []
    handle = idxc.PagedCache(kv[0].t, kv[1].t, *([s.t for s in scales] or [None, None]), bounds=edge[0].t if bounds else None)
    return handle, kv, scales, edge


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("lens,P,H,H_kv,d,n_step,k", [([1], 16, 1, 1, 64, 1, 0), ([700, 0, 65, 3], 16, 10, 2, 128, 1, 0), ([257, 31], 48, 33, 1, 64, 1, 0), ([5000, 7], 64, 128, 2, 128, 1, 0),
                                                      ([100, 333], 32, 100, 1, 128, 3, 0), ([63] * 90, 16, 16, 8, 64, 1, 0), ([900, 0, 1], 128, 24, 3, 64, 4, 0), ([2000, 90], 16, 8, 8, 128, 1, 7),
                                                      ([3000, 500, 0], 64, 40, 5, 64, 2, 9)])
def test_attention(lens, P, H, H_kv, d, n_step, k, eight):
    g = gen(sum(lens) + H)
    B = len(lens)
    table, n_pages = tables(lens, P, g)
    handle, kv, scales, _ = guarded_cache(n_pages, P, H_kv, d, eight, g, bounds=False)
    q = bf16((B, n_step, H, d), g).to(DEV)
    table, n, max_len = table.to(DEV), int32(lens), max(lens)
    pages = torch.randint(-1, max(1, max(lens) // P), (B, H_kv, k), generator=g).to(torch.int32).to(DEV) if k else None
    out, lse = Guarded((B, n_step, H, d), torch.bfloat16), Guarded((B, n_step, H), torch.float32)
    work = Guarded((idxc.paged_attention_workspace_bytes(n_step, H, H_kv, d),), torch.uint8)
    kept = [x.t.clone() for x in kv + scales] + [table.clone(), q.clone()]

    def run():
        work.t.random_(0, 256)
        assert idxc.lib().idxc_paged_attention(handle._p, q.data_ptr(), H * d, table.data_ptr(), table.shape[1], n.data_ptr(), B, n_step, max_len, H,
                                               pages.data_ptr() if k else None, k, ctypes.c_float(0.1), out.t.data_ptr(), lse.t.data_ptr(), work.t.data_ptr(), work.nbytes,
                                               None) == idxc.OK
        work.check("workspace of the paged attention")
    _twice(run, [out, lse], "paged attention")
    for a, b in zip([x.t for x in kv + scales] + [table, q], kept):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    for x in kv + scales:
        x.check("cache")
    assert not torch.isnan(out.t.float()).any() and not torch.isnan(lse.t).any()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("lens,new,P,H_kv,d", [([0], [1], 16, 1, 64), ([15, 3], [1, 1], 16, 8, 128), ([70, 0], [500, 33], 48, 3, 128), ([100], [5000], 64, 2, 64), ([5], [90], 16, 12, 128)])
def test_append_and_gather(lens, new, P, H_kv, d, eight):
    g = gen(sum(new))
    table, n_pages = tables([a + b for a, b in zip(lens, new)], P, g)
    handle, kv, scales, edge = guarded_cache(n_pages, P, H_kv, d, eight, g)
    slots = torch.cat([table[b, torch.arange(n, n + m) // P].long() * P + torch.arange(n, n + m) % P for b, (n, m) in enumerate(zip(lens, new))]).to(DEV)
    T = slots.shape[0]
    row = bf16((T, 3, H_kv, d), g).to(DEV)
    first = [x.t.clone() for x in kv + scales + edge]
    _twice(lambda: idxc.paged_append(handle, row[:, 0], row[:, 2], slots), kv + scales + edge, "append")
    touched = torch.zeros(n_pages * P, dtype=torch.bool, device=DEV)
    touched[slots] = True
    touched = touched.view(n_pages, P)
    for x, before in zip(kv, first[:2]):
        assert torch.equal(x.t.view(torch.uint8)[~touched], before.view(torch.uint8)[~touched])
    for x, before in zip(scales, first[2:2 + len(scales)]):
        dark = ~touched[:, None, :].expand(-1, H_kv, -1)
        assert torch.equal(x.t[dark], before[dark])
    dark = ~touched.any(dim=1)
    assert torch.equal(edge[0].t[dark], first[-1][dark])
    out = [Guarded((T, H_kv, d), torch.bfloat16) for _ in range(2)]
    _twice(lambda: idxc.paged_gather(handle, slots, out[0].t, out[1].t), out, "gather")


@pytest.mark.parametrize("lens,P,H,H_kv,d,n_step", [([1], 16, 1, 1, 64, 1), ([777, 0, 16], 16, 32, 8, 128, 1), ([3000, 20], 48, 24, 3, 64, 3), ([1000], 16, 128, 1, 128, 1)])
def test_scores(lens, P, H, H_kv, d, n_step):
    g = gen(H)
    table, n_pages = tables(lens, P, g)
    bounds, q = bf16((n_pages, H_kv, 2, d), g).to(DEV), bf16((len(lens), n_step, H, d), g).to(DEV)
    B, ld = table.shape
    scores, n = Guarded((B * H_kv, ld + 3), torch.float32, 7.0), Guarded((B * H_kv,), torch.int32)
    table = table.to(DEV)
    _twice(lambda: idxc.page_scores(bounds, q, table, int32(lens), P, 0.1, scores.t, n.t), [scores, n], "scores")
    for b, m in enumerate(lens):
        assert bool((scores.t.view(B, H_kv, -1)[b, :, -(-m // P):] == 7.0).all())


@pytest.mark.parametrize("B,P,tokens", [(1, 16, 40), (37, 48, 500), (1300, 16, 4000), (5, 64, 9000)])
def test_tables(B, P, tokens):
    g = gen(B)
    new = torch.randint(0, 2 * tokens // B + 1, (B,), generator=g).to(torch.int32)
    ld, n_pages = 2 * (2 * tokens // B) // P + 3, 4 * tokens // P + 2 * B
    table, lens = Guarded((B, ld), torch.int32, -1), Guarded((B,), torch.int32, 5)
    free, count = Guarded((n_pages,), torch.int32), Guarded((1,), torch.int32, n_pages)
    free.t.copy_(torch.randperm(n_pages, generator=g).to(torch.int32).to(DEV))
    table.t[:, 0] = 3
    n = int(new.sum()) + 3
    slots, begin, start, seq = Guarded((n,), torch.int64), Guarded((B + 1,), torch.int32), Guarded((B,), torch.int32), Guarded((n,), torch.int32)
    new = new.to(DEV)
    every = [table, lens, free, count, slots, begin, start, seq]
    _twice(lambda: idxc.page_tables(table.t, lens.t, new, free.t, count.t, P, slots.t, begin.t, start.t, seq.t), every, "tables")
    pos, rows = torch.randint(-1, ld * P, (B, 9), generator=g).to(torch.int32).to(DEV), Guarded((B, 9), torch.int32)
    _twice(lambda: idxc.page_rows(table.t, pos, P, rows.t), [rows], "rows")
    keep = torch.randint(0, 30, (B,), generator=g).to(torch.int32).to(DEV)
    _twice(lambda: idxc.page_release(table.t, lens.t, keep, free.t, count.t, P), [table, lens, free, count], "release")
