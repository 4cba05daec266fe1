"""A cache that has no page yet: every token sees nothing, every page of a request is none of the cache's."""
import pytest
import torch

from paper_2603_12201_b200 import binding as idxc
from tests.paged_util import DEV, int32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,H,H_kv,n_step", [(1, 8, 8, 1), (3, 16, 2, 2), (300, 8, 4, 1), (2, 32, 1, 2), (2, 16, 2, 40), (200, 64, 1, 1)])
def test_attention_sees_nothing(B, H, H_kv, n_step, d, eight):
    P = 16
    kv = torch.empty((0, P, H_kv, d), dtype=torch.float8_e4m3fn if eight else torch.bfloat16, device=DEV)
    scales = [torch.empty((0, H_kv, P), device=DEV) if eight else None for _ in range(2)]
    cache = idxc.PagedCache(kv, kv.clone(), *scales)
    table = torch.zeros((B, 5), dtype=torch.int32, device=DEV)
    q = torch.randn((B, n_step, H, d), device=DEV).to(torch.bfloat16)
    pages = torch.zeros((B, H_kv, 2), dtype=torch.int32, device=DEV)
    for sel in (None, pages):
        out, lse = idxc.paged_attention(cache, q, table, int32([70] * B), 80, 0.1, pages=sel)
        assert not out.any() and bool(torch.isneginf(lse).all())
    idxc.poll_device_status()


def test_rows_and_scores():
    P, H_kv, d = 16, 2, 64
    kv = torch.empty((0, P, H_kv, d), dtype=torch.bfloat16, device=DEV)
    cache = idxc.PagedCache(kv, kv.clone(), bounds=torch.empty((0, H_kv, 2, d), dtype=torch.bfloat16, device=DEV))
    rows, slots = torch.ones((3, H_kv, d), dtype=torch.bfloat16, device=DEV), torch.arange(3, device=DEV)
    idxc.paged_append(cache, rows, rows, slots)
    k, v = torch.ones_like(rows), torch.ones_like(rows)
    idxc.paged_gather(cache, slots, k, v)
    assert not k.any() and not v.any()
    scores, n = torch.zeros((H_kv, 4), device=DEV), torch.zeros(H_kv, dtype=torch.int32, device=DEV)
    idxc.page_scores(cache.bounds, torch.ones((1, 1, 4, d), dtype=torch.bfloat16, device=DEV), torch.zeros((1, 4), dtype=torch.int32, device=DEV), int32([40]), P, 1.0,
                     scores, n, 1, 0)
    low = torch.tensor(-3e38).item()
    assert n.tolist() == [3, 3] and scores[:, 1:].tolist() == [[low, low, 0.0]] * 2 and bool((scores[:, 0] == 3e38).all())
