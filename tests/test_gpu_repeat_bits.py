"""The order of all sums is fixed by the sizes, so a call on the same inputs gives the same bits however often it is made. What varies from call to call is
when copies land and warps run, so many calls in a row find what a comparison of one call with the oracle passes over: a slot of a ring that is
refilled while it is still read."""
import numpy as np
import pytest
import torch

from tests.latent_util import bf16_rows, cache_rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def idxc():
    from paper_2603_12201_b200 import binding
    binding.lib()
    return binding


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def same_every_time(call, n):
    """call() -> tensors; n calls, the first's outputs bit for bit."""
    words = lambda t: t.view({2: torch.int16, 4: torch.int32}[t.element_size()])
    first = [t.clone() for t in call()]
    differ = torch.zeros((), dtype=torch.int64, device=DEV)
    for _ in range(n):
        got = call()
        differ += torch.stack([(words(a) != words(b)).any() for a, b in zip(got, first)]).any()
    assert int(differ) == 0, f"{int(differ)} of {n} calls differ from the first"


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("lens,H,n_step", [([260], 128, 200), ([9000] * 40, 128, 1), ([5000, 3000, 777], 128, 1), ([77, 400], 20, 77), ([900] * 90, 16, 3)])
def test_latent_attention(idxc, lens, H, n_step, four):
    g, B = gen(n_step + H), len(lens)
    kv = cache_rows(sum(lens), four, g).to(DEV)
    q = bf16_rows(B * n_step * H, g, 0.5).view(B, n_step, H, 576).to(DEV)
    base = torch.tensor(np.concatenate([[0], np.cumsum(lens)[:-1]]), device=DEV)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    same_every_time(lambda: idxc.latent_attention(q, kv, base, n, max(lens) + 9, 512, 1 / 24), 1000)
    idxc.poll_device_status()


@pytest.mark.parametrize("H", [16, 128])
def test_selected_latent_rows(idxc, H):
    g, n_q, n_kv, k = gen(H), 300, 5000, 700
    kv = cache_rows(n_kv, True, g).to(DEV)
    q = bf16_rows(n_q * H, g, 0.5).view(n_q, H, 576).to(DEV)
    topk = torch.stack([torch.randperm(n_kv, generator=g)[:k] for _ in range(n_q)]).to(torch.int32).to(DEV)
    same_every_time(lambda: idxc.sparse_attention_q4(q, kv, topk, 512, 1 / 24), 500)
    idxc.poll_device_status()


def tables(lens, P, g):
    """Pages of all requests in no order: table, number of pages."""
    pages = [-(-n // P) for n in lens]
    perm = torch.randperm(sum(pages) + 5, generator=g).to(torch.int32)
    table, at = torch.full((len(lens), max(pages) + 1), -1, dtype=torch.int32), 0
    for b, n in enumerate(pages):
        table[b, :n] = perm[at:at + n]
        at += n
    return table.to(DEV), sum(pages) + 5


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv,n_step", [(64, 8, 1), (10, 5, 1), (64, 2, 4)])
def test_page_scores(idxc, H, Hkv, n_step, d):
    g, P = gen(H + d), 16
    lens = [3000 + 1777 * b for b in range(24)]
    table, n_pages = tables(lens, P, g)
    bounds = (torch.randn((n_pages, Hkv, 2, d), generator=g)).sort(dim=2).values.to(torch.bfloat16).to(DEV).contiguous()
    q = torch.randn((len(lens), n_step, H, d), generator=g).to(torch.bfloat16).to(DEV)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    scores = torch.zeros((len(lens) * Hkv, (table.shape[1] + 3) // 4 * 4), device=DEV)
    count = torch.empty((len(lens) * Hkv,), dtype=torch.int32, device=DEV)

    def call():
        idxc.page_scores(bounds, q, table, n, P, d ** -0.5, scores, count)
        return scores, count

    same_every_time(call, 1000)
    idxc.poll_device_status()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("H,Hkv,n_step", [(32, 8, 1), (32, 4, 2), (32, 2, 2), (32, 2, 5), (16, 2, 80)])
def test_paged_attention(idxc, H, Hkv, n_step, eight, d):
    """8, 16, 32, 80 and 640 rows of a key head."""
    g, P = gen(H + d), 32
    lens = [200 + 333 * b for b in range(24)]
    table, n_pages = tables(lens, P, g)
    k, v = [torch.randn((n_pages, P, Hkv, d), generator=g).to(torch.float8_e4m3fn if eight else torch.bfloat16).to(DEV) for _ in range(2)]
    scales = [torch.rand((n_pages, Hkv, P), generator=g).to(DEV) + 0.5 if eight else None for _ in range(2)]
    cache = idxc.PagedCache(k, v, *scales)
    q = torch.randn((len(lens), n_step, H, d), generator=g).to(torch.bfloat16).to(DEV)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    same_every_time(lambda: idxc.paged_attention(cache, q, table, n, max(lens), d ** -0.5), 500)
    idxc.poll_device_status()
