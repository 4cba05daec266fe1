"""Out-of-bounds writes and run-to-run determinism of the latent-cache calls, as tests/test_gpu_guard_bands.py has them for the others: every
output, workspace and updated buffer between sentinel bands, which have to hold after the call; entries that a call must leave alone are
compared with their first fill; every call runs twice and has to give the same bits."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2603_12201_b200 import binding as idxc
from tests.latent_util import bf16_rows, cache_rows
from tests.test_gpu_guard_bands import Guarded, _twice

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SCALE = 1 / 24


def gen(seed):
    return torch.Generator().manual_seed(seed)


def at(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def ragged(lens, gap=2):
    """First rows of sequences that lie one behind the other with a gap, and the rows of the cache."""
    base, row = [], gap
    for n in lens:
        base.append(row)
        row += n + gap
    return torch.tensor(base, dtype=torch.int64, device=DEV), row


def int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("lens,H,n_step", [([1], 1, 1), ([700, 0, 65, 3], 5, 1), ([64, 129, 1], 64, 1), ([257, 31], 33, 3), ([900, 0, 1], 128, 1), ([100, 333], 70, 2),
                                           ([63] * 90, 16, 1), ([130] * 40, 100, 1), ([5000, 7], 128, 2)])
def test_dense_attention(lens, H, n_step, four):
    g = gen(sum(lens) + H)
    B, (base, rows) = len(lens), ragged(lens)
    kv = cache_rows(rows, four, g).to(DEV)
    q = bf16_rows(B * n_step * H, g).view(B, n_step, H, 576).to(DEV)
    n, max_len = int32(lens), max(lens) + 7
    out, lse = Guarded((B, n_step, H, 512), torch.bfloat16), Guarded((B, n_step, H), torch.float32)
    work = Guarded((idxc.latent_attention_workspace_bytes(B, n_step, max_len, H),), torch.uint8)
    kept = kv.clone(), q.clone()

    def run():
        work.t.random_(0, 256)
        assert idxc.lib().idxc_latent_attention(at(q), at(kv), int(four), rows, at(base), at(n), B, n_step, max_len, H, 576, 512, ctypes.c_float(SCALE), at(out.t), at(lse.t),
                                                at(work.t), work.nbytes, None) == idxc.OK
        work.check("workspace of the dense attention")
    _twice(run, [out, lse], "dense attention")
    assert torch.equal(kv.view(torch.uint8), kept[0].view(torch.uint8)) and torch.equal(q, kept[1])
    assert torch.isfinite(out.t.float()).all() and not torch.isnan(lse.t).any()


@pytest.mark.parametrize("n_q,H,k_top", [(1, 1, 1), (3, 128, 65), (70, 16, 130), (5, 64, 2048), (80, 100, 200), (200, 128, 63)])
def test_sparse_attention_over_4_bit_rows(n_q, H, k_top):
    g = gen(n_q + H)
    rows = 3000
    kv = cache_rows(rows, True, g).to(DEV)
    q = bf16_rows(n_q * H, g).view(n_q, H, 576).to(DEV)
    topk = torch.randint(-50, rows + 50, (n_q, k_top), generator=g, dtype=torch.int32)
    topk[0] = -1
    topk = topk.to(DEV)
    out, lse = Guarded((n_q, H, 512), torch.bfloat16), Guarded((n_q, H), torch.float32)
    work = Guarded((idxc.latent_attention_workspace_bytes(n_q, 1, k_top, H),), torch.uint8)

    def run():
        work.t.random_(0, 256)
        assert idxc.lib().idxc_sparse_attention_q4(at(q), at(kv), at(topk), None, n_q, rows, H, 576, 512, k_top, ctypes.c_float(SCALE), at(out.t), at(lse.t), at(work.t),
                                                   work.nbytes, None) == idxc.OK
        work.check("workspace of the sparse attention")
    _twice(run, [out, lse], "sparse attention over 4-bit rows")
    assert bool((out.t[0] == 0).all()) and bool(torch.isneginf(lse.t[0]).all())


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("lens,H,n_step,beta", [([1], 1, 1, 1.0), ([127, 0, 300], 100, 1, 0.5), ([129, 5], 16, 4, 1.0), ([1000, 257], 128, 2, 0.0)])
def test_dense_weights(lens, H, n_step, beta, four):
    g = gen(sum(lens) + H)
    B, (base, rows) = len(lens), ragged(lens)
    kv = cache_rows(rows, four, g).to(DEV)
    q = bf16_rows(B * n_step * H, g).view(B, n_step, H, 576).to(DEV)
    n = int32(lens)
    _, lse = idxc.latent_attention(q, kv, base, n, max(lens), 512, SCALE)
    acc = Guarded((B, max(lens) + 5), torch.float32, fill=7.0)
    _twice(lambda: idxc.attention_weights(q, kv, lse, acc.t, SCALE, kv_base=base, lens=n, max_len=max(lens), beta=beta), [acc], "dense weights")
    for b, length in enumerate(lens):
        assert bool((acc.t[b, length:] == 7).all()), "entries behind a sequence's length were written"


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("H", [3, 128])
def test_weights_of_a_selection(H, four):
    g = gen(H)
    rows, B, k, ld = 900, 3, 333, 700
    kv = cache_rows(rows, four, g).to(DEV)
    q = bf16_rows(B * H, g).view(B, H, 576).to(DEV)
    topk = torch.stack([torch.randperm(1000, generator=g)[:k] for _ in range(B)]).to(torch.int32)      # positions at or past ld, and past the cache
    topk[:, ::9] = -1
    lse = torch.full((B, H), 3.0, device=DEV)
    acc = Guarded((B, ld), torch.float32, fill=7.0)
    _twice(lambda: idxc.attention_weights(q, kv, lse, acc.t, SCALE, topk=topk.to(DEV)), [acc], "weights of a selection")
    named = torch.zeros((B, 1000), dtype=torch.bool)
    for b in range(B):
        named[b, topk[b][topk[b] >= 0].long()] = True
    assert bool((acc.t[~named[:, :ld].to(DEV)] == 7).all()), "positions that are not selected were written"


@pytest.mark.parametrize("n", [1, 31, 500])
def test_rows_in_4_bits(n):
    g = gen(n)
    x = bf16_rows(n, g).to(DEV)
    cache = Guarded((n, 416), torch.uint8)
    _twice(lambda: idxc.quantize_q4(x, cache.t), [cache], "quantiser")
    wide = Guarded((n + 9, 416), torch.uint8, fill=3)
    dst = (torch.randperm(n + 9, generator=g)[:n]).to(DEV)
    dst[0] = n + 9
    _twice(lambda: idxc.quantize_q4(x, wide.t, dst_rows=dst), [wide], "quantiser, scattered")
    left = torch.ones(n + 9, dtype=torch.bool, device=DEV)
    left[dst[1:]] = False
    assert bool((wide.t[left] == 3).all()), "rows that no token goes to were written"
    out = Guarded((n, 576), torch.bfloat16)
    _twice(lambda: idxc.dequantize_q4(cache.t, out.t), [out], "read-back")
    src = torch.randint(-2, n + 2, (n,), generator=g).to(DEV)
    _twice(lambda: idxc.dequantize_q4(cache.t, out.t, src_rows=src), [out], "read-back, gathered")


@pytest.mark.parametrize("ld,lens,budget,recent", [(1, [1, 0], 1, 0), (333, [333, 100, 7], 99, 13), (16384, [16384, 9000], 1000, 0), (16385, [16385, 3], 1001, 1000), (50001, [50001], 50000, 1)])
def test_choice(ld, lens, budget, recent):
    acc = torch.rand((len(lens), ld), generator=gen(ld)).to(DEV)
    keep, new = Guarded((len(lens), budget), torch.int32), Guarded((len(lens),), torch.int32)
    kept = acc.clone()
    _twice(lambda: idxc.evict_select(acc, int32(lens), budget, recent, keep.t, new.t), [keep, new], "choice")
    assert torch.equal(acc, kept)


@pytest.mark.parametrize("shape,dtype", [((416,), torch.uint8), ((576,), torch.bfloat16), ((), torch.float32), ((5,), torch.float32), ((128,), torch.uint8)])
def test_compaction(shape, dtype):
    g = gen(5)
    lens, budget = [700, 90, 0, 333], 128
    base, rows = ragged(lens)
    keep, new = torch.full((4, budget), -1, dtype=torch.int32), [min(n, budget) for n in lens]
    for b, n in enumerate(lens):
        keep[b, :new[b]] = torch.randperm(n, generator=g)[:new[b]].sort().values.to(torch.int32)
    keep, n_keep = keep.to(DEV), int32(new)
    first = torch.randint(0, 120, (rows, *shape), generator=g).to(dtype).to(DEV)
    dst, at_row = Guarded((4 * (budget + 1), *shape), dtype, fill=99), torch.arange(4, device=DEV) * (budget + 1)
    src = Guarded((rows, *shape), dtype)
    src.t.copy_(first)
    _twice(lambda: idxc.compact_rows(src.t, dst.t, keep, n_keep, base, at_row), [dst, src], "compaction elsewhere")
    for b in range(4):
        assert bool((dst.t[b * (budget + 1) + new[b]:(b + 1) * (budget + 1)] == 99).all()), "rows behind a sequence's last were written"
    assert torch.equal(src.t, first)
    _twice(lambda: idxc.compact_rows(src.t, src.t, keep, n_keep, base), [src], "compaction in place")
    for b, n in enumerate(lens):
        end = int(base[b]) + new[b]
        assert torch.equal(src.t[end:int(base[b]) + n + 2], first[end:int(base[b]) + n + 2]), "rows behind a sequence's last were written"
    assert torch.equal(src.t[:2], first[:2])
