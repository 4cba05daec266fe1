"""Attention over pages with many query rows a key head (chunks of prompts, large groups) against the oracle: blocks of rows that are full, ragged or
see nothing, requests shorter than their new tokens, units that runs cut, selections, and what lies in masked places."""
import numpy as np
import pytest
import torch

from oracle import paged as oracle
from paper_2603_12201_b200 import binding as idxc
from tests.paged_util import DEV, check_call, int32
from tests.test_gpu_paged_attention import run, setup
from tests.test_gpu_paged_guard_bands import test_attention as guarded_attention

pytestmark = pytest.mark.gpu

# lens, page size, H, H_kv, n_step: rows of a key head are n_step * H / H_kv
SHAPES = [([700, 64, 5, 0], 16, 8, 2, 64), ([400, 129, 128, 127], 32, 65, 1, 2), ([500, 33, 260], 64, 24, 2, 32), ([10, 300, 99, 100, 101], 16, 4, 1, 100),
          ([1500, 90], 48, 33, 3, 6), ([257], 128, 64, 1, 1), ([1000, 2, 640], 16, 33, 1, 1), ([300] * 9, 16, 12, 1, 32), ([383, 1025], 64, 2, 1, 192),
          ([700, 300], 1024, 16, 8, 64), ([520, 40], 16, 128, 1, 3), ([450, 17], 80, 22, 11, 40)]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,P,H,H_kv,n_step", SHAPES)
def test_against_the_oracle(eight, d, lens, P, H, H_kv, n_step):
    cache, q, table, n, _ = setup(lens, P, H, H_kv, d, eight, n_step)
    out, lse = run(cache, q, table, n, max(lens), d ** -0.5)
    check_call(cache, q, table, lens, d ** -0.5, out, lse)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("d,rows", [(64, (70, 1)), (128, (70, 1)), (64, (8, 32)), (128, (5, 33)), (128, (8, 50))])
def test_few_long_requests(eight, d, rows):
    """Units that many runs cut: pieces of both slots, with a ragged last block of rows."""
    group, n_step = rows
    lens = [9000, 31, 4100]
    cache, q, table, n, _ = setup(lens, 16, group * 2, 2, d, eight, n_step, gain=3.0)
    out, lse = run(cache, q, table, n, 9000, d ** -0.5)
    check_call(cache, q, table, lens, d ** -0.5, out, lse, only={(0, 1), (1, 0), (2, 1)})


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("group,n_step", [(80, 1), (12, 20)])
def test_selected_pages(eight, group, n_step):
    """Orders of their own, entries without a page, fewer pages than asked for."""
    lens, P, k = [900, 50, 333], 16, 37
    cache, q, table, n, g = setup(lens, P, group * 2, 2, 128, eight, n_step)
    sel = torch.full((3, 2, k), -1, dtype=torch.int32)
    for b, m in enumerate(lens):
        for h in range(2):
            pick = torch.randperm(oracle.ceil_div(m, P), generator=g)[:k].to(torch.int32)
            sel[b, h, :len(pick)] = pick
    sel[0, 0, 3], sel[0, 1, 0] = -1, 57                # (57: behind the request's last page)
    out, lse = run(cache, q, table, n, 900, 0.09, pages=sel.to(DEV))
    check_call(cache, q, table, lens, 0.09, out, lse, pages=sel)


@pytest.mark.parametrize("scale", [-0.3, 0.0, 4.0])
@pytest.mark.parametrize("eight", [False, True])
def test_scales(scale, eight):
    cache, q, table, n, _ = setup([90, 633], 16, 70, 1, 64, eight, 2)
    out, lse = run(cache, q, table, n, 633, scale)
    check_call(cache, q, table, [90, 633], scale, out, lse)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("H,n_step", [(160, 1), (16, 20)])
def test_rows_that_nobody_sees_and_rows_that_are_no_numbers(eight, H, n_step):
    lens, P = [137, 700, 16, 1], 64
    cache, q, table, n, _ = setup(lens, P, H, 2, 128, eight, n_step)
    want = run(cache, q, table, n, 700, 0.09)
    seen = torch.zeros(cache.shape[:2], dtype=torch.bool)
    for b, m in enumerate(lens):
        pos = torch.arange(m)
        seen[table[b].cpu()[pos // P].long(), pos % P] = True
    dark = (~seen).to(DEV)
    for x in (cache.k, cache.v):
        (x.view(torch.uint8) if eight else x)[dark] = 0x7F if eight else float("nan")
    if eight:
        for s in (cache.k_scale, cache.v_scale):
            s.masked_fill_(dark[:, None, :].expand_as(s), float("nan"))
    got = run(cache, q, table, n, 700, 0.09)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    q2 = q.clone()
    q2[1, n_step - 1, 5, 3] = float("nan")
    out, lse = run(cache, q2, table, n, 700, 0.09)
    assert torch.isnan(out[1, n_step - 1, 5]).all() and torch.isnan(lse[1, n_step - 1, 5])
    keep = torch.ones(q.shape[:3], dtype=torch.bool, device=DEV)
    keep[1, n_step - 1, 5] = False
    assert torch.equal(out[keep], want[0][keep]) and torch.equal(lse[keep], want[1][keep])


def test_references_that_rise_all_the_way():
    """Scores that grow by more than 2^8 from tile to tile: every row's reference moves at every tile, and its output with it."""
    lens, P, H = [1500], 16, 100
    cache, q, table, n, _ = setup(lens, P, H, 1, 64, False)
    q[...] = 0
    q[:, :, :, 0] = torch.linspace(0.25, 2.0, H, device=DEV).to(torch.bfloat16)
    pos = torch.arange(1500)
    cache.k[table[0].cpu()[pos // P].long(), pos % P, 0, 0] = (pos.float() / 4).to(torch.bfloat16).to(DEV)
    out, lse = run(cache, q, table, n, 1500, 1.0)
    check_call(cache, q, table, lens, 1.0, out, lse)


@pytest.mark.parametrize("eight", [False, True])
def test_chunks_are_the_prompt(eight):
    """A prompt in chunks of other sizes, each over the cache so far, gives each token what it gets from the prompt at once, up to the order of sums."""
    cache, q, table, n, _ = setup([640], 32, 16, 2, 128, eight, 640)
    whole, whole_lse = run(cache, q, table, n, 640, 0.09)
    k, v = (torch.from_numpy(x[table[0].cpu().numpy()[np.arange(640) // 32], np.arange(640) % 32]) for x in cache.values())      # [640, 2, 128]
    reach = 0.09 * float(torch.einsum("thd,shd->hts", q[0].double().cpu().abs(), k.abs().repeat_interleave(8, dim=1)).max())
    e = 2.0 ** -16 * reach + 640 * 2.0 ** -22                      # of a score (q's 8-bit form too), and of the sums
    at = 0
    for size in (1, 3, 17, 299, 320):
        out, lse = run(cache, q[:, at:at + size].contiguous(), table, int32([at + size]), at + size, 0.09)
        # probabilities rounded to 2^-8 and the output's own half step, on either side
        assert (out.float() - whole[:, at:at + size].float()).abs().max() <= (2.0 ** -6 * (1 + 2.0 ** -6) + 4 * e) * float(v.abs().max())
        assert (lse - whole_lse[:, at:at + size]).abs().max() <= 2 * e + 2.0 ** -19 * float(whole_lse.abs().max())
        at += size


def test_results_repeat_and_do_not_depend_on_the_workspaces_contents():
    lens = [5000, 17, 900, 64]
    cache, q, table, n, _ = setup(lens, 16, 16, 2, 128, False, 24)
    nb = idxc.paged_attention_workspace_bytes(24, 16, 2, 128)
    first = None
    for fill in (0, 255, 127):
        ws = torch.full((nb,), fill, dtype=torch.uint8, device=DEV)
        out, lse = run(cache, q, table, n, 5000, 0.1, workspace=ws)
        if first is None:
            first = out.clone(), lse.clone()
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    with pytest.raises(idxc.IdxcError):
        idxc.paged_attention(cache.handle, q, table, n, 5000, 0.1, workspace=torch.empty(nb - 1, dtype=torch.uint8, device=DEV))


def test_captured_and_replayed_over_other_lengths():
    cache, q, table, n, _ = setup([900, 400], 16, 16, 2, 64, False, 16)
    out = torch.empty_like(q)
    ws = torch.empty(idxc.paged_attention_workspace_bytes(16, 16, 2, 64), dtype=torch.uint8, device=DEV)
    idxc.paged_attention(cache.handle, q, table, n, 900, 0.1, out=out, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _, lse = idxc.paged_attention(cache.handle, q, table, n, 900, 0.1, out=out, workspace=ws)
    for lens in ([900, 400], [5, 0], [16, 399]):
        n.copy_(int32(lens))
        g.replay()
        torch.cuda.synchronize()
        idxc.poll_device_status()
        check_call(cache, q, table, lens, 0.1, out, lse)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("lens,P,H,H_kv,d,n_step,k", [([1], 16, 33, 1, 64, 1, 0), ([700, 0, 65, 3], 16, 10, 2, 128, 40, 0), ([3000], 48, 64, 1, 64, 1, 0),
                                                      ([257, 31], 64, 26, 2, 128, 11, 0), ([63] * 40, 16, 16, 8, 64, 9, 0), ([2000, 90, 0], 16, 16, 2, 128, 5, 7)])
def test_nothing_is_written_beside_the_outputs(lens, P, H, H_kv, d, n_step, k, eight):
    guarded_attention(lens, P, H, H_kv, d, n_step, k, eight)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("n_step", [6, 40])
def test_selections_that_name_nothing_and_no_lse(eight, n_step):
    lens, P = [500, 0, 77], 32
    cache, q, table, n, _ = setup(lens, P, 20, 2, 64, eight, n_step)
    sel = torch.full((3, 2, 5), -1, dtype=torch.int32)
    sel[2, 1] = torch.tensor([2, 1, 0, 9, 2 ** 31 - 1], dtype=torch.int32)
    out, lse = run(cache, q, table, n, 500, 0.1, pages=sel.to(DEV))
    check_call(cache, q, table, lens, 0.1, out, lse, pages=sel)
    assert torch.isneginf(lse[:2]).all() and not out[:2].any()
    again, none = run(cache, q, table, n, 500, 0.1, pages=sel.to(DEV), want_lse=False)
    assert none is None and torch.equal(again, out)


@pytest.mark.parametrize("eight", [False, True])
def test_calls_on_two_streams_at_once(eight):
    jobs = []
    for seed, (lens, n_step) in enumerate([([2000, 90], 33), ([1500], 5)]):
        cache, q, table, n, _ = setup(lens, 16, 16, 2, 128, eight, n_step, seed=seed)
        jobs.append((cache, q, table, n, max(lens), run(cache, q, table, n, max(lens), 0.09), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for cache, q, table, n, top, want, stream in jobs:
            got.append((idxc.paged_attention(cache.handle, q, table, n, top, 0.09, stream=stream), want))
    torch.cuda.synchronize()
    idxc.poll_device_status()
    for (out, lse), want in got:
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
