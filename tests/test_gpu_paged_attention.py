"""Attention over pages against the oracle: types, head layouts, lengths, page sizes, selections, masks and what lies in masked places."""
import numpy as np
import pytest
import torch

from oracle import paged as oracle
from paper_2603_12201_b200 import binding as idxc
from tests.paged_util import DEV, Cache, bf16, check_call, gen, int32, tables

pytestmark = pytest.mark.gpu


def setup(lens, P, H, H_kv, d, eight, n_step=1, layout="tokens", seed=0, gain=1.0):
    g = gen(seed + sum(lens) + H * d + n_step)
    table, n_pages = tables(lens, P, g)
    cache = Cache(n_pages, P, H_kv, d, eight, g, layout)
    q = bf16((len(lens), n_step, H, d), g, gain).to(DEV)
    return cache, q, table.to(DEV), int32(lens), g


def run(cache, q, table, lens, max_len, scale, **kw):
    out, lse = idxc.paged_attention(cache.handle, q, table, lens, max_len, scale, **kw)
    idxc.poll_device_status()
    return out, lse


SHAPES = [
    ([1], 16, 1, 1, 1, "tokens"), ([64], 64, 8, 8, 1, "heads"), ([777], 16, 32, 8, 1, "tokens"), ([5, 0, 130, 64, 63, 65], 16, 6, 2, 1, "pair"),
    ([300, 1, 2], 48, 16, 1, 1, "tokens"), ([500, 3, 90], 32, 34, 2, 1, "heads"), ([200, 700], 64, 35, 1, 1, "tokens"), ([900], 128, 128, 2, 1, "pair"),
    ([150, 333], 16, 128, 1, 1, "tokens"), ([400, 2, 1], 16, 8, 2, 4, "tokens"), ([129, 40], 32, 40, 4, 3, "pair"), ([70, 1000], 16, 100, 1, 3, "tokens"),
    ([2500], 96, 7, 7, 2, "tokens"), ([10, 260], 16, 4, 2, 33, "heads"), ([1100], 64, 2, 1, 1024, "tokens"), ([2100, 40], 1024, 8, 2, 1, "pair"),
    ([70, 200], 16, 22, 11, 1, "tokens"), ([70, 500], 32, 24, 12, 1, "heads"), ([333], 16, 48, 16, 2, "tokens"), ([600, 1], 80, 260, 4, 1, "tokens")]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,P,H,H_kv,n_step,layout", SHAPES)
def test_against_the_oracle(eight, d, lens, P, H, H_kv, n_step, layout):
    cache, q, table, n, _ = setup(lens, P, H, H_kv, d, eight, n_step, layout)
    scale = d ** -0.5
    out, lse = run(cache, q, table, n, max(lens) + 5 if max(lens) + 5 <= table.shape[1] * P else max(lens), scale)
    check_call(cache, q, table, lens, scale, out, lse)


@pytest.mark.parametrize("eight,d", [(False, 64), (False, 128), (True, 64), (True, 128)])
@pytest.mark.parametrize("lens,P,H,H_kv,n_step,layout", SHAPES)
def test_short_requests_under_a_high_bound(eight, d, lens, P, H, H_kv, n_step, layout):
    """Where max_len allows long requests the work is cut into runs over all units, and segments go through the merge, however short the requests are."""
    cache, q, table, n, _ = setup(lens, P, H, H_kv, d, eight, n_step, layout)
    wide = torch.full((len(lens), 1 + 100000 // P), -1, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    scale = d ** -0.5
    out, lse = run(cache, q, wide, n, 100000, scale)
    check_call(cache, q, table, lens, scale, out, lse)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("B,H_kv,top", [(1, 1, 64), (1, 1, 5000), (3, 8, 1000), (9, 4, 600), (18, 8, 700), (37, 8, 300), (140, 2, 500), (20, 2, 129)])
def test_units_of_clusters(eight, B, H_kv, top):
    """Every size of cluster, units whose CTAs have no tile, and requests without keys among them."""
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, top + 1, B)]
    lens[0] = top
    cache, q, table, n, _ = setup(lens, 16, 8 * H_kv, H_kv, 128, eight)
    out, lse = run(cache, q, table, n, top, 0.09)
    check_call(cache, q, table, lens, 0.09, out, lse)


@pytest.mark.parametrize("eight", [False, True])
def test_many_requests_and_runs(eight):
    """Whole segments, segments cut by runs, and empty requests in one call."""
    rng = np.random.default_rng(1)
    lens = [int(x) for x in rng.integers(0, 700, 150)]
    lens[3] = lens[77] = 0
    lens[10] = 6000
    cache, q, table, n, _ = setup(lens, 16, 8, 2, 64, eight)
    out, lse = run(cache, q, table, n, 6000, 0.1)
    check_call(cache, q, table, lens, 0.1, out, lse)


def test_one_long_request_over_all_ctas():
    cache, q, table, n, _ = setup([30011], 64, 8, 1, 128, False)
    out, lse = run(cache, q, table, n, 30011, 0.088)
    check_call(cache, q, table, [30011], 0.088, out, lse)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,n_step", [(8, 1), (16, 1), (8, 4), (60, 1), (32, 4), (100, 2)])
def test_rings_that_go_round(eight, d, group, n_step):
    """Runs of many tiles, so that every stage of the ring is used several times, for every number of rows a CTA takes."""
    lens, H_kv = [21011, 9000], 8
    cache, q, table, n, _ = setup(lens, 64, group * H_kv, H_kv, d, eight, n_step)
    out, lse = run(cache, q, table, n, 21011, d ** -0.5)
    check_call(cache, q, table, lens, d ** -0.5, out, lse, only=[(0, 0), (0, 5), (1, 7)])


def test_more_requests_than_threads():
    rng = np.random.default_rng(2)
    lens = [int(x) for x in rng.integers(0, 40, 1000)]
    lens[500:800] = [0] * 300
    cache, q, table, n, _ = setup(lens, 16, 2, 1, 64, False)
    out, lse = run(cache, q, table, n, 40, 0.2)
    check_call(cache, q, table, lens, 0.2, out, lse)


def test_the_most_requests():
    B, P, g = 65535, 16, gen(6)
    lens = torch.randint(0, 2, (B,), generator=g)
    lens[::4099] = 16
    n_pages = 300
    cache = Cache(n_pages, P, 1, 64, False, g)
    table = torch.randint(0, n_pages, (B, 1), generator=g).to(torch.int32).to(DEV)
    q = bf16((B, 1, 1, 64), g).to(DEV)
    out, lse = run(cache, q, table, lens.to(torch.int32).to(DEV), 16, 0.2)
    k, v = cache.k[:, 0, 0].double(), cache.v[:, 0, 0]
    one = (lens == 1).to(DEV)
    page = table[one, 0].long()
    assert torch.equal(out[one, 0, 0], v[page])                       # a single key: its value
    x = 0.2 * (q[one, 0, 0].double() * k[page]).sum(dim=1)
    assert torch.all((lse[one, 0, 0].double() - x).abs() <= 2.0 ** -16 * 0.2 * (q[one, 0, 0].double() * k[page]).abs().sum(dim=1) + 2.0 ** -19 * (1 + x.abs()))
    none = (lens == 0).to(DEV)
    assert not out[none].any() and torch.isneginf(lse[none]).all()
    some = torch.arange(0, B, 4099)
    check_call(cache, q[some.to(DEV)], table[some.to(DEV)], [16] * some.numel(), 0.2, out[some.to(DEV)], lse[some.to(DEV)])


def test_all_requests_empty():
    cache, q, table, n, _ = setup([0, 0, 0], 16, 4, 2, 64, False)
    out, lse = run(cache, q, table, n, 20, 0.2)
    assert not out.any() and torch.isneginf(lse).all()
    out, lse = run(cache, q, table, int32([-4, 0, -1]), 20, 0.2)
    assert not out.any() and torch.isneginf(lse).all()
    out, lse = run(cache, q, table, int32([5, 6, 7]), 0, 0.2)                  # max_len 0 cuts all
    assert not out.any() and torch.isneginf(lse).all()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("P,k", [(16, 3), (16, 40), (48, 5), (64, 4), (128, 2), (32, 1)])
def test_selected_pages(eight, P, k):
    lens = [1, P, 5 * P + 1, 17 * P - 3, 0, 9 * P]
    H, H_kv, d = 12, 3, 128
    cache, q, table, n, g = setup(lens, P, H, H_kv, d, eight, seed=k)
    sel = torch.full((len(lens), H_kv, k), -1, dtype=torch.int32)
    for b, m in enumerate(lens):
        pages = oracle.ceil_div(m, P)
        for h in range(H_kv):
            pick = torch.randperm(pages, generator=g)[:k].sort().values
            sel[b, h, :pick.numel()] = pick.to(torch.int32)
    out, lse = run(cache, q, table, n, max(lens), 0.09, pages=sel.to(DEV))
    check_call(cache, q, table, lens, 0.09, out, lse, pages=sel)
    flat, flat_lse = run(cache, q, table, n, max(lens), 0.09, pages=sel.to(DEV).reshape(-1, k))
    assert torch.equal(out, flat) and torch.equal(lse, flat_lse)


def test_selections_with_holes_repeats_and_foreign_entries():
    P, lens = 16, [100, 200, 90]
    cache, q, table, n, _ = setup(lens, P, 4, 2, 64, False, n_step=3)
    sel = torch.tensor([[[3, -1, 0, 3, 6, 5, 2], [6, 6, 6, 6, 6, 6, 6]], [[12, 0, 13, 400, 2 ** 31 - 1, -7, 5], [-1] * 7], [[5, 4, 3, 2, 1, 0, 0], [1, 2, 3, 4, 99, 0, 5]]], dtype=torch.int32)
    out, lse = run(cache, q, table, n, 200, 0.1, pages=sel.to(DEV))
    check_call(cache, q, table, lens, 0.1, out, lse, pages=sel)


def test_all_pages_selected_is_the_dense_result():
    lens, P = [333, 40, 1000], 32
    cache, q, table, n, _ = setup(lens, P, 8, 2, 128, False)
    sel = torch.arange(40, dtype=torch.int32, device=DEV).expand(3, 2, 40).contiguous()
    a, b = run(cache, q, table, n, 1000, 0.1), run(cache, q, table, n, 1000, 0.1, pages=sel)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("eight", [False, True])
def test_rows_that_nobody_sees_may_hold_anything(eight):
    lens, P = [37, 100, 16, 1], 64
    cache, q, table, n, _ = setup(lens, P, 8, 2, 64, eight, n_step=2)
    want = run(cache, q, table, n, 100, 0.125)
    seen = torch.zeros(cache.shape[:2], dtype=torch.bool)
    for b, m in enumerate(lens):
        pos = torch.arange(m)
        seen[table[b].cpu()[pos // P].long(), pos % P] = True
    dark = (~seen).to(DEV)
    nan = 0x7F if eight else float("nan")
    for x in (cache.k, cache.v):
        (x.view(torch.uint8) if eight else x)[dark] = nan
    if eight:
        for s in (cache.k_scale, cache.v_scale):
            s.masked_fill_(dark[:, None, :].expand_as(s), float("nan"))
    got = run(cache, q, table, n, 100, 0.125)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for x in (cache.k, cache.v):
        if not eight:
            x[dark] = float("inf")
    got = run(cache, q, table, n, 100, 0.125)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_pages_that_are_none_of_the_caches_take_no_part():
    lens, P = [200, 150, 60], 16
    cache, q, table, n, _ = setup(lens, P, 4, 2, 64, False)
    table[0, 3], table[0, 7], table[1, 0], table[2, :] = -1, cache.shape[0], 2 ** 31 - 1, -9
    out, lse = run(cache, q, table, n, 200, 0.2)
    assert torch.isneginf(lse[2]).all() and not out[2].any()
    check_call(cache, q, table, lens, 0.2, out, lse)


def test_lengths_above_the_bound_are_cut_to_it():
    cache, q, table, n, _ = setup([300, 500], 16, 4, 2, 64, False)
    out, lse = run(cache, q, table, n, 320, 0.2)
    check_call(cache, q, table, [300, 320], 0.2, out, lse)


@pytest.mark.parametrize("scale", [-0.3, 0.0, 4.0])
def test_scales(scale):
    cache, q, table, n, _ = setup([90, 333], 16, 8, 2, 64, False)
    out, lse = run(cache, q, table, n, 333, scale)
    check_call(cache, q, table, [90, 333], scale, out, lse)


def test_a_visible_score_that_is_no_number_spoils_its_rows_alone():
    cache, q, table, n, _ = setup([100, 3000], 16, 8, 2, 64, False)
    want = run(cache, q, table, n, 3000, 0.1)
    q2 = q.clone()
    q2[1, 0, 5, 3] = float("nan")
    out, lse = run(cache, q2, table, n, 3000, 0.1)
    assert torch.isnan(out[1, 0, 5]).all() and torch.isnan(lse[1, 0, 5])
    keep = torch.ones((2, 1, 8), dtype=torch.bool, device=DEV)
    keep[1, 0, 5] = False
    assert torch.equal(out[keep], want[0][keep]) and torch.equal(lse[keep], want[1][keep])


def test_scores_of_minus_infinity():
    """All visible scores -inf: as one that sees nothing. Some: they have weight 0."""
    cache, q, table, n, _ = setup([40, 40], 16, 1, 1, 64, False)
    q[:, 0, 0] = 0
    q[:, 0, 0, 0] = 1.0
    pos = torch.arange(40)
    page = table[0].cpu()[pos // 16].long()
    cache.k[page, pos % 16, 0, 0] = float("-inf")
    page = table[1].cpu()[pos // 16].long()
    cache.k[page[::2], (pos % 16)[::2], 0, 0] = float("-inf")
    cache.k[:, :, :, 1:] = cache.k[:, :, :, 1:].clamp(-3, 3)
    out, lse = run(cache, q, table, n, 40, 0.1)
    assert not out[0].any() and torch.isneginf(lse[0]).all()
    assert torch.isfinite(out[1]).all() and torch.isfinite(lse[1]).all()
    v = cache.v[page[1::2], (pos % 16)[1::2], 0].double()
    x = 0.1 * cache.k[page[1::2], (pos % 16)[1::2], 0, 0].double()
    want = torch.softmax(x, 0) @ v
    assert torch.all((out[1, 0, 0].double() - want).abs() <= 2.0 ** -7 * (torch.softmax(x, 0) @ v.abs()) + 2.0 ** -8 * want.abs())


def test_8_bit_scales_far_apart():
    """Value scales over 2^-40 .. 2^40 in one request, and one tiny q beside a large one: every product of probability and scale keeps its place."""
    lens, P = [500], 16
    cache, q, table, n, g = setup(lens, P, 8, 2, 64, True)
    e = torch.randint(-40, 41, cache.v_scale.shape, generator=g).to(DEV)
    cache.v_scale.copy_(torch.exp2(e.float()))
    cache.k_scale.copy_(torch.exp2(torch.randint(-12, -4, cache.k_scale.shape, generator=g).float()).to(DEV))
    q[0, 0, 3] *= 2.0 ** -60
    q[0, 0, 4] *= 2.0 ** 20
    out, lse = run(cache, q, table, n, 500, 0.1)
    check_call(cache, q, table, lens, 0.1, out, lse)


@pytest.mark.parametrize("eight", [False, True])
def test_queries_inside_a_projections_output(eight):
    lens = [200, 31, 90]
    cache, _, table, n, g = setup(lens, 16, 8, 2, 128, eight, n_step=2)
    row = bf16((3, 2, 12, 128), g).to(DEV)
    q = row[:, :, :8]
    out, lse = run(cache, q, table, n, 200, 0.1)
    again = run(cache, q.contiguous(), table, n, 200, 0.1)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    check_call(cache, q.contiguous(), table, lens, 0.1, out, lse)


def test_results_repeat_and_do_not_depend_on_the_workspaces_contents():
    lens = [5000, 17, 900, 64]
    cache, q, table, n, _ = setup(lens, 16, 16, 2, 128, False)
    nb = idxc.paged_attention_workspace_bytes(1, 16, 2, 128)
    first = None
    for fill in (0, 255, 127):
        ws = torch.full((nb,), fill, dtype=torch.uint8, device=DEV)
        out, lse = run(cache, q, table, n, 5000, 0.1, workspace=ws)
        if first is None:
            first = out.clone(), lse.clone()
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    with pytest.raises(idxc.IdxcError):
        idxc.paged_attention(cache.handle, q, table, n, 5000, 0.1, workspace=torch.empty(nb - 1, dtype=torch.uint8, device=DEV))


def test_offsets_beyond_32_bits():
    """A cache of more than 2^31 elements and 4 GB: its last pages are read where they are."""
    P, H_kv, d = 64, 8, 128
    n_pages = 2 ** 32 // (P * H_kv * d * 2) * 5 // 4
    k = torch.zeros((n_pages, P, H_kv, d), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros((n_pages, P, H_kv, d), dtype=torch.bfloat16, device=DEV)
    g = gen(1)
    last = bf16((2, 3, P, H_kv, d), g).to(DEV)
    k[-3:], v[-3:] = last[0], last[1]
    k[:3], v[:3] = 5.0, 7.0                                     # where a wrapped offset would land
    cache = idxc.PagedCache(k, v)
    small = idxc.PagedCache(last[0].contiguous(), last[1].contiguous())
    q, n = bf16((1, 1, 16, d), g).to(DEV), int32([3 * P - 5])
    far = idxc.paged_attention(cache, q, int32([[n_pages - 1, n_pages - 3, n_pages - 2]]), n, 3 * P, 0.1)
    near = idxc.paged_attention(small, q, int32([[2, 0, 1]]), n, 3 * P, 0.1)
    assert torch.equal(far[0], near[0]) and torch.equal(far[1], near[1])
    slots = torch.tensor([(n_pages - 1) * P + 7, n_pages * P - 1], device=DEV)
    new = bf16((2, H_kv, d), g).to(DEV)
    idxc.paged_append(cache, new, new, slots)
    out = torch.empty((2, H_kv, d), dtype=torch.bfloat16, device=DEV)
    idxc.paged_gather(cache, slots, out, torch.empty_like(out))
    assert torch.equal(out, new) and torch.equal(k[-1, 7], new[0]) and torch.equal(v[-1, P - 1], new[1])
    idxc.poll_device_status()
