"""Rows written to a paged cache, its pages' bounds, and rows read back, against the oracle: every number has to be equal."""
import numpy as np
import pytest
import torch

from oracle import paged as oracle
from paper_2603_12201_b200 import binding as idxc
from tests.paged_util import DEV, Cache, bf16, gen, tables
from tests.util import codes

pytestmark = pytest.mark.gpu


def slots_of(table, lens, new, P):
    out = []
    for b, (n, m) in enumerate(zip(lens, new)):
        pos = torch.arange(n, n + m)
        out.append(table[b, pos // P].to(torch.int64) * P + pos % P)
    return torch.cat(out)


def expect(cache, k, v, slots):
    """(codes or bits of k and v, scales, bounds) that the cache has to hold afterwards."""
    n_pages, P, H_kv, d = cache.shape
    eight = cache.scale is not None
    store = [codes(x).copy() for x in (cache.k, cache.v)]
    scale = [None if s is None else s.cpu().numpy().copy() for s in (cache.k_scale, cache.v_scale)]
    newest = {}
    for t, slot in enumerate(slots.tolist()):
        if not 0 <= slot < n_pages * P:
            continue
        page, row = divmod(slot, P)
        newest[page] = max(newest.get(page, -1), row)
        for which, x in enumerate((k, v)):
            for h in range(H_kv):
                bits = codes(x[t, h])
                if eight:
                    store[which][page, row, h], scale[which][page, h, row] = oracle.quantize_row(bits)
                else:
                    store[which][page, row, h] = bits
    edge = None
    if cache.bounds is not None:
        edge = oracle.bf16_rows(codes(cache.bounds)).copy()
        for page, row in newest.items():
            for h in range(H_kv):
                if eight:
                    rows = (oracle.e4m3_values(store[0][page, :row + 1, h]).astype(np.float32) * scale[0][page, h, :row + 1, None]).astype(np.float64)
                    rows = oracle.to_bf16(rows)
                else:
                    rows = oracle.bf16_rows(store[0][page, :row + 1, h])
                edge[page, h] = oracle.bounds(rows)
    return store, scale, edge


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("lens,new,P,H_kv,d,layout", [
    ([0], [1], 16, 1, 64, "tokens"), ([15], [3], 16, 1, 128, "heads"), ([5, 40, 0], [1, 1, 1], 16, 8, 128, "pair"), ([17, 3, 100], [60, 0, 29], 48, 3, 128, "tokens"),
    ([7], [300], 128, 5, 64, "heads"), ([0, 31], [64, 33], 32, 2, 64, "tokens"), ([1000, 5], [1, 2], 1024, 9, 128, "tokens"), ([33], [200], 16, 20, 128, "pair")])
def test_append_and_gather(eight, lens, new, P, H_kv, d, layout):
    g = gen(sum(lens) + sum(new) + d)
    table, n_pages = tables([n + m for n, m in zip(lens, new)], P, g)
    cache = Cache(n_pages, P, H_kv, d, eight, g, layout, bounds=True)
    slots = slots_of(table, lens, new, P)
    T = slots.shape[0]
    row = bf16((T, 3, H_kv, d), g, 2.0)
    row[T // 2, 1] = 0                                               # a row of zeros
    k, v = row.to(DEV)[:, 1], row.to(DEV)[:, 2]                      # as a projection leaves them: side by side
    store, scale, edge = expect(cache, row[:, 1], row[:, 2], slots)
    idxc.paged_append(cache.handle, k, v, slots.to(DEV))
    for which, (x, s) in enumerate(((cache.k, cache.k_scale), (cache.v, cache.v_scale))):
        assert np.array_equal(codes(x), store[which])
        if eight:
            assert np.array_equal(s.cpu().numpy(), scale[which])
    assert np.array_equal(oracle.bf16_rows(codes(cache.bounds)), edge)

    where = torch.cat([slots, torch.tensor([-1, n_pages * P, 0])]).to(DEV)
    out = [torch.full((T + 3, H_kv, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    idxc.paged_gather(cache.handle, where, *out)
    for x, values, s in zip(out, cache.values(), (cache.k_scale, cache.v_scale)):
        flat = values.reshape(n_pages * P, H_kv, d)
        want = flat[np.r_[slots.numpy(), [0, 0, 0]]]
        if eight:                                                     # code * scale is rounded to fp32, then to bf16
            want = oracle.to_bf16(want.astype(np.float32).astype(np.float64))
        want[T:T + 2] = 0
        assert np.array_equal(oracle.bf16_rows(codes(x)), want)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("P,H_kv,d", [(64, 2, 64), (16, 1, 128), (1024, 1, 64), (48, 3, 64)])
def test_long_prompts(eight, P, H_kv, d):
    """More tokens than the threshold of one CTA a token; runs that begin and end inside the CTAs' chunks."""
    g = gen(11)
    lens, new = [9, 0, 70], [3001, 17, 1500]
    table, n_pages = tables([n + m for n, m in zip(lens, new)], P, g)
    cache = Cache(n_pages, P, H_kv, d, eight, g, bounds=True)
    slots = slots_of(table, lens, new, P)
    k, v = bf16((slots.shape[0], H_kv, d), g), bf16((slots.shape[0], H_kv, d), g)
    store, scale, edge = expect(cache, k, v, slots)
    idxc.paged_append(cache.handle, k.to(DEV), v.to(DEV), slots.to(DEV))
    assert np.array_equal(codes(cache.k), store[0]) and np.array_equal(codes(cache.v), store[1])
    assert np.array_equal(oracle.bf16_rows(codes(cache.bounds)), edge)


def test_slots_that_are_none_and_a_cache_without_bounds():
    g = gen(2)
    cache = Cache(6, 16, 2, 128, False, g)
    slots = torch.tensor([-1, 3, 4, -5, 6 * 16, 95, 2 ** 40, 16], dtype=torch.int64)
    k, v = bf16((8, 2, 128), g), bf16((8, 2, 128), g)
    store, _, _ = expect(cache, k, v, slots)
    idxc.paged_append(cache.handle, k.to(DEV), v.to(DEV), slots.to(DEV))
    assert np.array_equal(codes(cache.k), store[0]) and np.array_equal(codes(cache.v), store[1])


def test_values_at_the_ends_of_the_types():
    g = gen(4)
    cache = Cache(2, 16, 1, 64, True, g, bounds=True)
    x = bf16((5, 1, 64), g)
    x[0] = 3e38
    x[1, 0, :32], x[1, 0, 32:] = 1e-30, -1e-38
    x[2, 0, ::2], x[2, 0, 1::2] = -448.0, 448.0
    x[3, 0, 0] = 1e6
    slots = torch.arange(5) + 7
    store, scale, edge = expect(cache, x, -x, slots)
    idxc.paged_append(cache.handle, x.to(DEV), (-x).to(DEV), slots.to(DEV))
    assert np.array_equal(codes(cache.k), store[0]) and np.array_equal(codes(cache.v), store[1])
    assert np.array_equal(cache.k_scale.cpu().numpy(), scale[0])


def test_handle_refusals():
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)
    e = lambda *s: torch.zeros(s, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
    f = lambda *s: torch.zeros(s, device=DEV)
    good = z(4, 16, 2, 64)
    idxc.PagedCache(good, z(4, 16, 2, 64))
    for args, kw in (((good, z(4, 16, 2, 128)), {}), ((good, z(4, 2, 16, 64).permute(0, 2, 1, 3)), {}), ((good[:, :, :, ::2], good[:, :, :, ::2]), {}),
                     ((good, good, f(4, 2, 16)), {}), ((e(4, 16, 2, 64), e(4, 16, 2, 64)), {}), ((e(4, 16, 2, 64), e(4, 16, 2, 64), f(4, 16, 2), f(4, 16, 2)), {}),
                     ((e(4, 16, 2, 64), e(4, 16, 2, 64), f(4, 2, 32)[:, :, ::2], f(4, 2, 16)), {}),
                     ((good, good), dict(bounds=z(4, 2, 64))), ((good, good), dict(bounds=z(4, 2, 2, 64).cpu()))):
        with pytest.raises(ValueError):
            idxc.PagedCache(*args, **kw)
    with pytest.raises(TypeError):
        idxc.PagedCache(good.float(), good.float())
    odd = idxc.PagedCache(z(4, 16, 2, 72)[..., :64], z(4, 16, 2, 72)[..., :64])         # strides of 144 bytes: multiples of 16
    idxc.paged_append(odd, z(1, 2, 64), z(1, 2, 64), torch.zeros(1, dtype=torch.int64, device=DEV))
    bad = idxc.PagedCache(z(4, 16, 2, 68)[..., :64], z(4, 16, 2, 68)[..., :64])         # 136: not
    with pytest.raises(idxc.IdxcError):
        idxc.paged_append(bad, z(1, 2, 64), z(1, 2, 64), torch.zeros(1, dtype=torch.int64, device=DEV))
    cache = idxc.PagedCache(good, good.clone())
    s = torch.zeros(2, dtype=torch.int64, device=DEV)
    for k, v in ((z(2, 2, 64), z(1, 2, 64)), (z(2, 3, 64), z(2, 2, 64)), (z(2, 64, 2).transpose(1, 2), z(2, 2, 64))):
        with pytest.raises(ValueError):
            idxc.paged_append(cache, k, v, s)
    with pytest.raises(TypeError):
        idxc.paged_append(cache, z(2, 2, 64).float(), z(2, 2, 64), s)
