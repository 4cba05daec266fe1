"""Scales and bounds that the 8-bit append writes, for long inputs (whose CTAs look at several tokens) and at the ends of the types; long inputs read back."""
import numpy as np
import pytest
import torch

from oracle import paged as oracle
from paper_2603_12201_b200 import binding as idxc
from tests.paged_util import DEV, Cache, bf16, gen, tables
from tests.test_gpu_paged_cache import expect, slots_of
from tests.util import codes

pytestmark = pytest.mark.gpu


def written_as_expected(cache, store, scale, edge):
    for which, (x, s) in enumerate(((cache.k, cache.k_scale), (cache.v, cache.v_scale))):
        assert np.array_equal(codes(x), store[which])
        if s is not None:
            assert np.array_equal(s.cpu().numpy(), scale[which])
    assert np.array_equal(oracle.bf16_rows(codes(cache.bounds)), edge)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("P,H_kv,d,layout", [(64, 2, 64, "tokens"), (16, 1, 128, "heads"), (1024, 1, 64, "pair"), (48, 3, 64, "tokens")])
def test_long_inputs(eight, P, H_kv, d, layout):
    g = gen(P + d)
    lens, new = [9, 0, 70], [3001, 17, 1500]
    table, n_pages = tables([n + m for n, m in zip(lens, new)], P, g)
    cache = Cache(n_pages, P, H_kv, d, eight, g, layout, bounds=True)
    slots = slots_of(table, lens, new, P)
    T = slots.shape[0]
    assert T > 4096
    k, v = bf16((T, H_kv, d), g), bf16((T, H_kv, d), g, 3.0)
    want = expect(cache, k, v, slots)
    idxc.paged_append(cache.handle, k.to(DEV), v.to(DEV), slots.to(DEV))
    written_as_expected(cache, *want)
    out = [torch.full((T, H_kv, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    idxc.paged_gather(cache.handle, slots.to(DEV), *out)
    for x, values in zip(out, cache.values()):
        rows = values.reshape(n_pages * P, H_kv, d)[slots.numpy()]
        if eight:                                                     # code * scale is rounded to fp32, then to bf16
            rows = oracle.to_bf16(rows.astype(np.float32).astype(np.float64))
        assert np.array_equal(oracle.bf16_rows(codes(x)), rows)


@pytest.mark.parametrize("n", [5, 4200])
def test_ends_of_the_types(n):
    """The same five rows once, and again and again in an input of the other path."""
    P, g = 16, gen(4)
    cache = Cache(n // P + 2, P, 1, 64, True, g, bounds=True)
    x = bf16((5, 1, 64), g)
    x[0] = 3e38
    x[1, 0, :32], x[1, 0, 32:] = 1e-30, -1e-38
    x[2, 0, ::2], x[2, 0, 1::2] = -448.0, 448.0
    x[3, 0, 0] = 1e6
    x = x.repeat(n // 5, 1, 1)
    slots = torch.arange(n) + 7
    want = expect(cache, x, -x, slots)
    idxc.paged_append(cache.handle, x.to(DEV), (-x).to(DEV), slots.to(DEV))
    written_as_expected(cache, *want)
