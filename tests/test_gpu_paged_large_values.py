"""Attention over 8-bit rows of very large values: value scales up to 2^100, as the append writes them for bf16 elements up to 448 * 2^100."""
import pytest
import torch

from paper_2603_12201_b200 import binding as idxc
from tests.paged_util import DEV, Cache, bf16, check_call, gen, int32, tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,H_kv,n_step", [(8, 2, 1), (16, 1, 1), (32, 1, 1), (64, 1, 1), (16, 2, 40)])
@pytest.mark.parametrize("low,high", [(61, 100), (-60, 100), (100, 100)])
def test_value_scales(low, high, H, H_kv, n_step, d):
    """Few and many rows a key head, one CTA's share of the keys and joined ones."""
    lens, P, g = [500, 37, 3000], 16, gen(H + d + high - low)
    table, n_pages = tables(lens, P, g)
    cache = Cache(n_pages, P, H_kv, d, True, g)
    cache.v_scale.copy_(torch.exp2(torch.randint(low, high + 1, cache.v_scale.shape, generator=g).float()).to(DEV))
    q, table = bf16((len(lens), n_step, H, d), g).to(DEV), table.to(DEV)
    out, lse = idxc.paged_attention(cache.handle, q, table, int32(lens), 3000, 0.1)
    assert bool(torch.isfinite(out).all())
    check_call(cache, q, table, lens, 0.1, out, lse, only={(0, 0), (1, H_kv - 1), (2, 0)})


@pytest.mark.parametrize("n_step", [1, 40])
def test_what_the_append_writes(n_step):
    P, H, H_kv, d, n = 32, 8, 2, 128, 333
    g = gen(n_step)
    table, n_pages = tables([n], P, g)
    cache = Cache(n_pages, P, H_kv, d, True, g)
    pos = torch.arange(n)
    slots = table[0, pos // P].to(torch.int64) * P + pos % P
    v = (bf16((n, H_kv, d), g).clamp(-4, 4).float() * torch.exp2(torch.randint(0, 106, (n, H_kv, 1), generator=g).float())).to(torch.bfloat16)
    idxc.paged_append(cache.handle, bf16((n, H_kv, d), g).to(DEV), v.to(DEV), slots.to(DEV))
    assert float(cache.v_scale.max()) > 2.0 ** 90
    q, table = bf16((1, n_step, H, d), g).to(DEV), table.to(DEV)
    out, lse = idxc.paged_attention(cache.handle, q, table, int32([n]), n, 0.1)
    assert bool(torch.isfinite(out).all())
    check_call(cache, q, table, [n], 0.1, out, lse)
