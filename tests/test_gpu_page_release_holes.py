"""Giving back requests some of whose table entries are no page: these stay off the stack."""
import numpy as np
import pytest
import torch

from oracle import paged as oracle
from paper_2603_12201_b200 import binding as idxc
from tests.paged_util import DEV, int32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,ld,capacity", [(1, 5, 100), (5, 9, 100), (7, 3000, 30000), (1024, 4, 9000), (1500, 7, 20000), (1500, 7, 3000), (2100, 40, 90000)])
def test_entries_that_are_no_page(B, ld, capacity):
    P, rng = 16, np.random.default_rng(B + ld)
    lens = rng.integers(0, ld * P + 1, B)
    lens[rng.random(B) < 0.2] = 0
    keep = np.where(rng.random(B) < 0.5, 0, rng.integers(-3, ld * P + 1, B))
    table = np.full((B, ld), -1, dtype=np.int64)
    page = 0
    for b in range(B):
        n = oracle.ceil_div(int(lens[b]), P)
        table[b, :n] = page + np.arange(n)
        page += n
    table[rng.random((B, ld)) < 0.3] = -1
    table[rng.random((B, ld)) < 0.02] = -5
    free = np.full(capacity, 777777, dtype=np.int64)
    free[:3] = (-9, 800000, 800001)
    dev = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in (table, lens, free)]
    count = int32([3])
    idxc.page_release(dev[0], dev[1], int32(keep.tolist()), dev[2], count, P)
    want = oracle.page_release(table, lens, keep, free, 3, P)
    for name, a, b in zip(("table", "lens", "free", "count"), (*dev, count), want):
        assert np.array_equal(a.cpu().numpy().reshape(-1), np.asarray(b).reshape(-1)), name
    stack = dev[2][3:int(count)].cpu().numpy()
    assert (stack >= 0).all() and np.unique(stack).size == stack.size


def test_what_was_given_back_is_handed_out_again():
    """A request with a hole: its pages, and only they, serve the next one."""
    P, table, lens = 16, int32([[3, -1, 5, 2]]), int32([60])
    free, count = torch.full((8,), -1, dtype=torch.int32, device=DEV), int32([0])
    idxc.page_release(table, lens, None, free, count, P)
    assert count.tolist() == [3] and free[:3].tolist() == [2, 5, 3] and table.tolist() == [[-1] * 4]
    slots, begin, start = torch.zeros(48, dtype=torch.int64, device=DEV), int32([0, 0]), int32([0])
    idxc.page_tables(table, lens, int32([48]), free, count, P, slots, begin, start)
    assert start.tolist() == [0] and table.tolist() == [[3, 5, 2, -1]] and bool((slots >= 0).all())
    idxc.page_tables(table, lens, int32([1]), free, count, P, slots, begin, start)
    assert start.tolist() == [-1]
