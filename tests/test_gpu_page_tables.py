"""Block tables, slots, release and rows of a paged cache against the oracle: every number has to be equal."""
import numpy as np
import pytest
import torch

from oracle import paged as oracle
from paper_2603_12201_b200 import binding as idxc
from tests.paged_util import DEV, gen, int32

pytestmark = pytest.mark.gpu


class State:
    def __init__(self, B, ld, n_pages, P, seed, capacity=None):
        g = gen(seed)
        self.P = P
        self.table = torch.full((B, ld), -1, dtype=torch.int32, device=DEV)
        self.lens = torch.zeros(B, dtype=torch.int32, device=DEV)
        self.free = torch.full((capacity or n_pages,), -7, dtype=torch.int32, device=DEV)
        self.free[:n_pages] = torch.randperm(n_pages, generator=g).to(torch.int32).to(DEV)
        self.count = int32([n_pages])

    def host(self):
        return self.table.cpu().numpy(), self.lens.cpu().numpy(), self.free.cpu().numpy(), int(self.count)

    def grow(self, new, n_slots, with_seq=True):
        B = self.table.shape[0]
        slots = torch.full((n_slots,), 12345, dtype=torch.int64, device=DEV)
        seq = torch.full((n_slots,), 12345, dtype=torch.int32, device=DEV) if with_seq else None
        begin, start = torch.full((B + 1,), 99, dtype=torch.int32, device=DEV), torch.full((B,), 99, dtype=torch.int32, device=DEV)
        table, lens, free, count = self.host()
        idxc.page_tables(self.table, self.lens, int32(new), self.free, self.count, self.P, slots, begin, start, seq)
        want = oracle.page_tables(table, lens, new, free, count, self.P, n_slots)
        got = (self.table, self.lens, self.count, begin, start, slots, seq)
        for name, a, b in zip(("table", "lens", "count", "begin", "start", "slots", "seq"), got, want):
            if a is not None:
                assert np.array_equal(a.cpu().numpy().reshape(-1), np.asarray(b).reshape(-1)), name
        assert np.array_equal(self.free.cpu().numpy(), free)
        return slots, begin, start

    def cut(self, keep):
        table, lens, free, count = self.host()
        idxc.page_release(self.table, self.lens, None if keep is None else int32(keep), self.free, self.count, self.P)
        want = oracle.page_release(table, lens, np.zeros_like(lens) if keep is None else keep, free, count, self.P)
        for name, a, b in zip(("table", "lens", "free", "count"), (self.table, self.lens, self.free, self.count), want):
            assert np.array_equal(a.cpu().numpy().reshape(-1), np.asarray(b).reshape(-1)), name


@pytest.mark.parametrize("B,P,top", [(1, 16, 300), (7, 48, 100), (64, 16, 5), (1024, 64, 40), (1025, 16, 3), (3000, 32, 9)])
def test_steps_of_a_serving_loop(B, P, top):
    rng = np.random.default_rng(B)
    n_pages = 3 * B * max(1, top // P) + 2
    s = State(B, 4 + 3 * top // P, n_pages, P, B)
    for step in range(6):
        new = rng.integers(0, top + 1, B)
        if step == 3:
            new[:] = 0
        s.grow(new.tolist(), int(new.sum()) + (0 if step % 2 else 5), with_seq=step != 1)
        lens = s.lens.cpu().numpy()
        s.cut(rng.integers(0, lens + 1).tolist() if step % 3 else (lens - rng.integers(0, 2, B)).tolist())
    s.cut(None)
    assert int(s.count) == n_pages and not s.lens.any() and bool((s.table == -1).all())


def test_taking_and_giving_back_is_the_identity():
    s = State(50, 9, 300, 16, 3)
    rng = np.random.default_rng(0)
    s.grow(rng.integers(1, 90, 50).tolist(), 5000)
    table, lens, free, count = s.host()
    s.grow(rng.integers(0, 30, 50).tolist(), 2000)
    s.cut(lens.tolist())
    for a, b in zip(s.host(), (table, lens, free, count)):
        assert np.array_equal(a, b)


@pytest.mark.parametrize("B", [5, 1500])
def test_refusals_are_a_suffix(B):
    s = State(B, 6, 2 * B, 16, 1)
    rng = np.random.default_rng(B)
    _, _, start = s.grow(rng.integers(1, 80, B).tolist(), 200 * B)      # the stack runs out
    assert (start < 0).any() and (start >= 0).any()
    s = State(B, 4, 8 * B, 16, 1)
    _, _, start = s.grow([16] * (B // 2) + [65] + [1] * (B - B // 2 - 1), 20 * B + 100)      # one does not fit its row of the table
    assert (start >= 0).sum() == B // 2
    s = State(B, 4, 8 * B, 16, 1)
    _, _, start = s.grow([3] * B, 3 * (B - 1))                          # one token's slot is missing
    assert (start >= 0).sum() == B - 1


def test_many_tokens_take_the_second_kernel():
    s = State(9, 700, 4000, 16, 5)
    s.grow([1000, 0, 7000, 1, 10, 2500, 0, 4000, 15], 15000)
    s.grow([3, 9000, 0, 0, 1, 1, 2, 1, 0], 9008)
    s.cut([0, 5, 7000, 1, 0, 2500, 1, 3999, 16])


def test_many_requests_whose_sums_pass_int_range_are_refused():
    s = State(40, 3, 10, 16, 5)
    B = 40
    slots = torch.zeros(4, dtype=torch.int64, device=DEV)
    begin, start = torch.zeros(B + 1, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    idxc.page_tables(s.table, s.lens, int32([1] + [2 ** 30] * (B - 1)), s.free, s.count, 16, slots, begin, start)
    assert start.tolist() == [0] + [-1] * (B - 1) and int(s.count) == 9 and begin.tolist()[:3] == [0, 1, 2 ** 30 + 1] and begin.tolist()[3:] == [2 ** 31 - 1] * (B - 2)
    assert slots.tolist()[1:] == [-1] * 3 and slots[0] >= 0


def test_no_requests_and_no_tokens():
    e = torch.zeros(0, dtype=torch.int32, device=DEV)
    free, count, begin = int32([4, 5]), int32([2]), int32([77])
    slots = torch.zeros(3, dtype=torch.int64, device=DEV)
    idxc.page_tables(torch.zeros((0, 4), dtype=torch.int32, device=DEV), e, e, free, count, 16, slots, begin, e.clone())
    assert begin.tolist() == [0] and slots.tolist() == [-1] * 3 and count.tolist() == [2]
    s = State(3, 2, 4, 16, 0)
    s.grow([0, 0, 0], 0)


def test_a_stack_without_room_drops_pages():
    s = State(2, 4, 6, 16, 2)
    s.grow([40, 20], 60)
    s.free = s.free[:3].contiguous()
    s.cut([0, 0])
    assert int(s.count) == 3


def test_a_count_above_the_capacity_is_the_capacity():
    s = State(1, 8, 3, 16, 2)
    s.count.fill_(1000)
    slots, begin, start = torch.zeros(40, dtype=torch.int64, device=DEV), int32([0, 0]), int32([0])
    idxc.page_tables(s.table, s.lens, int32([40]), s.free, s.count, 16, slots, begin, start)
    assert start.tolist() == [0] and int(s.count) == 0
    s.count.fill_(-5)
    idxc.page_tables(s.table, s.lens, int32([40]), s.free, s.count, 16, slots, begin, start)
    assert start.tolist() == [-1] and int(s.count) == 0 and slots.tolist() == [-1] * 40


@pytest.mark.parametrize("k", [1, 4, 7, 2048])
def test_rows(k):
    g = gen(k)
    B, ld, P = 13, 40, 48
    table = torch.randint(-1, 5000, (B, ld), generator=g).to(torch.int32)
    pos = torch.randint(-2, ld * P + 30, (29, k), generator=g).to(torch.int32)
    pos[0, 0] = 2 ** 31 - 1
    seq = torch.randint(-1, B + 1, (29,), generator=g).to(torch.int32)
    out = torch.full((29, k), 55, dtype=torch.int32, device=DEV)
    idxc.page_rows(table.to(DEV), pos.to(DEV), P, out, seq.to(DEV))
    assert np.array_equal(out.cpu().numpy(), oracle.page_rows(table.numpy(), pos.numpy(), P, seq.numpy()))
    own = pos[:B].to(DEV).contiguous()
    idxc.page_rows(table.to(DEV), own, P, own)                    # in place, row r is request r
    assert np.array_equal(own.cpu().numpy(), oracle.page_rows(table.numpy(), pos[:B].numpy(), P))
