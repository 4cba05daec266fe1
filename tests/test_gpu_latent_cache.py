"""GPU: 4-bit rows written and read back, positions chosen for eviction, rows brought together."""
import numpy as np
import pytest
import torch

from oracle import latent as oracle
from tests.latent_util import bf16_rows, cache_rows, q4_rows, stored

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def idxc():
    from paper_2603_12201_b200 import binding
    return binding


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


# ------------------------------------------------------------------ quantise / dequantise
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 257])
def test_quantize_bytes_match_the_definition(idxc, n):
    g = gen(n)
    x = bf16_rows(n, g) * torch.exp(torch.randn((n, 576), generator=g) * 2).to(torch.bfloat16)
    x[0, :64] = 0                                                     # groups of zeros
    x[n // 2, 64:96] = torch.tensor([7.0, 0.5, 1.5, -2.5, 3.5, -0.5, 6.5, -6.5] * 4).to(torch.bfloat16)     # ties
    cache = torch.full((n + 2, 416), 0xA5, dtype=torch.uint8, device=DEV)
    idxc.quantize_q4(x.to(DEV), cache[:n])
    got = cache.cpu().numpy()
    assert np.array_equal(got[:n], oracle.quantize_rows(x.double().numpy()))
    assert np.all(got[n:] == 0xA5)
    out = torch.full((n + 1, 576), -3.0, dtype=torch.bfloat16, device=DEV)
    idxc.dequantize_q4(cache[:n], out[:n])
    assert np.array_equal(out[:n].double().cpu().numpy(), oracle.row_values(got[:n]))
    assert bool((out[n:] == -3.0).all())


def test_quantize_every_quotient_near_a_border(idxc):
    """Every bf16 magnitude of one binade under every 5-bit scale of a binade: halves and their neighbours among them."""
    m = torch.arange(128, 256, dtype=torch.float32) / 128.0
    rows = []
    for e in range(-4, 4):
        for s in range(16, 32):
            vals = (m * 2.0 ** e)[m * 2.0 ** e <= 7 * s / 16]
            row = torch.zeros(512)
            row[:vals.numel()] = vals
            row = row.reshape(16, 32)
            row[:, 31] = torch.where(row[:, 31] != 0, row[:, 31], torch.tensor(7.0 * s / 16))
            rows.append(torch.cat([row.reshape(512), torch.zeros(64)]))
    x = torch.stack(rows).to(torch.bfloat16)
    cache = torch.empty((x.shape[0], 416), dtype=torch.uint8, device=DEV)
    idxc.quantize_q4(x.to(DEV), cache)
    assert np.array_equal(cache.cpu().numpy(), oracle.quantize_rows(x.double().numpy()))


def test_quantize_extreme_magnitudes(idxc):
    x = torch.zeros((4, 576))
    x[0, :32] = torch.logspace(-38, -30, 32)
    x[1, :32] = torch.linspace(-1, 1, 32) * 3.3e38      # (a linspace between the ends would overflow on their distance)
    x[2, 0] = 2.0 ** -126
    x[3, 5] = 7 * 2.0 ** -100
    x = x.to(torch.bfloat16)
    cache = torch.empty((4, 416), dtype=torch.uint8, device=DEV)
    out = torch.empty((4, 576), dtype=torch.bfloat16, device=DEV)
    idxc.quantize_q4(x.to(DEV), cache)
    idxc.dequantize_q4(cache, out)
    v = out.double().cpu().numpy()
    assert np.all(np.isfinite(v))
    assert np.array_equal(cache.cpu().numpy()[[0, 2, 3]], oracle.quantize_rows(x.double().numpy()[[0, 2, 3]]))
    # the largest scale, 1.3125 * 2^123: half a step off at most, or the clipped end
    xs = x.double().numpy()[1, :32]
    assert np.all(np.abs(v[1, :32] - xs) <= np.maximum(0.5 * 1.3125 * 2.0 ** 123, np.abs(xs) - 7 * 1.3125 * 2.0 ** 123) * (1 + 1e-12))


def test_scatter_writes_its_rows_only(idxc):
    g = gen(5)
    x = bf16_rows(40, g).to(DEV)
    cache = torch.full((100, 416), 7, dtype=torch.uint8, device=DEV)
    dst = torch.randperm(100, generator=g)[:40].to(DEV)
    dst[3], dst[9] = -1, 100                                          # outside: not written
    idxc.quantize_q4(x, cache, dst_rows=dst)
    want = np.full((100, 416), 7, dtype=np.uint8)
    rows = oracle.quantize_rows(x.double().cpu().numpy())
    for r, d in enumerate(dst.tolist()):
        if 0 <= d < 100:
            want[d] = rows[r]
    assert np.array_equal(cache.cpu().numpy(), want)
    out = torch.empty((40, 576), dtype=torch.bfloat16, device=DEV)
    idxc.dequantize_q4(cache, out, src_rows=dst)
    v = oracle.row_values(rows)
    v[[3, 9]] = 0
    assert np.array_equal(out.double().cpu().numpy(), v)


def test_rows_past_four_gigabytes(idxc):
    n = (1 << 32) // 416 + 100
    cache = torch.empty((n, 416), dtype=torch.uint8, device=DEV)
    x = bf16_rows(64, gen(6)).to(DEV)
    dst = torch.arange(n - 64, n, device=DEV)
    idxc.quantize_q4(x, cache, dst_rows=dst)
    assert np.array_equal(cache[n - 64:].cpu().numpy(), oracle.quantize_rows(x.double().cpu().numpy()))
    out = torch.empty((64, 576), dtype=torch.bfloat16, device=DEV)
    idxc.dequantize_q4(cache, out, src_rows=dst)
    assert np.array_equal(out.double().cpu().numpy(), oracle.row_values(cache[n - 64:].cpu().numpy()))


# ------------------------------------------------------------------ which positions stay
def select(idxc, acc, lens, budget, recent):
    B = acc.shape[0]
    keep = torch.full((B, budget), -77, dtype=torch.int32, device=DEV)
    new = torch.full((B,), -77, dtype=torch.int32, device=DEV)
    idxc.evict_select(acc.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), budget, recent, keep, new)
    return keep.cpu().numpy(), new.cpu().numpy()


@pytest.mark.parametrize("ld,lens,budget,recent", [
    (1, [1, 0], 1, 1), (7, [7, 3, 0, 5], 3, 1), (64, [64, 63, 1], 63, 63), (1000, [1000, 999, 500, 512], 512, 0), (5000, [5000, 4097, 1024], 1, 0),
    (5000, [5000, 4999, 4096], 4095, 17), (20001, [20001, 16384, 9], 2048, 128), (131072, [131072, 131071, 70000], 32768, 512),
    (300000, [300000, 262145], 100001, 1000)])
@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "signed"])
def test_select_matches_the_definition(idxc, ld, lens, budget, recent, kind):
    rng = np.random.default_rng(ld + budget)
    B = len(lens)
    acc = {"spread": lambda: rng.random((B, ld)) ** 12, "ties": lambda: rng.integers(0, 5, (B, ld)) / 4.0, "equal": lambda: np.full((B, ld), 0.25),
           "signed": lambda: rng.standard_normal((B, ld)) * 10.0 ** rng.integers(-40, 30, (B, ld))}[kind]().astype(np.float32)
    if kind == "signed":
        acc[:, ::7] = -0.0
        acc[:, 3::7] = 0.0
    keep, new = select(idxc, torch.from_numpy(acc), lens, budget, recent)
    for b, n in enumerate(lens):
        want = oracle.evict(acc[b], n, budget, recent)
        assert new[b] == len(want)
        assert np.array_equal(keep[b, :len(want)], want) and np.all(keep[b, len(want):] == -1)


def test_select_clamps_lengths_and_stands_not_a_number(idxc):
    acc = torch.rand(3, 100)
    keep, new = select(idxc, acc, [200, -5, 50], 60, 10)
    assert new.tolist() == [60, 0, 50]
    assert np.array_equal(keep[0], oracle.evict(acc[0].numpy(), 100, 60, 10))
    acc[:] = float("nan")
    acc[1, 5] = float("inf")
    keep, new = select(idxc, acc, [100, 100, 100], 60, 10)
    assert np.all(new == 60) and np.all(np.diff(keep, axis=1) > 0) and keep.min() >= 0 and keep.max() < 100
    assert 5 in keep[1]


# ------------------------------------------------------------------ rows brought together
def make_keep(rng, lens, budget):
    keep = np.full((len(lens), budget), -1, dtype=np.int32)
    new = np.zeros(len(lens), dtype=np.int32)
    for b, n in enumerate(lens):
        m = min(n, budget)
        keep[b, :m] = np.sort(rng.choice(n, m, replace=False)) if n else []
        new[b] = m
    return keep, new


@pytest.mark.parametrize("shape,dtype", [((576,), torch.bfloat16), ((416,), torch.uint8), ((128,), torch.uint8), ((), torch.float32), ((5,), torch.float32), ((7, 2), torch.bfloat16)])
@pytest.mark.parametrize("lens,budget", [([5, 0, 1], 3), ([300, 40, 299], 100), ([9000, 4097, 2048, 100], 2048), ([70000], 33333)])
def test_compaction(idxc, shape, dtype, lens, budget):
    rng = np.random.default_rng(sum(lens) + budget)
    base = np.cumsum([2] + [n + 3 for n in lens])[:-1]
    rows = int(base[-1] + lens[-1] + 4)
    src = torch.from_numpy(rng.integers(0, 120, (rows, *shape)).astype(np.int64)).to(dtype).to(DEV)
    keep, new = make_keep(rng, lens, budget)
    k, n = torch.from_numpy(keep).to(DEV), torch.from_numpy(new).to(DEV)
    sb = torch.from_numpy(base).to(DEV)
    before = src.clone()
    # to another buffer
    db = torch.arange(len(lens), device=DEV) * (budget + 1) + 1
    dst = torch.full((len(lens) * (budget + 1) + 2, *shape), 99, device=DEV).to(dtype)
    want = dst.clone()
    for b in range(len(lens)):
        if new[b]:
            want[int(db[b]):int(db[b]) + int(new[b])] = before[sb[b] + k[b, :int(new[b])].long()]
    idxc.compact_rows(src, dst, k, n, sb, db)
    assert torch.equal(dst, want) and torch.equal(src, before)
    # in place, twice from the same start
    for _ in range(2):
        got = before.clone()
        want = before.clone()
        for b in range(len(lens)):
            if new[b]:
                want[int(base[b]):int(base[b]) + int(new[b])] = before[sb[b] + k[b, :int(new[b])].long()]
        idxc.compact_rows(got, got, k, n, sb)
        assert torch.equal(got, want)


def test_compaction_ignores_entries_that_name_no_row(idxc):
    src = torch.arange(20, dtype=torch.float32, device=DEV)
    keep = torch.tensor([[2, -1, 30, 7, 9]], dtype=torch.int32, device=DEV)
    zero = torch.zeros(1, dtype=torch.int64, device=DEV)
    dst = torch.full((4,), -1.0, device=DEV)
    idxc.compact_rows(src, dst, keep, torch.tensor([9], dtype=torch.int32, device=DEV), zero, zero)
    assert dst.tolist() == [2.0, -1.0, -1.0, 7.0]                      # place 4 is no row of dst, n_keep is clamped to 5
    idxc.compact_rows(src, src, keep, torch.tensor([5], dtype=torch.int32, device=DEV), zero)
    assert src[:5].tolist() == [2.0, 1.0, 2.0, 7.0, 9.0]


def test_evicted_cache_reads_as_the_selection(idxc):
    """Choosing, compacting and then attending the smaller cache = sparse attention over the chosen positions of the old one."""
    g = gen(11)
    lens, budget, recent = [700, 90, 333], 128, 16
    base = torch.tensor([0, 700, 790], device=DEV)
    kv = q4_rows(1123, g).to(DEV)
    acc = torch.rand((3, 700), generator=g).to(DEV)
    q = bf16_rows(3 * 16, g).reshape(3, 16, 576).to(DEV)
    keep = torch.empty((3, budget), dtype=torch.int32, device=DEV)
    new = torch.empty(3, dtype=torch.int32, device=DEV)
    idxc.evict_select(acc, torch.tensor(lens, dtype=torch.int32, device=DEV), budget, recent, keep, new)
    want, want_lse = idxc.sparse_attention_q4(q, kv, keep, 512, 0.05, kv_base=base)
    idxc.compact_rows(kv, kv, keep, new, base)
    got, lse = idxc.latent_attention(q.unsqueeze(1), kv, base, new, budget, 512, 0.05)
    assert torch.allclose(lse.squeeze(1), want_lse, atol=1e-5)
    assert torch.allclose(got.squeeze(1).float(), want.float(), atol=2e-2, rtol=2e-2)


@pytest.mark.parametrize("shape,dtype", [((416,), torch.uint8), ((), torch.float32)])
def test_compaction_from_bases_far_outside_moves_nothing(idxc, shape, dtype):
    """Bases near the ends of 64 bits, where a base plus a position would wrap around into the array or far in front of it."""
    src = torch.arange(40, device=DEV).reshape(40, *[1] * len(shape)).expand(40, *shape).to(dtype).contiguous()
    before = src.clone()
    ends = [2 ** 63 - 1, 2 ** 63 - 3, 2 ** 63 - 10, -2 ** 63, -2 ** 63 + 2, -2 ** 31, -2 ** 31 - 1, 40, 2 ** 40]
    base = torch.tensor(ends, dtype=torch.int64, device=DEV)
    keep = torch.tensor([[1, 2, 5, 2 ** 31 - 1]], dtype=torch.int32, device=DEV).repeat(len(ends), 1)
    n = torch.full((len(ends),), 4, dtype=torch.int32, device=DEV)
    idxc.compact_rows(src, src, keep, n, base)
    assert torch.equal(src, before)
    dst = torch.full_like(src, 99)
    want = dst.clone()
    idxc.compact_rows(src, dst, keep, n, base, torch.zeros_like(base))
    assert torch.equal(dst, want)
    idxc.compact_rows(src, dst, keep, n, torch.zeros_like(base), base)
    assert torch.equal(dst, want) and torch.equal(src, before)
    # the edge itself: a base just in front of the array
    base = torch.tensor([-3], dtype=torch.int64, device=DEV)
    idxc.compact_rows(src, dst, keep[:1], n[:1], base, torch.zeros_like(base))
    want[2] = before[2]
    assert torch.equal(dst, want)


def test_choice_and_compaction_at_their_limits(idxc):
    """65535 sequences, and rows of 2^20 bytes."""
    B, ld, budget = 65535, 5, 3
    acc = torch.rand((B, ld), generator=gen(1)).to(DEV)
    lens = torch.randint(0, ld + 1, (B,), generator=gen(2), dtype=torch.int32).to(DEV)
    keep, new = torch.empty((B, budget), dtype=torch.int32, device=DEV), torch.empty((B,), dtype=torch.int32, device=DEV)
    idxc.evict_select(acc, lens, budget, 1, keep, new)
    base = torch.arange(B, device=DEV) * ld
    moved = acc.clone().view(-1)
    idxc.compact_rows(moved, moved, keep, new, base)
    moved, k = moved.view(B, ld).cpu().numpy(), keep.cpu().numpy()
    for b in list(range(0, B, 997)) + [B - 1]:
        want = oracle.evict(acc[b].cpu().numpy(), int(lens[b]), budget, 1)
        assert int(new[b]) == len(want) and np.array_equal(k[b, :len(want)], want)
        assert np.array_equal(moved[b, :len(want)], acc[b].cpu().numpy()[want])
    src = torch.randint(0, 2 ** 31 - 1, (9, 2 ** 18), generator=gen(3), dtype=torch.int32).to(DEV)
    pick = torch.tensor([[0, 3, 4, 8]], dtype=torch.int32, device=DEV)
    zero, n = torch.zeros(1, dtype=torch.int64, device=DEV), torch.tensor([4], dtype=torch.int32, device=DEV)
    dst = torch.zeros((4, 2 ** 18), dtype=torch.int32, device=DEV)
    idxc.compact_rows(src, dst, pick, n, zero)
    assert torch.equal(dst, src[pick[0].long()])
    idxc.compact_rows(src, src, pick, n, zero)
    assert torch.equal(src[:4], dst)


@pytest.mark.parametrize("binade", [0, -95, 60])
def test_quantize_every_quotient(idxc, binade):
    """Every bf16 magnitude of both signs that a 5-bit scale holds, down to 1/64 of the scale's binade, under all sixteen scales of a binade:
    31 values a group, and in the last column 7 steps, which make the scale."""
    m = torch.arange(128, 256, dtype=torch.float64) / 128.0
    mags = torch.cat([m * 2.0 ** e for e in range(-6, 4)])
    groups, scales, pairs = [], [], 0
    for s in range(16, 32):
        v = mags[mags <= 7 * s / 16]
        pairs += v.numel()
        v = torch.cat([v, -v])
        v = torch.cat([v, torch.zeros(-v.numel() % 31, dtype=torch.float64)]).view(-1, 31)
        groups.append(torch.cat([v, torch.full((v.shape[0], 1), 7 * s / 16, dtype=torch.float64)], dim=1))
        scales += [s / 16] * v.shape[0]
    rows = -(-len(scales) // 16)
    scales += [1.0] * (16 * rows - len(scales))
    last = torch.zeros((16 * rows, 32), dtype=torch.float64)
    last[:, 31] = 7.0
    every = torch.cat(groups)
    last[:every.shape[0]] = every
    x = torch.cat([last.view(rows, 512), torch.zeros((rows, 64), dtype=torch.float64)], dim=1) * 2.0 ** binade
    assert torch.equal(x.to(torch.bfloat16).double(), x)
    cache = torch.empty((rows, 416), dtype=torch.uint8, device=DEV)
    idxc.quantize_q4(x.to(torch.bfloat16).to(DEV), cache)
    got = cache.cpu()
    stored_scales = got[:, 256:288].contiguous().view(torch.bfloat16).double().reshape(-1)
    assert torch.equal(stored_scales, torch.tensor(scales, dtype=torch.float64) * 2.0 ** binade)
    met = torch.stack([torch.tensor(scales, dtype=torch.float64).repeat_interleave(31), (x[:, :512].reshape(-1, 32)[:, :31] * 2.0 ** -binade).reshape(-1)])
    assert torch.unique(met[:, met[1] != 0], dim=1).shape[1] == 2 * pairs
    assert np.array_equal(got.numpy(), oracle.quantize_rows(x.numpy()))


@pytest.mark.parametrize("B,ld", [(1, 8704), (1, 8705), (37, 27136), (37, 27137), (148, 60000), (148, 83969), (149, 46081), (300, 9000)])
def test_select_on_both_sides_of_its_rule(idxc, B, ld):
    """One block a sequence or eight, with keys that fit one block's shared memory and keys that do not."""
    g = gen(B + ld)
    lens = [ld - 13 * (b % 5) for b in range(B)]
    acc = torch.rand((B, ld), generator=g) ** 12
    acc[:, ::3] = 0.0                                    # ties, more of them than stay
    budget = ld // 3
    keep, new = select(idxc, acc, lens, budget, 100)
    for b in sorted({0, 1 % B, B // 2, B - 1}):
        want = oracle.evict(acc[b].numpy(), lens[b], budget, 100)
        assert new[b] == budget and np.array_equal(keep[b], want)
    assert np.all(np.diff(keep, axis=1) > 0) and np.all(new == budget)
