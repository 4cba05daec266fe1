"""Latent-cache operators at the edges: scores that are no numbers, rows of sums too long for shared memory, pairs whose second half is empty."""
import numpy as np
import pytest
import torch

from oracle import latent as oracle
from tests.latent_util import bf16_rows, cache_rows, check_attention, oracle_sequence, q4_rows, stored
from tests.test_gpu_latent_attention import weights_bound

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def idxc():
    from paper_2603_12201_b200 import binding
    return binding


def gen(seed):
    return torch.Generator().manual_seed(seed)


def set_nan(kv, row):
    """A positional column of a cache row becomes NaN: its score is none for every head, its values stay what they are."""
    if kv.dtype == torch.uint8:
        kv[row, 288 + 2 * 5 + 1] = 0x7F
        kv[row, 288 + 2 * 5] = 0xC0
    else:
        kv[row, 512 + 5] = float("nan")


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("H", [16, 128])
@pytest.mark.parametrize("lens,at", [([40, 70], 10), ([9000, 300], 0), ([9000, 300], 8999), ([64 * 300, 65], 9001)])
def test_a_visible_row_that_is_no_number_shows(idxc, lens, at, H, four):
    """In whichever piece of a cut sequence it lies; the other sequence does not notice."""
    g = gen(lens[0] + at + H)
    kv = cache_rows(sum(lens), four, g)
    set_nan(kv, at)
    q = bf16_rows(2 * H, g, 0.5).view(2, 1, H, 576)
    base = torch.tensor([0, lens[0]], device=DEV)
    out, lse = idxc.latent_attention(q.to(DEV), kv.to(DEV), base, torch.tensor(lens, dtype=torch.int32, device=DEV), max(lens), 512, 1 / 24)
    assert torch.isnan(out[0]).all() and torch.isnan(lse[0]).all()
    check_attention(out[1].reshape(H, 512), lse[1].reshape(H), *oracle_sequence(q[1], kv, lens[0], lens[1], 1, 1 / 24)[:4])


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("H,head", [(16, 3), (128, 0), (128, 127), (100, 64)])
def test_a_head_that_is_no_number_shows_alone(idxc, H, head, four):
    n = 5000
    g = gen(H + head)
    kv = cache_rows(n, four, g)
    q = bf16_rows(H, g, 0.5).view(1, 1, H, 576)
    clean = q.clone()
    q[0, 0, head, 100] = float("nan")
    out, lse = idxc.latent_attention(q.to(DEV), kv.to(DEV), None, torch.tensor([n], dtype=torch.int32, device=DEV), n, 512, 1 / 24)
    assert torch.isnan(out[0, 0, head]).all() and torch.isnan(lse[0, 0, head])
    others = [h for h in range(H) if h != head]
    want = oracle_sequence(clean[0], kv, 0, n, 1, 1 / 24)[:4]
    check_attention(out[0, 0, others], lse[0, 0, others], *(w[others] for w in want))


def test_a_selected_row_that_is_no_number_shows(idxc):
    g = gen(5)
    kv = q4_rows(3000, g)
    set_nan(kv, 1234)
    for H, k_top in ((128, 2048), (16, 100)):
        q = bf16_rows(2 * H, g, 0.5).view(2, H, 576)
        topk = torch.stack([torch.arange(k_top), torch.arange(k_top)]).to(torch.int32)
        topk[0, k_top - 1] = 1234
        topk[1][topk[1] == 1234] = -1
        out, lse = idxc.sparse_attention_q4(q.to(DEV), kv.to(DEV), topk.to(DEV), 512, 1 / 24)
        assert torch.isnan(out[0]).all() and torch.isnan(lse[0]).all()
        assert torch.isfinite(out[1].float()).all() and torch.isfinite(lse[1]).all()
        rows = topk[1][topk[1] >= 0].long()
        sub = kv[rows]
        check_attention(out[1], lse[1], *oracle_sequence(q[1:2], sub, 0, len(rows), 1, 1 / 24)[:4])


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("H,n_step", [(50, 3), (65, 1), (33, 4), (128, 3), (43, 3)])
def test_rows_that_end_inside_the_first_half_of_a_pair(idxc, H, n_step, four):
    """H n_step = 150, 65, 132, 384, 129: the last pair of a sequence has its second 64 rows in part or not at all."""
    lens = [700, 1, 130]
    g = gen(H)
    kv = cache_rows(sum(lens), four, g)
    q = bf16_rows(3 * n_step * H, g, 0.5).view(3, n_step, H, 576)
    base = torch.tensor(np.concatenate([[0], np.cumsum(lens)[:-1]]), device=DEV)
    out, lse = idxc.latent_attention(q.to(DEV), kv.to(DEV), base, torch.tensor(lens, dtype=torch.int32, device=DEV), max(lens), 512, 1 / 24)
    for b, n in enumerate(lens):
        check_attention(out[b].reshape(-1, 512), lse[b].reshape(-1), *oracle_sequence(q[b], kv, int(base[b]), n, n_step, 1 / 24)[:4], f"sequence {b}")


@pytest.mark.parametrize("kind", ["spread", "ties", "equal"])
def test_select_in_rows_longer_than_shared_memory_holds(idxc, kind):
    """Above 8 x 49152 positions a sequence the keys are read from global memory in every pass."""
    ld, lens, budget, recent = 500001, [500001, 393217, 400000, 77], 70001, 333
    rng = np.random.default_rng(11)
    acc = {"spread": rng.random((4, ld)) ** 12, "ties": rng.integers(0, 5, (4, ld)) / 4.0, "equal": np.full((4, ld), 0.25)}[kind].astype(np.float32)
    keep = torch.full((4, budget), -77, dtype=torch.int32, device=DEV)
    new = torch.full((4,), -77, dtype=torch.int32, device=DEV)
    idxc.evict_select(torch.from_numpy(acc).to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), budget, recent, keep, new)
    for b, n in enumerate(lens):
        want = oracle.evict(acc[b], n, budget, recent)
        m = len(want)
        assert int(new[b]) == m
        assert np.array_equal(keep[b, :m].cpu().numpy(), want)
        assert (keep[b, m:] == -1).all()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("H", [8, 72])
@pytest.mark.parametrize("B,n", [(2, 1700), (30, 300), (37, 500), (38, 300), (74, 65), (75, 64), (100, 129), (128, 64), (129, 200), (150, 70)])
def test_sequences_of_one_length(idxc, B, n, H, four):
    """Batches whose sequences are cut each by itself, or not at all, and every third batch with an empty and a longer one among them."""
    lens = [n] * B
    if B % 3 == 0:
        lens[B // 2], lens[-1] = 0, n + 3
    g = gen(B + H)
    total = sum(lens)
    kv = cache_rows(total, four, g)
    q = bf16_rows(B * H, g, 0.5).view(B, 1, H, 576)
    base = np.concatenate([[0], np.cumsum(lens)[:-1]])
    out, lse = idxc.latent_attention(q.to(DEV), kv.to(DEV), torch.tensor(base, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), max(lens), 512, 1 / 24)
    for b in sorted({0, 1, B // 3, B // 2, B - 2, B - 1}):
        check_attention(out[b, 0], lse[b, 0], *oracle_sequence(q[b], kv, int(base[b]), lens[b], 1, 1 / 24)[:4], f"sequence {b}")
    assert torch.isfinite(out.float()).all()


def test_captured_run_with_copies_forks_and_joins(idxc):
    """The cache's kernels behind a copy, a fill, each other and kernels of another stream, in a graph: every replay sees the inputs of its time."""
    n, budget = 600, 128
    g = gen(3)
    src, x, kept = bf16_rows(n, g).to(DEV), torch.zeros(n, 576, dtype=torch.bfloat16, device=DEV), torch.empty(n, 576, dtype=torch.bfloat16, device=DEV)
    cache, small = torch.zeros(n, 416, dtype=torch.uint8, device=DEV), torch.zeros(budget, 416, dtype=torch.uint8, device=DEV)
    back, side = torch.empty(n, 576, dtype=torch.bfloat16, device=DEV), torch.empty(budget, 576, dtype=torch.bfloat16, device=DEV)
    acc_src, acc = torch.rand(1, n, device=DEV), torch.zeros(1, n, device=DEV)
    lens, zero = torch.tensor([n], dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    keep, new = torch.empty(1, budget, dtype=torch.int32, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV)
    q = bf16_rows(16, g, 0.5).view(1, 1, 16, 576).to(DEV)

    def step():
        main, other = torch.cuda.current_stream(), torch.cuda.Stream()
        x.copy_(src)
        idxc.quantize_q4(x, cache)
        other.wait_stream(main)
        with torch.cuda.stream(other):
            acc.copy_(acc_src)
            idxc.evict_select(acc, lens, budget, 5, keep, new)
        idxc.dequantize_q4(cache, back)
        out, lse = idxc.latent_attention(q, cache, None, lens, n, 512, 1 / 24)
        main.wait_stream(other)
        idxc.compact_rows(cache, small, keep, new, zero)
        idxc.dequantize_q4(small, side)
        cache.zero_()
        idxc.quantize_q4(x, cache)
        idxc.dequantize_q4(cache, kept)
        return out, lse

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in range(3):
        src.copy_(bf16_rows(n, gen(seed), 1 + seed))
        acc_src.copy_(torch.rand(1, n, generator=gen(seed)))
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(stored(cache), oracle.quantize_rows(src.double().cpu().numpy()))
        for b in (back, kept):
            assert np.array_equal(b.double().cpu().numpy(), oracle.row_values(stored(cache)))
        want = oracle.evict(acc_src[0].cpu().numpy(), n, budget, 5)
        assert np.array_equal(keep[0].cpu().numpy(), want)
        assert torch.equal(side, back[torch.as_tensor(want, dtype=torch.int64, device=DEV)])
        check_attention(got[0][0, 0], got[1][0, 0], *oracle_sequence(q[0], cache, 0, n, 1, 1 / 24)[:4])


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("lens,H,n_step", [([260], 128, 200), ([77, 400], 20, 77), ([30, 150], 16, 130), ([193], 128, 2), ([64, 65, 3], 100, 5)])
def test_chunks_of_a_prompt(idxc, lens, H, n_step, four):
    """New tokens that fill many units, of which a prompt's first see few positions or none."""
    B = len(lens)
    g = gen(n_step + H)
    kv = cache_rows(sum(lens), four, g)
    q = bf16_rows(B * n_step * H, g, 0.5).view(B, n_step, H, 576)
    base = np.concatenate([[0], np.cumsum(lens)[:-1]])
    out, lse = idxc.latent_attention(q.to(DEV), kv.to(DEV), torch.tensor(base, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), max(lens) + 9, 512, 1 / 24)
    for b, n in enumerate(lens):
        check_attention(out[b].reshape(-1, 512), lse[b].reshape(-1), *oracle_sequence(q[b], kv, int(base[b]), n, n_step, 1 / 24)[:4], f"sequence {b}")


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("H", [16, 128])
def test_bases_far_outside_name_no_row(idxc, H, four):
    """Bases near the ends of 64 bits, where a base plus a position would wrap around: their sequences see nothing, the others everything."""
    n_kv, n = 1000, 700
    bases = [2 ** 63 - 1, 2 ** 63 - 151, 2 ** 63 - 300, 2 ** 63 - 700, -2 ** 63, -2 ** 63 + 200, -2 ** 31 - 1, -2 ** 31, 2 ** 40, n_kv, -n, 250]
    B, g = len(bases), gen(H)
    kv = cache_rows(n_kv, four, g).to(DEV)
    q = bf16_rows(B * H, g).view(B, 1, H, 576).to(DEV)
    base, lens = torch.tensor(bases, dtype=torch.int64, device=DEV), torch.full((B,), n, dtype=torch.int32, device=DEV)
    out, lse = idxc.latent_attention(q, kv, base, lens, n, 512, 1 / 24)
    topk = torch.arange(n, dtype=torch.int32, device=DEV).repeat(B, 1).contiguous()
    topk[:, -1] = 2 ** 31 - 1
    results = [(out[:, 0], lse[:, 0], n)]
    if four:
        results.append((*idxc.sparse_attention_q4(q[:, 0].contiguous(), kv, topk, 512, 1 / 24, kv_base=base), n - 1))
    for o, l, seen in results:
        assert bool((o[:-1] == 0).all()) and bool(torch.isneginf(l[:-1]).all())
        check_attention(o[-1], l[-1], *oracle_sequence(q[-1], kv, 250, seen, 1, 1 / 24)[:4])
    lse = lse.nan_to_num(neginf=0.0)
    for how in (dict(lens=lens, max_len=n), dict(topk=topk)):
        acc = torch.ones((B, n), device=DEV)
        idxc.attention_weights(q, kv, lse, acc, 1 / 24, kv_base=base, **how)
        assert bool((acc[:-1] == 1).all()) and bool((acc[-1, :n - 1] > 1).all())
    idxc.poll_device_status()


# ------------------------------------------------------------------ weights of tokens and heads without a log-sum-exp
@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("lens,H,n_step", [([300, 129], 20, 3), ([1000, 7], 128, 2), ([65, 200], 33, 4)])
def test_tokens_without_a_log_sum_exp_add_nothing(idxc, lens, H, n_step, bad, four):
    """A padding token (lse -inf) may hold anything in q, and so may a single head."""
    g = gen(lens[0] + H)
    kv, scale = cache_rows(sum(lens), four, g), 1 / 24
    q = bf16_rows(2 * n_step * H, g).view(2, n_step, H, 576)
    base = [0, lens[0]]
    seq = [oracle_sequence(q[b], kv, base[b], lens[b], n_step, scale) for b in range(2)]
    lse = torch.tensor(np.stack([s[1] for s in seq]), dtype=torch.float32).view(2, n_step, H)
    off = torch.zeros((2, n_step, H), dtype=torch.bool)
    off[0, n_step - 1] = True                            # the newest token, which sees every position
    off[1, 0, H - 1] = True
    off[1, 1, 0] = True
    q[off] = bad
    lse[off] = float("-inf")
    start = torch.rand((2, max(lens) + 3), generator=g)
    acc = start.clone().to(DEV)
    idxc.attention_weights(q.to(DEV), kv.to(DEV), lse.to(DEV), acc, scale, kv_base=torch.tensor(base, device=DEV),
                           lens=torch.tensor(lens, dtype=torch.int32, device=DEV), max_len=max(lens))
    got = acc.double().cpu().numpy()
    for b, n in enumerate(lens):
        _, _, _, reach, p = seq[b]
        p = np.where(off[b].reshape(-1, 1).numpy(), 0.0, p)
        want = start[b, :n].double().numpy() + p.sum(axis=0)
        # the launches of 128 query rows each round the sum once
        assert np.all(np.abs(got[b, :n] - want) <= weights_bound(p, reach, n_step * H) + 2.0 ** -23 * want), f"sequence {b}"
        assert np.array_equal(got[b, n:], start[b, n:].double().numpy())


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("H", [9, 128])
def test_heads_without_a_log_sum_exp_add_nothing_to_a_selection(idxc, H, four):
    g = gen(H)
    kv, k = cache_rows(400, four, g), 200
    q = bf16_rows(2 * H, g).view(2, H, 576)
    topk = torch.stack([torch.randperm(400, generator=g)[:k] for _ in range(2)]).to(torch.int32)
    lse = torch.empty((2, H))
    start = torch.rand((2, 400), generator=g)
    want, bound = start.double().numpy().copy(), np.zeros((2, 400))
    off = torch.zeros((2, H), dtype=torch.bool)
    off[0, H // 2] = True
    off[1, 1:] = True
    for b in range(2):
        rows = kv[topk[b].long()]
        _, l, _, reach, p = oracle_sequence(q[b:b + 1], rows, 0, k, 1, 0.05)
        lse[b] = torch.from_numpy(l).float()
        p = np.where(off[b].reshape(-1, 1).numpy(), 0.0, p)
        want[b, topk[b].numpy()] += p.sum(axis=0)
        bound[b, topk[b].numpy()] = weights_bound(p, reach, H)
    q[off], lse[off] = float("nan"), float("-inf")
    acc = start.clone().to(DEV)
    idxc.attention_weights(q.to(DEV), kv.to(DEV), lse.to(DEV), acc, 0.05, topk=topk.to(DEV))
    assert np.all(np.abs(acc.double().cpu().numpy() - want) <= bound + 2.0 ** -23 * want)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("H", [5, 40, 128])
def test_a_position_named_again_adds_the_same_number_in_any_order(idxc, H, four):
    """Several threads add to a position that a selection names several times, but all of them the same number: the sum is that of
    repeated fp32 additions, whichever tile, lane or block an entry falls to, and the same in every run."""
    g = gen(H + four)
    n, B, k = 3000, 3, 2001                              # the last tile is not full: its sums take the masked path
    kv = cache_rows(n, four, g).to(DEV)
    q = bf16_rows(B * H, g, 2.0).view(B, H, 576).to(DEV)
    once = torch.stack([torch.randperm(n, generator=g)[:40] for _ in range(B)])
    lse = torch.empty((B, H))
    for b in range(B):
        lse[b] = torch.from_numpy(oracle_sequence(q[b:b + 1].cpu(), kv[once[b].to(DEV)].cpu(), 0, 40, 1, 0.05)[1]).float()
    lse = lse.to(DEV)
    added = torch.zeros((B, n), device=DEV)
    idxc.attention_weights(q, kv, lse, added, 0.05, topk=once.to(torch.int32).to(DEV))
    added = added.cpu().numpy()                          # (0 + w is w)
    times = torch.randint(0, 40, (B, k), generator=g)
    topk = torch.gather(once, 1, times).to(torch.int32)
    start = torch.rand((B, n), generator=g) * 100.0
    want = start.numpy().copy()
    for b in range(B):
        for j in topk[b].tolist():
            want[b, j] = np.float32(want[b, j] + added[b, j])
    for _ in range(5):
        acc = start.clone().to(DEV)
        idxc.attention_weights(q, kv, lse, acc, 0.05, topk=topk.to(DEV))
        assert np.array_equal(acc.cpu().numpy(), want)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("H,n", [(16, 70), (16, 9000), (128, 70), (128, 9000)])
def test_scores_of_minus_infinity(idxc, H, n, four):
    """They have no weight; a token all of whose scores are -inf is as one that sees nothing, in a sequence that is cut as in one that is not."""
    g = gen(H + n)
    kv = cache_rows(2 * n, four, g)
    low = torch.zeros(2 * n, dtype=torch.bool)
    low[:n:3] = True
    low[n - 200 if n > 200 else 0:n] = True              # the first sequence's last rows, a whole tile and more; every row of the second
    low[n:] = True
    if n == 70:
        low[:64] = False
    rows = torch.nonzero(low)[:, 0]
    if four:
        kv[rows, 288 + 2 * 7], kv[rows, 288 + 2 * 7 + 1] = 0x80, 0xFF
    else:
        kv[rows, 512 + 7] = float("-inf")
    q = bf16_rows(2 * H, g, 0.5).view(2, 1, H, 576)
    q[..., 512 + 7] = 0.5
    out, lse = idxc.latent_attention(q.to(DEV), kv.to(DEV), torch.tensor([0, n], device=DEV), torch.tensor([n, n], dtype=torch.int32, device=DEV), n, 512, 1 / 24)
    assert bool((out[1] == 0).all()) and bool(torch.isneginf(lse[1]).all())
    seen = torch.nonzero(~low[:n])[:, 0]
    check_attention(out[0, 0], lse[0, 0], *oracle_sequence(q[0], kv[seen], 0, len(seen), 1, 1 / 24)[:4])
    if four:
        topk = torch.stack([torch.randperm(n, generator=g), torch.randperm(n, generator=g)])[:, :min(n, 2048)].to(torch.int32)
        out, lse = idxc.sparse_attention_q4(q[:, 0].contiguous().to(DEV), kv.to(DEV), topk.to(DEV), 512, 1 / 24, kv_base=torch.tensor([0, n], device=DEV))
        assert bool((out[1] == 0).all()) and bool(torch.isneginf(lse[1]).all())
        pick = topk[0].long()
        pick = pick[~low[pick]]
        check_attention(out[0], lse[0], *oracle_sequence(q[:1, 0], kv[pick], 0, len(pick), 1, 1 / 24)[:4])
