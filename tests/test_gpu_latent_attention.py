"""GPU: dense attention over latent rows (bf16 and 4 bits), sparse attention over 4-bit rows, and the head-summed weights,
against the float64 oracle with bounds from the arithmetic (tests/latent_util.py)."""
import numpy as np
import pytest
import torch

from oracle import latent as oracle
from tests.latent_util import bf16_rows, bits, cache_rows, check_attention, oracle_sequence, q4_rows, score_error, stored

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


def poisoned(n, four):
    """Rows that give NaN in every column wherever they are read."""
    if not four:
        return torch.full((n, 576), float("nan"), dtype=torch.bfloat16)
    t = torch.full((n, 416), 255, dtype=torch.uint8)
    return t


def batch(lens, four, g, gap=3):
    """Sequences one behind the other, rows of NaN between them and at both ends."""
    parts, base, at = [], [], 0
    for n in lens:
        parts.append(poisoned(gap, four))
        at += gap
        base.append(at)
        parts.append(cache_rows(n, four, g))
        at += n
    parts.append(poisoned(gap, four))
    return torch.cat(parts).to(DEV), torch.tensor(base, dtype=torch.int64, device=DEV)


def run_dense(idxc, lens, H, n_step, four, seed=0, gain=1.5, scale=1 / 24, max_len=None):
    g = gen(seed)
    kv, base = batch(lens, four, g)
    B = len(lens)
    q = bf16_rows(B * n_step * H, g, gain).reshape(B, n_step, H, 576).to(DEV)
    lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)
    out, lse = idxc.latent_attention(q, kv, base, lens_t, max(lens) if max_len is None else max_len, 512, scale)
    idxc.poll_device_status()
    for b, n in enumerate(lens):
        o, l, spread, reach, _ = oracle_sequence(q[b], kv, int(base[b]), n, n_step, scale)
        check_attention(out[b].reshape(-1, 512), lse[b].reshape(-1), o, l, spread, reach, f"sequence {b} of {n}")
    return q, kv, base, lens_t, out, lse


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("lens,H,n_step", [
    ([1], 1, 1), ([1], 128, 1), ([2, 1, 3], 5, 3), ([0], 16, 1), ([0, 7, 0, 64], 128, 1), ([63, 64, 65], 64, 1), ([127, 128, 129, 1], 100, 1),
    ([31, 33, 95, 97], 16, 4), ([200], 128, 2), ([150, 3], 65, 2), ([257, 1025], 128, 1), ([777], 128, 1), ([2049, 100], 16, 1), ([5, 500], 33, 8)])
def test_dense_matches_the_oracle(idxc, lens, H, n_step, four):
    run_dense(idxc, lens, H, n_step, four, seed=sum(lens) + H)


@pytest.mark.parametrize("four", [False, True])
def test_dense_long_ragged_batch(idxc, four):
    run_dense(idxc, [5000, 17, 9000, 1234, 4096, 1, 0, 3333], 16, 1, four, seed=3)


@pytest.mark.parametrize("four", [False, True])
def test_dense_many_short_sequences(idxc, four):
    """More sequences than thread blocks, most of them of one tile or less."""
    rng = np.random.default_rng(4)
    run_dense(idxc, rng.integers(0, 130, 333).tolist(), 8, 1, four, seed=4)


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("gain,scale", [(30.0, 1 / 24), (1e-3, 1 / 24), (1.5, -1 / 24), (1.5, 0.0), (3.0, 1.0)])
def test_dense_peaked_flat_and_negative_scales(idxc, gain, scale, four):
    run_dense(idxc, [300, 1000], 32, 1, four, seed=5, gain=gain, scale=scale)


@pytest.mark.parametrize("four", [False, True])
def test_scores_that_grow_along_the_sequence(idxc, four):
    """The running maximum moves at every tile, by a lot: rows grow with their position."""
    g = gen(6)
    n, H = 900, 128
    kv = bf16_rows(n, g)
    kv[:, :512] = (kv[:, :512].float() * torch.linspace(0.1, 8, n)[:, None]).to(torch.bfloat16)
    kv = kv.to(DEV)
    if four:
        store = torch.empty((n, 416), dtype=torch.uint8, device=DEV)
        idxc.quantize_q4(kv, store)
        kv = store
    q = bf16_rows(H, g, 2.0).reshape(1, 1, H, 576).to(DEV)
    out, lse = idxc.latent_attention(q, kv, None, torch.tensor([n], dtype=torch.int32, device=DEV), n, 512, 1 / 24)
    o, l, spread, reach, _ = oracle_sequence(q[0], kv, 0, n, 1, 1 / 24)
    check_attention(out[0, 0], lse[0, 0], o, l, spread, reach)


@pytest.mark.parametrize("four", [False, True])
def test_rows_outside_the_cache_take_no_part(idxc, four):
    g = gen(7)
    kv = cache_rows(200, four, g).to(DEV)
    base = torch.tensor([-50, 150, 500, -500], dtype=torch.int64, device=DEV)
    lens = torch.tensor([100, 100, 100, 100], dtype=torch.int32, device=DEV)
    q = bf16_rows(4 * 8, g).reshape(4, 1, 8, 576).to(DEV)
    out, lse = idxc.latent_attention(q, kv, base, lens, 100, 512, 0.05)
    for b in range(4):
        o, l, spread, reach, _ = oracle_sequence(q[b], kv, int(base[b]), 100, 1, 0.05)
        check_attention(out[b, 0], lse[b, 0], o, l, spread, reach, f"sequence {b}")
    # an empty cache
    out, lse = idxc.latent_attention(q, kv[:0], base, lens, 100, 512, 0.05)
    assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())


def test_lengths_are_clamped_to_the_host_bound(idxc):
    g = gen(8)
    kv = bf16_rows(300, g).to(DEV)
    q = bf16_rows(2 * 4, g).reshape(2, 1, 4, 576).to(DEV)
    out, lse = idxc.latent_attention(q, kv, None, torch.tensor([300, -4], dtype=torch.int32, device=DEV), 100, 512, 0.05)
    o, l, spread, reach, _ = oracle_sequence(q[0], kv, 0, 100, 1, 0.05)
    check_attention(out[0, 0], lse[0, 0], o, l, spread, reach)
    assert bool((out[1] == 0).all()) and bool(torch.isneginf(lse[1]).all())
    out, lse = idxc.latent_attention(q, kv, None, torch.tensor([300, 5], dtype=torch.int32, device=DEV), 0, 512, 0.05)
    assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())


def test_no_sequences(idxc):
    q = torch.empty((0, 1, 16, 576), dtype=torch.bfloat16, device=DEV)
    kv = torch.empty((10, 576), dtype=torch.bfloat16, device=DEV)
    out, lse = idxc.latent_attention(q, kv, None, torch.empty(0, dtype=torch.int32, device=DEV), 10, 512, 0.05)
    assert out.shape == (0, 1, 16, 512) and lse.shape == (0, 1, 16)


@pytest.mark.parametrize("four", [False, True])
def test_cache_past_four_gigabytes(idxc, four):
    width = 416 if four else 1152
    n = (1 << 32) // width + 1000
    kv = torch.empty((n, 416), dtype=torch.uint8, device=DEV) if four else torch.empty((n, 576), dtype=torch.bfloat16, device=DEV)
    g = gen(9)
    kv[n - 500:] = cache_rows(500, four, g).to(DEV)
    q = bf16_rows(16, g).reshape(1, 1, 16, 576).to(DEV)
    out, lse = idxc.latent_attention(q, kv, torch.tensor([n - 500], device=DEV), torch.tensor([500], dtype=torch.int32, device=DEV), 500, 512, 0.05)
    o, l, spread, reach, p = oracle.attention(bits(q).reshape(16, 576), stored(kv[n - 500:]), 0.05, np.full(16, 500))
    check_attention(out[0, 0], lse[0, 0], o, l, spread, reach)
    acc = torch.zeros((1, 500), device=DEV)
    idxc.attention_weights(q, kv, lse, acc, 0.05, kv_base=torch.tensor([n - 500], device=DEV), lens=torch.tensor([500], dtype=torch.int32, device=DEV), max_len=500)
    assert np.allclose(acc[0].cpu().numpy(), p.sum(axis=0), rtol=1e-3)


@pytest.mark.parametrize("four", [False, True])
def test_result_is_the_same_every_time(idxc, four):
    q, kv, base, lens, out, lse = run_dense(idxc, [3000, 50, 700], 128, 1, four, seed=10)
    junk = torch.empty(idxc.latent_attention_workspace_bytes(3, 1, 3000, 128), dtype=torch.uint8, device=DEV)
    for fill in (0, 255):
        junk.fill_(fill)
        o2, l2 = idxc.latent_attention(q, kv, base, lens, 3000, 512, 1 / 24, workspace=junk)
        assert torch.equal(out, o2) and torch.equal(lse, l2)


def test_outputs_stay_in_their_rows(idxc):
    g = gen(12)
    kv = bf16_rows(300, g).to(DEV)
    for H, n_step in ((5, 1), (128, 1), (70, 2)):
        q = bf16_rows(2 * n_step * H, g).reshape(2, n_step, H, 576).to(DEV)
        whole = torch.full((2 * n_step * H + 2, 512), 7.0, dtype=torch.bfloat16, device=DEV)
        out = whole[1:-1].view(2, n_step, H, 512)
        idxc.latent_attention(q, kv, None, torch.tensor([300, 0], dtype=torch.int32, device=DEV), 300, 512, 0.05, out=out)
        assert bool((whole[0] == 7).all()) and bool((whole[-1] == 7).all()) and bool((out[1] == 0).all())


# ------------------------------------------------------------------ sparse, 4-bit rows
def check_sparse(idxc, q, kv, topk, base, scale):
    out, lse = idxc.sparse_attention_q4(q, kv, topk, 512, scale, kv_base=base)
    idxc.poll_device_status()
    n_kv = kv.shape[0]
    t = topk.cpu().numpy().astype(np.int64)
    raw = stored(kv)
    for i in range(q.shape[0]):
        pick = t[i][t[i] >= 0] + (int(base[i]) if base is not None else 0)
        pick = pick[(pick >= 0) & (pick < n_kv)]
        o, l, spread, reach, _ = oracle.attention(bits(q[i]), raw[pick], scale, np.full(q.shape[1], len(pick)))
        check_attention(out[i], lse[i], o, l, spread, reach, f"query {i}")
    return out, lse


@pytest.mark.parametrize("n_q,H,k_top,n_kv", [(1, 128, 1, 1), (1, 1, 64, 200), (3, 128, 65, 500), (2, 100, 2048, 2500), (70, 16, 128, 300), (5, 64, 63, 64), (160, 128, 33, 1000)])
def test_sparse_q4_matches_the_oracle(idxc, n_q, H, k_top, n_kv):
    g = gen(n_q + H + k_top)
    kv = q4_rows(n_kv, g).to(DEV)
    q = bf16_rows(n_q * H, g, 1.5).reshape(n_q, H, 576).to(DEV)
    topk = torch.stack([torch.randperm(max(n_kv, k_top), generator=g)[:k_top] for _ in range(n_q)]).to(torch.int32)
    topk[topk >= n_kv] = -1
    check_sparse(idxc, q, kv, topk.to(DEV), None, 1 / 24)


def test_sparse_q4_holes_repeats_bases_and_empty_queries(idxc):
    g = gen(21)
    kv = torch.cat([q4_rows(400, g), poisoned(100, True)]).to(DEV)      # rows 400.. hold NaN and are never named
    q = bf16_rows(6 * 24, g).reshape(6, 24, 576).to(DEV)
    topk = torch.randint(-3, 200, (6, 150), generator=g, dtype=torch.int32)
    topk[0] = -1
    topk[1, :] = -1
    topk[1, 149] = 5                                                    # one entry, the last
    topk[2, :100] = 2 ** 31 - 1
    topk[3] = 17                                                        # the same row 150 times
    base = torch.tensor([0, 100, 200, 37, -20, 200], dtype=torch.int64, device=DEV)
    out, lse = check_sparse(idxc, q, kv, topk.to(DEV), base, 0.06)
    assert bool((out[0] == 0).all()) and bool(torch.isneginf(lse[0]).all())


def test_sparse_q4_agrees_with_the_bf16_path_on_the_same_values(idxc):
    g = gen(22)
    store = q4_rows(3000, g).to(DEV)
    wide = torch.empty((3000, 576), dtype=torch.bfloat16, device=DEV)
    idxc.dequantize_q4(store, wide)
    q = bf16_rows(9 * 128, g, 2.0).reshape(9, 128, 576).to(DEV)
    topk = torch.stack([torch.randperm(3000, generator=g)[:2048] for _ in range(9)]).to(torch.int32).to(DEV)
    a, la = idxc.sparse_attention_q4(q, store, topk, 512, 1 / 24)
    b, lb = idxc.sparse_attention(q, wide, topk, 512, 1 / 24)
    assert torch.allclose(la, lb, atol=1e-4)
    assert (a.float() - b.float()).norm() <= 2.0 ** -7 * b.float().norm()


# ------------------------------------------------------------------ attention weights
def weights_bound(p, reach, rows):
    """Each probability is off by a factor within exp(score error + the 2^-20 of exp2 and of an lse in fp32); up to 2^10 fp32 adds."""
    return (p * (2 * score_error(reach)[:, None] + 2.0 ** -18)).sum(axis=0) + 2.0 ** -20 * p.sum(axis=0) + 1e-30


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("lens,H,n_step", [([1], 1, 1), ([0, 5, 64], 128, 1), ([127, 128, 129], 100, 1), ([300, 2, 1000], 16, 4), ([700], 128, 2), ([65, 90], 33, 8)])
@pytest.mark.parametrize("beta", [0.0, 1.0, 0.5])
def test_weights_match_the_oracle(idxc, lens, H, n_step, four, beta):
    g = gen(sum(lens) + H)
    kv, base = batch(lens, four, g)
    B, ld, scale = len(lens), max(lens) + 5, 1 / 24
    q = bf16_rows(B * n_step * H, g, 1.5).reshape(B, n_step, H, 576).to(DEV)
    lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)
    start = torch.rand((B, ld), generator=g)
    if beta == 0:
        start[:] = float("nan")
    acc = start.clone().to(DEV)
    seq = [oracle_sequence(q[b], kv, int(base[b]), n, n_step, scale) for b, n in enumerate(lens)]
    lse = torch.tensor(np.stack([s[1] for s in seq]), dtype=torch.float32).reshape(B, n_step, H).to(DEV)
    idxc.attention_weights(q, kv, lse, acc, scale, kv_base=base, lens=lens_t, max_len=max(lens), beta=beta)
    idxc.poll_device_status()
    got = acc.double().cpu().numpy()
    for b, n in enumerate(lens):
        _, _, _, reach, p = seq[b]
        old = np.zeros(n) if beta == 0 else beta * start[b, :n].double().numpy()
        want = old + p.sum(axis=0)
        assert np.all(np.abs(got[b, :n] - want) <= weights_bound(p, reach, n_step * H) + 2.0 ** -23 * want), f"sequence {b}"
        tail = start[b, n:].numpy()
        assert np.array_equal(got[b, n:].astype(np.float32), tail, equal_nan=True)


@pytest.mark.parametrize("four", [False, True])
def test_weights_of_a_selection(idxc, four):
    g = gen(31)
    kv = cache_rows(500, four, g).to(DEV)
    B, H, k, ld = 5, 40, 130, 300
    q = bf16_rows(B * H, g).reshape(B, H, 576).to(DEV)
    topk = torch.randint(-2, 320, (B, k), generator=g, dtype=torch.int32)       # repeats, holes, positions at or past ld
    topk[4] = -1
    base = torch.tensor([0, 100, 250, -10, 0], dtype=torch.int64, device=DEV)
    raw, t = stored(kv), topk.numpy().astype(np.int64)
    acc = torch.rand((B, ld), generator=g)
    want, bound, lse = acc.double().numpy().copy(), np.full((B, ld), 1e-30), torch.empty((B, H))
    for b in range(B):
        row = t[b] + int(base[b])
        use = (t[b] >= 0) & (row >= 0) & (row < 500)
        _, l, _, reach, p = oracle.attention(bits(q[b]), raw[row[use]], 0.05, np.full(H, use.sum()))
        lse[b] = torch.from_numpy(l).float()
        for j, s in enumerate(t[b][use]):
            if s < ld:
                want[b, s] += p[:, j].sum()
                bound[b, s] += weights_bound(p[:, j:j + 1], reach, H)[0]
    acc = acc.to(DEV)
    idxc.attention_weights(q, kv, lse.to(DEV), acc, 0.05, kv_base=base, topk=topk.to(DEV))
    idxc.poll_device_status()
    assert np.all(np.abs(acc.double().cpu().numpy() - want) <= bound + 2.0 ** -20 * want)


@pytest.mark.parametrize("four", [False, True])
def test_weights_without_visible_rows(idxc, four):
    """An empty cache, sequences outside it and tokens that see nothing: the old sums are scaled, nothing is added."""
    g = gen(33)
    kv = cache_rows(70, four, g).to(DEV)
    q = bf16_rows(3 * 2 * 5, g).reshape(3, 2, 5, 576).to(DEV)
    lens = torch.tensor([60, 1, 0], dtype=torch.int32, device=DEV)
    base = torch.tensor([-60, 70, 0], device=DEV)
    start = torch.rand((3, 64), generator=g)
    for rows, b in ((kv[:0], None), (kv, base)):
        lse = torch.full((3, 2, 5), float("-inf"), device=DEV)
        acc = start.clone().to(DEV)
        idxc.attention_weights(q, rows, lse, acc, 0.05, kv_base=b, lens=lens, max_len=60, beta=0.25)
        want = start.clone()
        want[0, :60] *= 0.25
        want[1, :1] *= 0.25
        assert torch.equal(acc.cpu(), want)
        lse.fill_(0.0)                                   # a finite lse of tokens whose rows do not exist
        idxc.attention_weights(q, rows, lse, acc, 0.05, kv_base=b, lens=lens, max_len=60)
        assert torch.equal(acc.cpu(), want)


def test_weights_ignore_query_rows_of_the_next_sequence(idxc):
    """The matrix product's padding reads query rows behind the sequence's own; whatever they hold adds nothing."""
    g = gen(34)
    kv = bf16_rows(200, g).to(DEV)
    q = bf16_rows(2 * 5, g).reshape(2, 1, 5, 576)
    q[1] = float("nan")
    q = q.to(DEV)
    lens = torch.tensor([200, 0], dtype=torch.int32, device=DEV)
    out, lse = idxc.latent_attention(q, kv, None, lens, 200, 512, 0.05)
    acc = torch.zeros((2, 200), device=DEV)
    idxc.attention_weights(q, kv, lse, acc, 0.05, lens=lens, max_len=200)
    o, l, spread, reach, p = oracle.attention(bits(q[0, 0]), stored(kv), 0.05, np.full(5, 200))
    check_attention(out[0, 0], lse[0, 0], o, l, spread, reach)
    assert np.allclose(acc[0].cpu().numpy(), p.sum(axis=0), rtol=1e-4)


# ------------------------------------------------------------------ as a serving loop uses them
def test_append_attend_weigh_evict_loop(idxc):
    """Prompt and steps into a 4-bit cache, dense attention, weights, eviction when full; against the same loop in float64."""
    g = gen(41)
    B, H, cap, budget, recent, scale = 3, 16, 160, 96, 16, 1 / 24
    base = torch.arange(B, device=DEV) * cap
    cache = torch.zeros((B * cap, 416), dtype=torch.uint8, device=DEV)
    acc = torch.zeros((B, cap), device=DEV)
    lens = [100, 37, 150]
    mirror = []
    for b, n in enumerate(lens):
        x = bf16_rows(n, g)
        idxc.quantize_q4(x.to(DEV), cache, dst_rows=torch.arange(n, device=DEV) + b * cap)
        mirror.append(oracle.quantize_rows(x.double().numpy()))
    sums = [np.zeros(n) for n in lens]
    lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)
    new_lens, keep = torch.empty_like(lens_t), torch.empty((B, budget), dtype=torch.int32, device=DEV)
    for step in range(14):
        x = bf16_rows(B, g)
        idxc.quantize_q4(x.to(DEV), cache, dst_rows=base + lens_t)
        lens_t += 1
        rows = oracle.quantize_rows(x.double().numpy())
        q = bf16_rows(B * H, g, 2.0).reshape(B, 1, H, 576).to(DEV)
        out, lse = idxc.latent_attention(q, cache, base, lens_t, cap, 512, scale)
        idxc.attention_weights(q, cache, lse, acc, scale, kv_base=base, lens=lens_t, max_len=cap)
        for b in range(B):
            mirror[b] = np.concatenate([mirror[b], rows[b:b + 1]])
            o, l, spread, reach, p = oracle.attention(bits(q[b, 0]), mirror[b], scale, np.full(H, len(mirror[b])))
            check_attention(out[b, 0], lse[b, 0], o, l, spread, reach, f"step {step} sequence {b}")
            sums[b] = np.concatenate([sums[b], [0.0]]) + p.sum(axis=0)
            assert np.allclose(acc[b, :len(sums[b])].cpu().numpy(), sums[b], rtol=1e-4, atol=1e-6)
        if int(lens_t.max()) >= cap - 1:
            before = acc.cpu().numpy()
            idxc.evict_select(acc, lens_t, budget, recent, keep, new_lens)
            idxc.compact_rows(cache, cache, keep, new_lens, base)
            idxc.compact_rows(acc.view(-1), acc.view(-1), keep, new_lens, base)
            for b in range(B):
                k = keep[b, :int(new_lens[b])].cpu().numpy()
                assert np.array_equal(k, oracle.evict(before[b], len(mirror[b]), budget, recent))
                mirror[b], sums[b] = mirror[b][k], sums[b][k]
            lens_t.copy_(new_lens)
            for b in range(B):
                acc[b, int(lens_t[b]):] = 0
                got = cache[b * cap:b * cap + int(lens_t[b])].cpu().numpy()
                assert np.array_equal(got, mirror[b])
    assert int(lens_t.max()) < cap


def test_captured_calls_replay_on_new_data_and_other_streams(idxc):
    g = gen(42)
    kv = q4_rows(5000, g).to(DEV)
    B, H = 4, 128
    q = bf16_rows(B * H, g).reshape(B, 1, H, 576).to(DEV)
    base = torch.tensor([0, 1200, 2400, 3600], device=DEV)
    lens = torch.tensor([1000, 10, 0, 1200], dtype=torch.int32, device=DEV)
    acc = torch.zeros((B, 1200), device=DEV)
    keep, new = torch.empty((B, 300), dtype=torch.int32, device=DEV), torch.empty(B, dtype=torch.int32, device=DEV)

    def step():
        out, lse = idxc.latent_attention(q, kv, base, lens, 1200, 512, 1 / 24)
        idxc.attention_weights(q, kv, lse, acc, 1 / 24, kv_base=base, lens=lens, max_len=1200, beta=0.0)
        idxc.evict_select(acc, lens, 300, 10, keep, new)
        sp, _ = idxc.sparse_attention_q4(q[:, 0], kv, keep, 512, 1 / 24, kv_base=base)
        return out, lse, sp

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    results = []
    for gr in graphs:
        with torch.cuda.graph(gr):
            results.append(step())
    q.copy_(bf16_rows(B * H, g).reshape(B, 1, H, 576))
    lens.copy_(torch.tensor([7, 1200, 64, 0], dtype=torch.int32))
    for gr in graphs:
        gr.replay()
    torch.cuda.synchronize()
    want = step()
    for r in results:
        for a, b in zip(r, want):
            assert torch.equal(a, b)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for _ in range(5):                               # two calls at once, a workspace each
        a = idxc.latent_attention(q, kv, base, lens, 1200, 512, 1 / 24, stream=s1)
        b = idxc.latent_attention(q, kv, base, lens, 1200, 512, 1 / 24, stream=s2)
        outs += [a, b]
    torch.cuda.synchronize()
    for o, l in outs:
        assert torch.equal(o, want[0]) and torch.equal(l, want[1])
