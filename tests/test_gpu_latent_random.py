"""GPU: seeded random cases of the latent-cache operators (ragged lengths, head counts, new tokens, bases, both row formats, empty
sequences, lengths around tile borders), with the bounds of tests/latent_util.py; and what the binding refuses."""
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


def draw_lens(rng, B):
    around = [0, 1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 192, 193, 255, 256, 257]
    return [int(rng.choice(around)) if rng.random() < 0.5 else int(np.exp(rng.uniform(0, np.log(1500)))) for _ in range(B)]


@pytest.mark.parametrize("seed", range(40))
def test_random_dense_and_weights(idxc, seed):
    rng = np.random.default_rng(1000 + seed)
    g = torch.Generator()
    g.manual_seed(seed)
    four = bool(rng.integers(2))
    H = int(rng.choice([1, 3, 8, 16, 17, 40, 63, 64, 65, 96, 127, 128]))
    n_step = int(rng.choice([1, 1, 1, 2, 3, 5]))
    B = int(rng.integers(1, max(2, 1200 // (H * n_step)) + 1)) if rng.random() < 0.7 else 1
    B = min(B, 150)
    lens = draw_lens(rng, B)
    scale = float(rng.choice([1 / 24, 0.2, -0.1]))
    # sequences anywhere in the cache, overlapping or partly outside it
    n_kv = int(rng.integers(1, 4000))
    base = rng.integers(-40, n_kv + 40, B)
    kv = cache_rows(n_kv, four, g).to(DEV)
    q = bf16_rows(B * n_step * H, g, float(rng.choice([0.3, 1.0, 3.0]))).reshape(B, n_step, H, 576).to(DEV)
    lens_t, base_t = torch.tensor(lens, dtype=torch.int32, device=DEV), torch.tensor(base, dtype=torch.int64, device=DEV)
    max_len = max(lens) + int(rng.integers(0, 3))
    out, lse = idxc.latent_attention(q, kv, base_t, lens_t, max_len, 512, scale)
    idxc.poll_device_status()
    ld = max(max_len, 1) + 3
    start = torch.rand((B, ld), generator=g)
    acc, beta = start.clone().to(DEV), float(rng.choice([0.0, 0.5, 1.0]))
    idxc.attention_weights(q, kv, lse, acc, scale, kv_base=base_t, lens=lens_t, max_len=max_len, beta=beta)
    idxc.poll_device_status()
    got = acc.double().cpu().numpy()
    for b in rng.permutation(B)[:12]:
        o, l, spread, reach, p = oracle_sequence(q[b], kv, int(base[b]), lens[b], n_step, scale)
        check_attention(out[b].reshape(-1, 512), lse[b].reshape(-1), o, l, spread, reach, f"sequence {b}")
        n = lens[b]
        want = beta * start[b, :n].double().numpy() + p.sum(axis=0)
        # the probabilities use the GPU's own lse, itself within score_error + 2^-20 (1 + |lse|)
        slack = np.where(np.isfinite(l), 3 * score_error(reach) + 2.0 ** -17 * (1 + np.abs(np.where(np.isfinite(l), l, 0))), 0.0)
        assert np.all(np.abs(got[b, :n] - want) <= (p * slack[:, None]).sum(axis=0) + 2.0 ** -20 * want + 1e-30), f"weights of sequence {b}"
        assert np.array_equal(got[b, n:].astype(np.float32), start[b, n:].numpy())


@pytest.mark.parametrize("seed", range(24))
def test_random_sparse(idxc, seed):
    rng = np.random.default_rng(2000 + seed)
    g = torch.Generator()
    g.manual_seed(seed)
    H = int(rng.choice([1, 5, 16, 33, 64, 65, 100, 128]))
    n_q = int(rng.integers(1, 200 if rng.random() < 0.5 else 8))
    k_top = int(rng.choice([1, 31, 32, 33, 63, 64, 65, 100, 128, 300, 1000]))
    n_kv = int(rng.integers(1, 3000))
    kv = q4_rows(n_kv, g).to(DEV)
    q = bf16_rows(n_q * H, g, 1.5).reshape(n_q, H, 576).to(DEV)
    topk = torch.randint(-5 if rng.random() < 0.7 else 0, n_kv + 20, (n_q, k_top), generator=g, dtype=torch.int32)
    cut = torch.randint(0, k_top + 1, (n_q, 1), generator=g)
    topk[torch.arange(k_top)[None, :] >= cut] = -1                       # rows end anywhere, some hold nothing
    base = torch.randint(-30, 30, (n_q,), generator=g) if rng.random() < 0.5 else None
    out, lse = idxc.sparse_attention_q4(q, kv, topk.to(DEV), 512, 1 / 24, kv_base=None if base is None else base.to(DEV))
    idxc.poll_device_status()
    raw, t = stored(kv), topk.numpy().astype(np.int64)
    for i in rng.permutation(n_q)[:20]:
        pick = t[i][t[i] >= 0] + (0 if base is None else int(base[i]))
        pick = pick[(pick >= 0) & (pick < n_kv)]
        o, l, spread, reach, _ = oracle.attention(bits(q[i]), raw[pick], 1 / 24, np.full(H, len(pick)))
        check_attention(out[i], lse[i], o, l, spread, reach, f"query {i}")


def test_binding_refuses(idxc):
    q = torch.zeros((2, 1, 4, 576), dtype=torch.bfloat16, device=DEV)
    kv = torch.zeros((10, 576), dtype=torch.bfloat16, device=DEV)
    lens = torch.ones(2, dtype=torch.int32, device=DEV)
    ok = dict(q=q, kv=kv, kv_base=None, lens=lens, max_len=10, d_v=512, scale=1.0)
    idxc.latent_attention(**ok)
    for kw, err in ((dict(kv=kv[:, :512].contiguous()), ValueError), (dict(kv=kv.float()), ValueError), (dict(q=q.float()), TypeError), (dict(q=q[0]), ValueError),
                    (dict(lens=lens.long()), TypeError), (dict(lens=lens[:1]), ValueError), (dict(kv_base=lens), TypeError), (dict(lens=lens.cpu()), ValueError),
                    (dict(q=q.expand(2, 3, 4, 576)), ValueError), (dict(d_v=256), idxc.IdxcError), (dict(max_len=-1), idxc.IdxcError),
                    (dict(out=torch.zeros((2, 1, 4, 256), dtype=torch.bfloat16, device=DEV)), ValueError),
                    (dict(workspace=torch.zeros(16, dtype=torch.uint8, device=DEV)), idxc.IdxcError)):
        with pytest.raises(err):
            idxc.latent_attention(**{**ok, **kw})
    four = torch.zeros((10, 416), dtype=torch.uint8, device=DEV)
    with pytest.raises(ValueError):
        idxc.sparse_attention_q4(q[:, 0], kv, torch.zeros((2, 3), dtype=torch.int32, device=DEV), 512, 1.0)
    with pytest.raises(idxc.IdxcError):                                 # a view that starts off a 32-byte border
        idxc.dequantize_q4(torch.zeros(417 * 16, dtype=torch.uint8, device=DEV)[16:16 + 4160].view(10, 416), kv)
    with pytest.raises(ValueError):
        idxc.quantize_q4(kv, four[:5], dst_rows=torch.zeros(9, dtype=torch.int64, device=DEV))
    with pytest.raises(idxc.IdxcError):
        idxc.quantize_q4(kv, four[:5])
    acc = torch.zeros((2, 9), device=DEV)
    lse = torch.zeros((2, 1, 4), device=DEV)
    for kw in (dict(), dict(lens=lens), dict(lens=lens, max_len=9, topk=torch.zeros((2, 3), dtype=torch.int32, device=DEV))):
        with pytest.raises(ValueError):
            idxc.attention_weights(q, kv, lse, acc, 1.0, **kw)
    with pytest.raises(idxc.IdxcError):
        idxc.attention_weights(q, kv, lse, acc, 1.0, lens=lens, max_len=10)
    keep, new = torch.zeros((2, 3), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    with pytest.raises(idxc.IdxcError):
        idxc.evict_select(acc, lens, 3, 4, keep, new)
    with pytest.raises(idxc.IdxcError):
        idxc.evict_select(acc, new, 3, 1, keep, new)
    b = torch.zeros(2, dtype=torch.int64, device=DEV)
    with pytest.raises(idxc.IdxcError):                                 # the buffers overlap
        idxc.compact_rows(kv[:8], kv[2:], keep, new, b)
    with pytest.raises(idxc.IdxcError):                                 # in place, but to other places
        idxc.compact_rows(kv, kv, keep, new, b, b.clone())
    with pytest.raises(idxc.IdxcError):                                 # rows of 2 bytes
        idxc.compact_rows(kv.view(-1), torch.zeros_like(kv).view(-1), keep, new, b)


def test_not_a_number_in_one_group_stays_there(idxc):
    """Inputs are assumed finite; one that is not spoils its own group of 32 columns and nothing else."""
    g = torch.Generator()
    g.manual_seed(1)
    x = bf16_rows(3, g)
    want = oracle.quantize_rows(x.double().numpy())
    x[1, 40], x[1, 70] = float("nan"), float("inf")
    cache = torch.empty((3, 416), dtype=torch.uint8, device=DEV)
    idxc.quantize_q4(x.to(DEV), cache)
    got = cache.cpu().numpy()
    values = oracle.row_values(got)
    assert np.all(np.isfinite(values[:, :512]))
    same = np.ones((3, 416), dtype=bool)
    same[1, 16:48] = False                       # codes of columns 32..95
    same[1, 256 + 2:256 + 6] = False             # and their scales
    assert np.array_equal(got[same], want[same])
