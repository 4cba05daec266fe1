"""No GPU: the latent-cache calls refuse bad arguments before any device work, and the binding refuses bad tensors."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def idxc():
    from paper_2603_12201_b200 import build
    build.build()
    from paper_2603_12201_b200 import binding
    return binding


P = ctypes.c_void_p(4096)        # never dereferenced
ODD = ctypes.c_void_p(4100)
F = ctypes.c_float


def test_quantize_refusals(idxc):
    L = idxc.lib()
    bad, ok = idxc.ERR_INVALID_ARG, idxc.OK
    for f in (L.idxc_quantize_q4,):
        assert f(P, -1, P, 8, None, None) == bad
        assert f(P, 9, P, 8, None, None) == bad                 # more rows than the cache holds
        assert f(None, 1, P, 8, None, None) == bad
        assert f(P, 1, None, 8, None, None) == bad
        assert f(ODD, 1, P, 8, None, None) == bad
        assert f(P, 1, ODD, 8, None, None) == bad
        assert f(P, 1, P, 8, ODD, None) == bad
        assert f(P, 0, P, 8, None, None) == ok
    g = L.idxc_dequantize_q4
    assert g(P, 8, None, -1, P, None) == bad
    assert g(P, -1, None, 1, P, None) == bad
    assert g(None, 8, None, 1, P, None) == bad
    assert g(P, 8, None, 1, ODD, None) == bad
    assert g(P, 8, ODD, 1, P, None) == bad
    assert g(P, 8, None, 0, P, None) == ok


def dense(L, q=P, kv=P, fmt=0, n_kv=100, base=None, lens=P, B=2, n_step=1, max_len=10, H=16, d=576, dv=512, out=P, lse=None, ws=P, nb=1 << 30):
    return L.idxc_latent_attention(q, kv, fmt, n_kv, base, lens, B, n_step, max_len, H, d, dv, F(1.0), out, lse, ws, nb, None)


def test_dense_refusals(idxc):
    L, bad = idxc.lib(), idxc.ERR_INVALID_ARG
    for kw in (dict(B=-1), dict(n_step=0), dict(H=0), dict(n_kv=-1), dict(max_len=-1), dict(max_len=2 ** 30 + 1), dict(n_kv=2 ** 31), dict(fmt=2), dict(dv=0),
               dict(dv=577), dict(q=None), dict(q=ODD), dict(kv=None), dict(kv=ODD), dict(lens=None), dict(lens=ctypes.c_void_p(4098)), dict(base=ODD), dict(out=None),
               dict(out=ODD), dict(lse=ctypes.c_void_p(4098)), dict(B=2 ** 26, H=128, n_step=1), dict(B=2 ** 31), dict(n_step=2 ** 30, H=128)):
        assert dense(L, **kw) == bad, kw
    for kw in (dict(H=129), dict(d=512), dict(dv=256)):
        assert dense(L, **kw) == idxc.ERR_UNSUPPORTED, kw
    need = idxc.latent_attention_workspace_bytes(2, 1, 10, 16)
    for kw in (dict(ws=None), dict(nb=need - 1), dict(ws=ctypes.c_void_p(4096 + 64))):
        assert dense(L, **kw) == idxc.ERR_WORKSPACE, kw
    assert dense(L, B=0) == idxc.OK
    assert idxc.latent_attention_workspace_bytes(0, 1, 10, 16) == 0


def test_sparse_refusals(idxc):
    L, bad = idxc.lib(), idxc.ERR_INVALID_ARG

    def call(q=P, kv=P, topk=P, base=None, n_q=2, n_kv=10, H=16, d=576, dv=512, k=4, out=P, ws=P, nb=1 << 30):
        return L.idxc_sparse_attention_q4(q, kv, topk, base, n_q, n_kv, H, d, dv, k, F(1.0), out, None, ws, nb, None)

    for kw in (dict(topk=None), dict(k=0), dict(n_q=-1), dict(q=ODD), dict(topk=ctypes.c_void_p(4098)), dict(out=ODD), dict(dv=600)):
        assert call(**kw) == bad, kw
    assert call(H=200) == idxc.ERR_UNSUPPORTED
    assert call(ws=None) == idxc.ERR_WORKSPACE
    assert call(n_q=0) == idxc.OK


def test_weights_refusals(idxc):
    L, bad = idxc.lib(), idxc.ERR_INVALID_ARG

    def call(fmt=0, lens=P, topk=None, k=0, B=2, n_step=1, max_len=10, H=16, d=576, lse=P, beta=1.0, acc=P, ld=10, q=P):
        return L.idxc_attention_weights(q, P, fmt, 100, None, lens, topk, k, B, n_step, max_len, H, d, F(1.0), lse, F(beta), acc, ld, None)

    for kw in (dict(fmt=3), dict(ld=9), dict(lse=None), dict(acc=None), dict(lens=None), dict(q=None), dict(ld=-1), dict(topk=P, k=4),
               dict(topk=P, k=4, lens=None, n_step=2), dict(topk=P, k=4, lens=None, beta=0.5), dict(topk=P, k=0, lens=None)):
        assert call(**kw) == bad, kw
    assert call(d=100) == idxc.ERR_UNSUPPORTED
    assert call(B=0) == idxc.OK


def test_eviction_refusals(idxc):
    L, bad = idxc.lib(), idxc.ERR_INVALID_ARG
    Q = ctypes.c_void_p(8192)

    def sel(acc=P, ld=10, lens=P, B=2, budget=4, recent=1, keep=P, new=Q):
        return L.idxc_evict_select(acc, ld, lens, B, budget, recent, keep, new, None)

    for kw in (dict(acc=None), dict(ld=-1), dict(lens=None), dict(B=-1), dict(B=65536), dict(budget=0), dict(recent=5), dict(recent=-1), dict(keep=None), dict(new=None),
               dict(new=P)):
        assert sel(**kw) == bad, kw
    assert sel(B=0) == idxc.OK

    far = ctypes.c_void_p(1 << 30)

    def comp(src=P, dst=far, rb=16, sr=10, dr=10, sb=P, db=Q, keep=P, ldk=4, n=P, B=2):
        return L.idxc_compact_rows(src, dst, rb, sr, dr, sb, db, keep, ldk, n, B, None)

    for kw in (dict(rb=0), dict(rb=6), dict(sr=-1), dict(dr=-1), dict(B=-1), dict(src=None), dict(dst=None), dict(sb=None), dict(db=None), dict(keep=None), dict(n=None),
               dict(dst=P), dict(dst=P, db=P, dr=9), dict(dst=ctypes.c_void_p(4096 + 144)), dict(src=ctypes.c_void_p((1 << 30) + 16))):
        assert comp(**kw) == bad, kw
    assert comp(B=0) == idxc.OK


def test_binding_takes_cuda_tensors_only(idxc):
    q = torch.zeros((1, 1, 4, 576), dtype=torch.bfloat16)
    kv = torch.zeros((4, 576), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        idxc.latent_attention(q, kv, None, torch.ones(1, dtype=torch.int32), 4, 512, 1.0)
    with pytest.raises(ValueError):
        idxc.quantize_q4(kv, torch.zeros((4, 416), dtype=torch.uint8))
    with pytest.raises(ValueError):
        idxc.evict_select(torch.zeros(1, 4), torch.ones(1, dtype=torch.int32), 2, 1, torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32))


def test_compaction_refuses_more_entries_than_it_can_count(idxc):
    """Above 2^30 the row counter of the kernel in place would wrap; the same bound as the choice's budget."""
    L, far = idxc.lib(), ctypes.c_void_p(1 << 30)
    for dst, base in ((P, P), (far, P)):
        for ld_keep in (2 ** 30 + 1, 2 ** 31 - 1):
            assert L.idxc_compact_rows(P, dst, 4, 2 ** 32, 2 ** 32 if dst is P else 8, P, base, P, ld_keep, P, 1, None) == idxc.ERR_INVALID_ARG


def test_sizes_beyond_the_documented_limits(idxc):
    L, bad, Q, far = idxc.lib(), idxc.ERR_INVALID_ARG, ctypes.c_void_p(8192), ctypes.c_void_p(1 << 52)
    assert L.idxc_quantize_q4(P, 2 ** 31 + 1, P, 2 ** 40, None, None) == bad
    assert L.idxc_dequantize_q4(P, 2 ** 40, None, 2 ** 31 + 1, P, None) == bad
    for ld, B, budget in ((2 ** 30 + 1, 1, 4), (10, 65536, 4), (10, 1, 2 ** 30 + 1)):
        assert L.idxc_evict_select(P, ld, P, B, budget, 0, P, Q, None) == bad
    for rb, sr, dr, B in ((2 ** 20 + 4, 8, 8, 1), (16, 8, 8, 65536), (16, 2 ** 40 + 1, 8, 1), (16, 8, 2 ** 40 + 1, 1)):
        assert L.idxc_compact_rows(P, far, rb, sr, dr, P, Q, P, 4, P, B, None) == bad
