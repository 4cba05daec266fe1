"""No GPU: the paged-cache calls refuse bad arguments before any device work, and the binding refuses bad tensors."""
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
Q, R = ctypes.c_void_p(8192), ctypes.c_void_p(12288)
ODD, ODD4 = ctypes.c_void_p(4098), ctypes.c_void_p(4100)
F = ctypes.c_float
BIG = 2 ** 31


def test_tables(idxc):
    L, bad = idxc.lib(), idxc.ERR_INVALID_ARG

    def call(table=P, ld=4, lens=P, new=Q, B=2, page=16, free=P, cap=8, count=P, begin=P, start=R, slots=P, n=4, seq=None):
        return L.idxc_page_tables(table, ld, lens, new, B, page, free, cap, count, begin, start, slots, n, seq, None)

    for kw in (dict(table=None), dict(table=ODD), dict(ld=-1), dict(ld=BIG), dict(lens=None), dict(lens=Q), dict(lens=R), dict(new=R), dict(new=None), dict(B=-1), dict(B=65536),
               dict(B=65535, ld=2 ** 16), dict(page=0), dict(page=8), dict(page=24), dict(page=1040), dict(page=-16), dict(free=None), dict(cap=-1), dict(cap=BIG), dict(count=None),
               dict(begin=None), dict(begin=ODD), dict(start=None), dict(slots=None), dict(slots=ODD4), dict(n=-1), dict(n=BIG), dict(seq=ODD)):
        assert call(**kw) == bad, kw

    def release(table=P, ld=4, lens=P, keep=None, B=2, page=16, free=P, cap=8, count=P):
        return L.idxc_page_release(table, ld, lens, keep, B, page, free, cap, count, None)

    for kw in (dict(table=None), dict(ld=-1), dict(lens=None), dict(keep=P), dict(keep=ODD), dict(B=-1), dict(B=65536), dict(page=20), dict(free=None), dict(cap=-1), dict(count=None)):
        assert release(**kw) == bad, kw
    assert release(B=0) == idxc.OK

    def rows(table=P, ld=4, B=2, seq=None, pos=P, n=2, k=4, page=16, out=P):
        return L.idxc_page_rows(table, ld, B, seq, pos, n, k, page, out, None)

    for kw in (dict(table=None), dict(ld=-1), dict(B=-1), dict(n=3), dict(n=-1), dict(n=BIG, seq=P), dict(k=-1), dict(page=1), dict(pos=None), dict(pos=ODD), dict(out=None),
               dict(out=ODD), dict(seq=ODD)):
        assert rows(**kw) == bad, kw
    assert rows(n=0) == idxc.OK and rows(k=0) == idxc.OK


def cache(idxc, **kw):
    f = dict(k=4096, v=4096, k_scale=None, v_scale=None, bounds=None, n_pages=10, page_stride=16 * 2 * 64, token_stride=128, head_stride=64, page_size=16, H_kv=2, d=64, dtype=0)
    f.update(kw)
    return ctypes.byref(idxc._PagedCacheStruct(**f))


BAD_CACHES = [dict(k=None), dict(v=None), dict(k=4104), dict(v=4104), dict(bounds=4104), dict(n_pages=-1), dict(n_pages=2 ** 27), dict(page_stride=0), dict(token_stride=4),
              dict(head_stride=68), dict(page_stride=2 ** 38), dict(token_stride=-128), dict(page_size=0), dict(page_size=40), dict(page_size=2048), dict(H_kv=0), dict(H_kv=1025), dict(d=0),
              dict(dtype=2), dict(dtype=1), dict(dtype=1, k_scale=4096), dict(dtype=1, k_scale=4096, v_scale=4100), dict(dtype=1, k_scale=4096, v_scale=4096, token_stride=136)]


def test_caches(idxc):
    L, bad = idxc.lib(), idxc.ERR_INVALID_ARG
    for kw in BAD_CACHES:
        c = cache(idxc, **kw)
        assert L.idxc_paged_append(c, P, 128, P, 128, P, 1, None) == bad, kw
        assert L.idxc_paged_gather(c, P, 1, P, P, None) == bad, kw
        assert attend(L, c) == bad, kw
    assert L.idxc_paged_append(None, P, 128, P, 128, P, 1, None) == bad and attend(L, None) == bad
    for d in (32, 96, 256):
        assert attend(L, cache(idxc, d=d)) == idxc.ERR_UNSUPPORTED


def test_append_and_gather(idxc):
    L, bad, c = idxc.lib(), idxc.ERR_INVALID_ARG, cache(idxc)
    for kw in (dict(k=None), dict(v=None), dict(k=ODD), dict(ks=120), dict(vs=120), dict(ks=132), dict(vs=132), dict(slots=None), dict(slots=ODD4), dict(n=-1), dict(n=BIG)):
        a = dict(k=P, ks=128, v=P, vs=128, slots=P, n=2)
        a.update(kw)
        assert L.idxc_paged_append(c, a["k"], a["ks"], a["v"], a["vs"], a["slots"], a["n"], None) == bad, kw
    assert L.idxc_paged_append(c, None, 128, None, 128, None, 0, None) == idxc.OK
    assert L.idxc_paged_append(cache(idxc, n_pages=0, k=None, v=None), P, 128, P, 128, P, 4, None) == idxc.OK          # nowhere to write
    for a in ((None, 2, P, P), (P, -1, P, P), (P, BIG, P, P), (P, 2, None, P), (P, 2, P, ODD), (ODD4, 2, P, P)):
        assert L.idxc_paged_gather(c, *a, None) == bad, a
    assert L.idxc_paged_gather(c, None, 0, None, None, None) == idxc.OK


def attend(L, c, q=P, qs=512, table=P, ld=8, lens=P, B=2, n_step=1, max_len=100, H=8, pages=None, n_sel=0, scale=1.0, out=P, lse=None, ws=P, nb=1 << 40):
    return L.idxc_paged_attention(c, q, qs, table, ld, lens, B, n_step, max_len, H, pages, n_sel, F(scale), out, lse, ws, nb, None)


def test_attention(idxc):
    L, bad, c = idxc.lib(), idxc.ERR_INVALID_ARG, cache(idxc)
    for kw in (dict(q=None), dict(q=ODD), dict(qs=504), dict(qs=516), dict(table=None), dict(ld=-1), dict(lens=None), dict(lens=ODD), dict(B=-1), dict(B=65536), dict(n_step=0),
               dict(n_step=1025), dict(max_len=-1), dict(max_len=129), dict(max_len=2 ** 30 + 1, ld=2 ** 27), dict(H=0), dict(H=7), dict(H=1), dict(H=258, qs=258 * 64),
               dict(pages=P, n_sel=0), dict(pages=ODD, n_sel=2), dict(out=None), dict(out=ODD), dict(lse=ODD), dict(B=60000, n_step=1024, H=64, qs=64 * 64)):
        assert attend(L, c, **kw) == bad, kw
    need = idxc.paged_attention_workspace_bytes(1, 8, 2, 64)
    for kw in (dict(ws=None), dict(nb=need - 1), dict(ws=ctypes.c_void_p(4096 + 64))):
        assert attend(L, c, **kw) == idxc.ERR_WORKSPACE, kw
    assert attend(L, c, B=0) == idxc.OK
    for a in ((0, 8, 2, 64), (1, 7, 2, 64), (1, 8, 0, 64), (1, 8, 2, 96), (1, 1024, 2, 64), (1025, 8, 2, 64)):
        assert idxc.paged_attention_workspace_bytes(*a) == 0


def test_scores(idxc):
    L, bad = idxc.lib(), idxc.ERR_INVALID_ARG

    def call(bounds=P, n=10, page=16, H_kv=2, d=64, q=P, qs=512, table=P, ld=8, lens=P, B=2, n_step=1, H=8, first=1, last=1, scale=1.0, scores=P, lds=8, out=Q):
        return L.idxc_page_scores(bounds, n, page, H_kv, d, q, qs, table, ld, lens, B, n_step, H, first, last, F(scale), scores, lds, out, None)

    for kw in (dict(bounds=None), dict(bounds=ODD4), dict(n=-1), dict(n=BIG), dict(page=8), dict(H_kv=0), dict(H_kv=1025), dict(d=0), dict(q=None), dict(q=ODD), dict(qs=504), dict(qs=516),
               dict(table=None), dict(ld=9), dict(ld=-1), dict(lens=None), dict(B=-1), dict(B=65536), dict(n_step=0), dict(n_step=1025), dict(H=7), dict(H=1), dict(first=-1),
               dict(last=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(scores=None), dict(scores=ODD), dict(out=None), dict(out=P)):
        assert call(**kw) == bad, kw
    assert call(d=96) == idxc.ERR_UNSUPPORTED
    assert call(B=0) == idxc.OK


def test_binding_takes_cuda_tensors_only(idxc):
    z = torch.zeros
    i32 = torch.int32
    with pytest.raises(ValueError):
        idxc.PagedCache(z((4, 16, 2, 64), dtype=torch.bfloat16), z((4, 16, 2, 64), dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        idxc.page_tables(z((1, 2), dtype=i32), z(1, dtype=i32), z(1, dtype=i32), z(4, dtype=i32), z(1, dtype=i32), 16, z(2, dtype=torch.int64), z(2, dtype=i32), z(1, dtype=i32))
    with pytest.raises(ValueError):
        idxc.page_rows(z((1, 2), dtype=i32), z((1, 2), dtype=i32), 16, z((1, 2), dtype=i32))
    with pytest.raises(ValueError):
        idxc.page_release(z((1, 2), dtype=i32), z(1, dtype=i32), None, z(4, dtype=i32), z(1, dtype=i32), 16)
    with pytest.raises(ValueError):
        idxc.page_scores(z((4, 2, 2, 64), dtype=torch.bfloat16), z((1, 1, 4, 64), dtype=torch.bfloat16), z((1, 2), dtype=i32), z(1, dtype=i32), 16, 1.0, z((2, 4)), z(2, dtype=i32))


def test_token_strides(idxc):
    """The one stride of a tensor's tokens, or a refusal (the device check is passed by the index -1 of a CPU tensor)."""
    t = torch.zeros((3, 2, 10, 64), dtype=torch.bfloat16)
    assert idxc._token_stride(t, "q", 10, 64, -1) == 640
    assert idxc._token_stride(t[:, :, 2:8], "q", 6, 64, -1) == 640
    assert idxc._token_stride(t[:, :1, :4], "q", 4, 64, -1) == 1280
    assert idxc._token_stride(t[:1, :1, :4], "q", 4, 64, -1) == 256
    assert idxc._token_stride(t[:, 0, 4:8], "q", 4, 64, -1) == 1280
    assert idxc._token_stride(t[:, :, :, None, :].squeeze(3)[:, :, 3:4], "q", 1, 64, -1) == 640
    for bad in (t.permute(0, 2, 1, 3), torch.zeros((3, 4, 10, 64), dtype=torch.bfloat16)[:, ::3, :5], t[:, :, :, ::2], t[:, :, ::2]):
        with pytest.raises(ValueError):
            idxc._token_stride(bad, "q", bad.shape[-2], bad.shape[-1], -1)
    with pytest.raises(ValueError):
        idxc._token_stride(t, "q", 9, 64, -1)
    with pytest.raises(TypeError):
        idxc._token_stride(t.float(), "q", 10, 64, -1)
