"""The paged-cache calls together, as a serving program makes them: steps of a batch whose requests grow, shrink and end, against keys and values kept
request by request; the same steps captured and replayed; two batches on two streams at once; the latent cache and the indexer's selection over pages."""
import numpy as np
import pytest
import torch

from oracle import paged as oracle
from paper_2603_12201_b200 import binding as idxc
from tests.paged_util import DEV, bf16, check, gen, int32
from tests.util import codes

pytestmark = pytest.mark.gpu


class Server:
    """A program's state: cache, block tables, free pages, and the buffers of one step of up to `tokens` new tokens."""

    def __init__(self, B, P, H, H_kv, d, eight, n_pages, tokens, k_pages, seed=0):
        g = gen(seed)
        shape = (n_pages, P, H_kv, d)
        kind = torch.float8_e4m3fn if eight else torch.bfloat16
        self.k, self.v = [torch.zeros(shape, dtype=torch.uint8 if eight else torch.bfloat16, device=DEV).view(kind) for _ in range(2)]
        scales = [torch.zeros((n_pages, H_kv, P), device=DEV) for _ in range(2)] if eight else [None, None]
        self.bounds = torch.zeros((n_pages, H_kv, 2, d), dtype=torch.bfloat16, device=DEV)
        self.cache = idxc.PagedCache(self.k, self.v, *scales, bounds=self.bounds)
        self.B, self.P, self.H, self.H_kv, self.d, self.k_pages = B, P, H, H_kv, d, k_pages
        self.ld = (n_pages + 3) // 4 * 4
        self.table = torch.full((B, self.ld), -1, dtype=torch.int32, device=DEV)
        self.lens, self.count = int32([0] * B), int32([n_pages])
        self.free = torch.randperm(n_pages, generator=g).to(torch.int32).to(DEV)
        self.slots = torch.empty(tokens, dtype=torch.int64, device=DEV)
        self.begin, self.start = int32([0] * (B + 1)), int32([0] * B)
        self.scores = torch.zeros((B * H_kv, self.ld), device=DEV)
        self.n_pages, self.pages = int32([0] * (B * H_kv)), torch.zeros((B * H_kv, k_pages), dtype=torch.int32, device=DEV)
        self.out, self.sparse = [torch.zeros((B, 1, H, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        self.ws = torch.empty(idxc.paged_attention_workspace_bytes(1, H, H_kv, d), dtype=torch.uint8, device=DEV)

    def step(self, new, qkv, stream=None):
        """new [B] int32 tokens a request, qkv [tokens, H + 2 H_kv, d]: their projections; the last token of every request attends (q of request b: the
        first rows of qkv, for the test's sake)."""
        H, H_kv = self.H, self.H_kv
        idxc.page_tables(self.table, self.lens, new, self.free, self.count, self.P, self.slots, self.begin, self.start, stream=stream)
        idxc.paged_append(self.cache, qkv[:, H:H + H_kv], qkv[:, H + H_kv:], self.slots, stream=stream)
        q = qkv[:self.B, None, :H]
        idxc.page_scores(self.bounds, q, self.table, self.lens, self.P, 0.1, self.scores, self.n_pages, stream=stream)
        idxc.topk_rows(self.scores, self.k_pages, self.pages, lens=self.n_pages, stream=stream)
        _, lse = idxc.paged_attention(self.cache, q, self.table, self.lens, self.ld * self.P, 0.1, out=self.out, workspace=self.ws, stream=stream)
        _, lse_sparse = idxc.paged_attention(self.cache, q, self.table, self.lens, self.ld * self.P, 0.1, pages=self.pages, out=self.sparse, workspace=self.ws,
                                             stream=stream)
        return lse, lse_sparse


def rows64(x, eight):
    """Rows [n, H_kv, d] bf16 as the cache holds them, float64."""
    if not eight:
        return oracle.bf16_rows(codes(x))
    out = np.zeros(x.shape)
    for t in range(x.shape[0]):
        for h in range(x.shape[1]):
            c, s = oracle.quantize_row(codes(x[t, h]))
            out[t, h] = oracle.e4m3_values(c) * np.float64(s)
    return out


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("B,P,H,H_kv,d", [(5, 16, 8, 2, 64), (3, 32, 16, 1, 128), (4, 48, 6, 3, 64)])
def test_steps(eight, B, P, H, H_kv, d):
    rng, g = np.random.default_rng(B), gen(B)
    k_pages, T = 3, 16 * P
    s = Server(B, P, H, H_kv, d, eight, 16 * B, T, k_pages, seed=B)
    keys, values = [np.zeros((0, H_kv, d)) for _ in range(B)], [np.zeros((0, H_kv, d)) for _ in range(B)]
    group = H // H_kv
    for step in range(7):
        new = rng.integers(0, 3 * P if step in (0, 4) else 3, B)
        new[new > T // B] = T // B
        qkv = bf16((T, H + 2 * H_kv, d), g)
        lse, lse_sparse = s.step(int32(new.tolist()), qkv.to(DEV))
        idxc.poll_device_status()
        assert not (s.start < 0).any()
        at = 0
        for b in range(B):
            rows = qkv[at:at + int(new[b])]
            keys[b], values[b] = np.concatenate([keys[b], rows64(rows[:, H:H + H_kv], eight)]), np.concatenate([values[b], rows64(rows[:, H + H_kv:], eight)])
            at += int(new[b])
        assert s.lens.tolist() == [k.shape[0] for k in keys]
        q = oracle.bf16_rows(codes(qkv[:B, :H]))
        sel, n_pages = s.pages.view(B, H_kv, k_pages).cpu().numpy(), s.n_pages.view(B, H_kv).cpu().numpy()
        scores = s.scores.view(B, H_kv, -1).cpu().numpy()
        for b in range(B):
            n = keys[b].shape[0]
            pages = oracle.ceil_div(n, P)
            assert np.all(n_pages[b] == pages)
            for h in range(H_kv):
                part = slice(h * group, (h + 1) * group)
                size = 0.1 * np.abs(q[b, part]).max() * (np.abs(keys[b][:, h]).sum(axis=1).max() if n else 0.0)
                check(s.out[b, 0, part], lse[b, 0, part], oracle.attention(q[b, part], keys[b][:, h], values[b][:, h], 0.1, np.ones((group, n), dtype=bool)), eight, n,
                      f"step {step} request {b} head {h}", size)
                chosen = sel[b, h][sel[b, h] >= 0]
                assert chosen.size == min(pages, k_pages) and np.all(np.diff(chosen) > 0)
                # the first and the newest page, and the best of the others (a tie or a rounding apart)
                if pages:
                    assert 0 in chosen and pages - 1 in chosen
                    others = [p for p in range(1, pages - 1)]
                    best = sorted((scores[b, h, p] for p in others), reverse=True)[:max(0, k_pages - 2)]
                    assert sorted((scores[b, h, p] for p in chosen if 0 < p < pages - 1), reverse=True) == best
                    for p in others:
                        exact = 0.1 * np.maximum(q[b, part] * oracle.bounds(oracle.to_bf16(keys[b][p * P:(p + 1) * P, h]))[0],
                                                 q[b, part] * oracle.bounds(oracle.to_bf16(keys[b][p * P:(p + 1) * P, h]))[1]).sum(axis=1).max()
                        assert abs(scores[b, h, p] - exact) <= 2.0 ** -7 * (abs(exact) + 0.1 * np.abs(q[b, part]).sum(axis=1).max())
                seen = np.isin(np.arange(n) // P, chosen)
                check(s.sparse[b, 0, part], lse_sparse[b, 0, part],
                      oracle.attention(q[b, part], keys[b][:, h], values[b][:, h], 0.1, np.broadcast_to(seen, (group, n))), eight, n, f"selected, step {step} request {b}", size)
        # some requests lose their newest tokens, one ends
        lens = np.array([k.shape[0] for k in keys])
        keep = np.maximum(lens - rng.integers(0, P + 2, B) * (rng.random(B) < 0.4), 0)
        keep[step % B] = 0 if step % 3 == 2 else keep[step % B]
        idxc.page_release(s.table, s.lens, int32(keep.tolist()), s.free, s.count, P)
        for b in range(B):
            keys[b], values[b] = keys[b][:keep[b]], values[b][:keep[b]]
        held = sum(oracle.ceil_div(int(n), P) for n in keep)
        assert int(s.count) == 16 * B - held


@pytest.mark.parametrize("eight", [False, True])
def test_a_captured_step_follows_its_buffers(eight):
    """One graph of a decode step, replayed while requests grow on the device, against the same steps made eagerly."""
    args = (6, 16, 8, 2, 64, eight, 64, 6, 4)
    a, b = Server(*args, seed=3), Server(*args, seed=3)
    g = gen(5)
    first = bf16((6, 12, 64), g).to(DEV)
    new = int32([1] * 6)
    live = first.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.step(new, live)                                   # outside the capture
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            lse, lse_sparse = a.step(new, live)
    torch.cuda.current_stream().wait_stream(side)
    b.step(new, first)
    for i in range(40):
        qkv = bf16((6, 12, 64), g).to(DEV)
        live.copy_(qkv)
        graph.replay()
        want = b.step(new, qkv)
        for x, y in ((a.out, b.out), (a.sparse, b.sparse), (lse, want[0]), (lse_sparse, want[1]), (a.lens, b.lens), (a.table, b.table), (a.slots, b.slots),
                     (a.pages, b.pages), (a.bounds, b.bounds), (a.count, b.count)):
            assert torch.equal(x, y), i
    idxc.poll_device_status()


def test_two_batches_on_two_streams_at_once():
    g = gen(8)
    steps = [bf16((64, 12, 64), g).to(DEV) for _ in range(30)]
    new = int32([10, 0, 3, 20, 1, 5])
    want = []
    for eight in (False, True):
        s = Server(6, 16, 8, 2, 64, eight, 512, 64, 4, seed=1)
        for x in steps:
            s.step(new, x)
        want.append((s.out.clone(), s.sparse.clone(), s.pages.clone(), s.slots.clone()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    servers = [Server(6, 16, 8, 2, 64, eight, 512, 64, 4, seed=1) for eight in (False, True)]
    torch.cuda.synchronize()
    for x in steps:
        for s, stream in zip(servers, streams):
            with torch.cuda.stream(stream):
                s.step(new, x, stream=stream)
    torch.cuda.synchronize()
    idxc.poll_device_status()
    for s, w in zip(servers, want):
        for x, y in zip((s.out, s.sparse, s.pages, s.slots), w):
            assert torch.equal(x, y)


@pytest.mark.parametrize("four", [False, True])
def test_the_latent_cache_and_its_selection_over_pages(four):
    """Slots as the rows that latent rows and indexer keys are appended to, and selected positions turned into rows of a paged cache: the sparse attention
    over pages gives the bits it gives over contiguous caches."""
    g = gen(4)
    B, P, H, k_top = 4, 32, 16, 40
    lens = [100, 7, 64, 333]
    T = sum(lens)
    n_pages = sum(oracle.ceil_div(n, P) for n in lens) + 3
    table, start = torch.full((B, 16), -1, dtype=torch.int32, device=DEV), int32([0] * B)
    free, count, ln, begin = torch.randperm(n_pages, generator=g).to(torch.int32).to(DEV), int32([n_pages]), int32([0] * B), int32([0] * (B + 1))
    slots = torch.empty(T, dtype=torch.int64, device=DEV)
    idxc.page_tables(table, ln, int32(lens), free, count, P, slots, begin, start)
    x = bf16((T, 576), g).to(DEV)
    if four:
        paged, flat = torch.zeros((n_pages * P, 416), dtype=torch.uint8, device=DEV), torch.zeros((T, 416), dtype=torch.uint8, device=DEV)
        idxc.quantize_q4(x, paged, dst_rows=slots)
        idxc.quantize_q4(x, flat)
    else:
        paged, flat = torch.zeros((n_pages * P, 576), dtype=torch.bfloat16, device=DEV), x
        paged[slots] = x
    keys = bf16((T, 128), g).to(DEV)
    k8, ks = torch.zeros((n_pages * P, 128), dtype=torch.uint8, device=DEV), torch.zeros(n_pages * P, device=DEV)
    f8, fs = torch.zeros((T, 128), dtype=torch.uint8, device=DEV), torch.zeros(T, device=DEV)
    idxc.quantize_e4m3(keys, k8, ks, dst_rows=slots)
    idxc.quantize_e4m3(keys, f8, fs)
    assert torch.equal(k8[slots], f8) and torch.equal(ks[slots], fs)
    T_sel = torch.full((B, k_top), -1, dtype=torch.int32)
    for b, n in enumerate(lens):
        pick = torch.randperm(n, generator=g)[:k_top].sort().values
        T_sel[b, :pick.numel()] = pick.to(torch.int32)
    rows = torch.empty((B, k_top), dtype=torch.int32, device=DEV)
    idxc.page_rows(table, T_sel.to(DEV), P, rows)
    q = bf16((B, H, 576), g).to(DEV)
    attend = idxc.sparse_attention_q4 if four else idxc.sparse_attention
    got = attend(q, paged, rows, 512, 1 / 24)
    want = attend(q, flat, T_sel.to(DEV), 512, 1 / 24, kv_base=begin[:B].to(torch.int64))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    idxc.poll_device_status()


def test_the_schedule_of_shared_layers_serves_page_selections():
    """A page selection has the format of the indexer's: the overlap tool and a Shared layer's reuse work on it as they are."""
    s = Server(4, 16, 8, 2, 64, False, 200, 400, 4, seed=2)
    g = gen(3)
    for n in (100, 1, 1):
        s.step(int32([n] * 4), bf16((400, 12, 64), g).to(DEV))
    mean = idxc.topk_overlap([s.pages, s.pages.clone()])
    assert mean.tolist() == [1.0]
    q = bf16((4, 1, 8, 64), g).to(DEV)
    a = idxc.paged_attention(s.cache, q, s.table, s.lens, 200, 0.1, pages=s.pages)
    b = idxc.paged_attention(s.cache, q, s.table, s.lens, 200, 0.1, pages=s.pages.view(4, 2, 4))
    assert torch.equal(a[0], b[0])
