"""Caches, block tables and bounds for the paged-cache tests."""
import numpy as np
import torch

from oracle import paged as oracle
from paper_2603_12201_b200 import binding as idxc
from tests.util import codes

DEV = "cuda:0"


def gen(seed):
    return torch.Generator().manual_seed(seed)


def int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def bf16(shape, g, gain=1.0):
    return (torch.randn(shape, generator=g) * gain).to(torch.bfloat16)


class Cache:
    """A paged cache on the GPU and its values in float64. layout: "tokens" [pages, P, heads, d], "heads" [pages, heads, P, d], "pair": keys and
    values of a page in one array. Values are drawn; in 8 bits codes and scales are."""

    def __init__(self, n_pages, P, H_kv, d, eight, g, layout="tokens", bounds=False):
        self.shape = (n_pages, P, H_kv, d)
        if eight:
            x = torch.randn((2, *self.shape), generator=g).mul_(100.0).clamp_(-448, 448).to(torch.float8_e4m3fn)
            self.scale = torch.exp(torch.randn((2, n_pages, H_kv, P), generator=g)) * 0.01
        else:
            x, self.scale = bf16((2, *self.shape), g), None
        if layout == "heads":
            store = x.view(torch.uint8 if eight else torch.int16).permute(0, 1, 3, 2, 4).contiguous().to(DEV).view(x.dtype)
            k, v = store[0].permute(0, 2, 1, 3), store[1].permute(0, 2, 1, 3)
        elif layout == "pair":
            store = x.view(torch.uint8 if eight else torch.int16).permute(1, 0, 2, 3, 4).contiguous().to(DEV).view(x.dtype)
            k, v = store[:, 0], store[:, 1]
        else:
            k, v = x[0].to(DEV), x[1].to(DEV)
        self.k, self.v = k, v
        self.k_scale, self.v_scale = (None, None) if self.scale is None else (self.scale[0].to(DEV), self.scale[1].to(DEV))
        self.bounds = bf16((n_pages, H_kv, 2, d), g).to(DEV) if bounds else None
        self.handle = idxc.PagedCache(self.k, self.v, self.k_scale, self.v_scale, self.bounds)

    def values(self):
        """(k, v) [n_pages, P, H_kv, d] float64, read back from the device."""
        out = []
        for x, s in ((self.k, self.k_scale), (self.v, self.v_scale)):
            if s is None:
                out.append(oracle.bf16_rows(codes(x)))
            else:
                out.append(oracle.e4m3_values(codes(x)) * s.cpu().double().numpy().transpose(0, 2, 1)[..., None])
        return out


def tables(lens, P, g, spare=5, extra=2):
    """Block tables whose pages lie anywhere in the cache, and the cache's pages."""
    pages = [oracle.ceil_div(n, P) for n in lens]
    n_pages = sum(pages) + spare
    perm = torch.randperm(n_pages, generator=g).to(torch.int32)
    table = torch.full((len(lens), max(pages) + extra), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, n_pages


def check(out, lse, want, eight, keys, what="", q_size=0.0, under=0.0):
    """out [R, d] bf16, lse [R] against the oracle's (out, lse, spread, reach). Scores: products are exact in fp32 and summed in d / 16 <= 8 matrix
    steps of relative error at most 2^-21 each, then scaled: within 2^-17 of reach. In 8 bits q is f16 after a power of two that
    brings its largest element to [1, 2): off by at most 2^-25 of that element (q_size: scale * max|q| * max_s sum|k_s|), and two more
    scalings, 2^-23 of reach. Sums of probabilities and of values: at most 2^-23 a term. Probabilities are rounded to bf16 (half a step 2^-8) or f16 (2^-11),
    exp2 is off by 2^-21. The output is rounded to bf16, half a step of which is 2^-8. under: what f16's smallest steps add in 8 bits (underflow())."""
    o_out, o_lse, spread, reach = want
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    empty = np.isneginf(o_lse)
    assert np.array_equal(np.isneginf(lse), empty), f"{what}: rows that see nothing"
    assert np.all(out[empty] == 0), f"{what}: rows that see nothing"
    e = (2.0 ** -17 + 2.0 ** -23) * reach + (2.0 ** -24 * q_size if eight else 0.0)
    total = keys * 2.0 ** -23 + 2.0 ** -20
    rounding = 2.0 ** -11 if eight else 2.0 ** -8
    bound = spread * (rounding + 2 * e[:, None] + 2 * total) * (1 + 2.0 ** -7) + np.abs(o_out) * 2.0 ** -8 + under
    err = np.abs(out - o_out)
    assert np.all(err <= bound), f"{what}: out off by {(err / np.maximum(bound, 1e-300)).max():.2f} bounds"
    ok = ~empty
    l_bound = e[ok] + total + 2.0 ** -20 * np.abs(o_lse[ok])
    assert np.all(np.abs(lse[ok] - o_lse[ok]) <= l_bound), f"{what}: lse off by {(np.abs(lse[ok] - o_lse[ok]) / l_bound).max():.2f} bounds"


def underflow(rows, k, codes, v_scale, scale, mask, lse):
    """[R, d]. In 8 bits probability times scale times 2^6 is an f16, below 2^-14 off by up to 2^-25 whatever its size: 2^-31 |code| a key, over the sum of
    probabilities 2^(x - m). The reference m is at most the largest x + log2(v_scale), rounded up, so 2^m over that sum is at most twice the
    largest softmax * v_scale: in all 2^-30 max_s(softmax_s v_scale_s) sum_s |code_s|."""
    x = np.where(mask, scale * (rows @ k.T), -np.inf)
    w = np.exp(x - np.where(np.isneginf(lse), 0.0, lse)[:, None]) * v_scale
    return 2.0 ** -30 * w.max(axis=1, initial=0.0)[:, None] * (mask.astype(np.float64) @ np.abs(codes))


def oracle_attention(cache_values, q, table, lens, P, H_kv, scale, n_pages, pages=None, only=None, v_scale=None):
    """For every (request, key head) of `only` (all): (b, head, rows [n_step, group], oracle.attention's results, keys, q_size, underflow in 8 bits)."""
    k_all, v_all = cache_values
    B, n_step, H, d = q.shape
    group = H // H_kv
    qv = oracle.bf16_rows(codes(q))
    table = table.cpu().numpy()
    for b in range(B):
        n = max(int(lens[b]), 0)
        owned = oracle.ceil_div(n, P)
        for head in range(H_kv):
            if only is not None and (b, head) not in only:
                continue
            if pages is None:
                pos = np.arange(n)
            else:
                chosen = [int(p) for p in pages[b, head, :min(pages.shape[2], owned)] if 0 <= p < owned]
                pos = np.concatenate([np.arange(p * P, min(p * P + P, n)) for p in chosen]) if chosen else np.zeros(0, dtype=np.int64)
            page = table[b, pos // P] if pos.size else pos
            inside = (page >= 0) & (page < n_pages)
            at = np.where(inside, page, 0)
            k, v = k_all[at, pos % P, head], v_all[at, pos % P, head]
            rows = qv[b, :, head * group:(head + 1) * group].reshape(n_step * group, d)
            sees = np.repeat(n - (n_step - 1 - np.arange(n_step)), group)
            mask = inside[None, :] & (pos[None, :] < sees[:, None])
            used = mask.any(axis=0)
            size = abs(scale) * np.abs(rows).max() * np.abs(k[used]).sum(axis=1).max() if used.any() else 0.0
            want = oracle.attention(rows, k, v, scale, mask)
            under = 0.0
            if v_scale is not None and used.any():
                s = v_scale[at, head, pos % P][used]
                under = underflow(rows, k[used], v[used] / s[:, None], s, scale, mask[:, used], want[1])
            yield b, head, want, pos.size, size, under


def check_call(cache, q, table, lens, scale, out, lse, pages=None, only=None, what=""):
    n_pages, P, H_kv, d = cache.shape
    B, n_step, H, _ = q.shape
    group = H // H_kv
    v_scale = None if cache.v_scale is None else cache.v_scale.double().cpu().numpy()
    for b, head, want, keys, size, under in oracle_attention(cache.values(), q, table, lens, P, H_kv, scale, n_pages, pages, only, v_scale):
        part = slice(head * group, (head + 1) * group)
        check(out[b, :, part].reshape(n_step * group, d), lse[b, :, part].reshape(-1), want, cache.scale is not None, keys, f"{what} request {b} head {head}", size, under)
