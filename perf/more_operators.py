"""The operators of serving from a paged key/value cache: each in its plain form and as the library's calls.

A paged cache holds keys and values as [n_pages, page_size, H_kv, D], in bf16, or as e4m3 codes with one fp32 scale per token and
head ([n_pages, H_kv, page_size]; value = code * scale). Logical page p of request b is physical page table[b, p]; the slot of a
position is table[b, position / page_size] * page_size + position % page_size.

  tables     pages for the new tokens of a batch of requests, taken from a stack of free pages; the new tokens' slots; selected
             positions turned into cache rows; the pages given back
  append     keys and values of new tokens written to their slots, the touched pages' bounds (smallest and largest value of every
             key column) brought up to date, and the rows read back
  attend     query heads of new tokens over their request's pages, H / H_kv heads to a key head; token i of `steps` sees
             len - (steps - 1 - i) keys
  scores     the largest score that any key of a page could reach, from the page's bounds: max over the heads and new tokens of a
             key head of sum_d max(q_d lo_d, q_d hi_d)
  pages      the k pages of largest score for every request and key head, and the attention over the keys of those pages only
"""
import math

import torch

own = False

DEV = "cuda:0"
BF16, FP32 = torch.bfloat16, torch.float32
FORCED = 3.0e38          # score of the pages that are always kept


# ------------------------------------------------------------------ cases
def listed():
    return [
        # a verify step: 256 requests, four drafted tokens each, all rejected in the end; 2048 selected positions of each become rows
        {"name": "tables_draft_256", "op": "tables", "B": 256, "new_lo": 4, "new_hi": 4, "lo": 17, "hi": 9000, "page": 16, "k": 2048},
        # prompts admitted to an empty cache, and released
        {"name": "tables_prompts_24", "op": "tables", "B": 24, "new_lo": 100, "new_hi": 9003, "lo": 0, "hi": 0, "page": 64, "k": 2048},
        # a decode step's 32 new tokens: latency alone
        {"name": "append_bf16_32", "op": "append", "eight": False, "B": 32, "new_lo": 1, "new_hi": 1, "lo": 100, "hi": 3001, "H": 32, "Hkv": 8, "D": 128, "page": 16},
        # the tokens of a few long prompts at once, 8 bits
        {"name": "append_e4m3_prompts_6", "op": "append", "eight": True, "B": 6, "new_lo": 5000, "new_hi": 16383, "lo": 0, "hi": 130, "H": 32, "Hkv": 8, "D": 128, "page": 64},
        # one short conversation, one new token: latency
        {"name": "attend_bf16_1x777", "op": "attend", "eight": False, "B": 1, "steps": 1, "H": 32, "Hkv": 8, "D": 128, "lo": 777, "hi": 777, "page": 16},
        # a serving batch of long and ragged conversations
        {"name": "attend_bf16_32x4k_32k", "op": "attend", "eight": False, "B": 32, "steps": 1, "H": 64, "Hkv": 8, "D": 128, "lo": 4096, "hi": 32768, "page": 64},
        # eight full 131072-token contexts in 8 bits
        {"name": "attend_e4m3_8x131072", "op": "attend", "eight": True, "B": 8, "steps": 1, "H": 64, "Hkv": 8, "D": 128, "lo": 131072, "hi": 131072, "page": 64},
        # many conversations of a few thousand tokens on one GPU of several, narrow heads, three drafted tokens beside the new one
        {"name": "attend_bf16_96x2k_d64_s4", "op": "attend", "eight": False, "B": 96, "steps": 4, "H": 16, "Hkv": 2, "D": 64, "lo": 301, "hi": 4001, "page": 16},
        # the pages of one long conversation scored
        {"name": "scores_1x131071", "op": "scores", "B": 1, "steps": 1, "H": 64, "Hkv": 8, "D": 128, "lo": 131071, "hi": 131071, "page": 16},
        # the pages of a batch scored
        {"name": "scores_32x8k_64k", "op": "scores", "B": 32, "steps": 1, "H": 64, "Hkv": 8, "D": 128, "lo": 8192, "hi": 65536, "page": 16},
        # a decode step over 64 of up to 2048 pages for each key head
        {"name": "pages_bf16_16x65536", "op": "pages", "eight": False, "B": 16, "steps": 1, "H": 64, "Hkv": 8, "D": 128, "lo": 20000, "hi": 65536, "page": 32, "k": 64},
        # the same for a large batch in 8 bits, some of whose requests have fewer pages than are asked for
        {"name": "pages_e4m3_128x500_9k", "op": "pages", "eight": True, "B": 128, "steps": 1, "H": 32, "Hkv": 4, "D": 128, "lo": 500, "hi": 9001, "page": 64, "k": 32},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "append", "attend", "attend", "attend", "scores", "pages", "pages"])
    page = rng.choice([16, 32, 48, 64, 128])
    if op == "tables":
        B = _log_int(rng, 1, 512)
        new_hi = _log_int(rng, 1, max(1, 100000 // B))
        hi = rng.choice([0, _log_int(rng, 1, 9000)])
        return {"op": op, "B": B, "new_lo": int(new_hi * rng.random()), "new_hi": new_hi, "lo": int(hi * rng.random()), "hi": hi, "page": page,
                "k": rng.choice([2048, _log_int(rng, 1, 2048)])}
    Hkv, D = rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
    H = Hkv * rng.choice([1, 2, 4, 5, 7, 8, 16])
    if op == "append":
        B = _log_int(rng, 1, 256)
        new_hi = rng.choice([1, _log_int(rng, 1, max(1, 60000 // B))])
        return {"op": op, "eight": rng.random() < 0.5, "B": B, "new_lo": int(new_hi * rng.random()), "new_hi": new_hi, "lo": 0, "hi": _log_int(rng, 1, 300),
                "H": H, "Hkv": Hkv, "D": D, "page": page}
    B = _log_int(rng, 1, 256)
    hi = _log_int(rng, 1, min(131072, 4700000 // (B * Hkv)))
    case = {"op": op, "B": B, "steps": rng.choice([1, 1, 2, 4]), "H": H, "Hkv": Hkv, "D": D, "lo": max(1, int(hi * rng.random())), "hi": hi, "page": page}
    if op != "scores":
        case["eight"] = rng.random() < 0.5
    if op == "pages":
        case["k"] = _log_int(rng, 1, 512)
    return case


def _spread(n, lo, hi):
    """n lengths between lo and hi, in no order, the largest among them."""
    return [hi if b == n // 2 else lo + (hi - lo) * ((b * 7919 + 13) % 101) // 100 for b in range(n)]


def _lens(case):
    return _spread(case["B"], case["lo"], case["hi"])


def _new(case):
    return _spread(case["B"], case["new_lo"], case["new_hi"])


def _ceil(a, b):
    return -(-a // b)


# ------------------------------------------------------------------ inputs
def _normal(shape, gen, gain=1.0):
    out = torch.empty(shape, dtype=BF16, device=DEV)
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        n = min(1 << 28, flat.numel() - i)
        flat[i:i + n] = torch.randn((n,), generator=gen, device=DEV) * gain
    return out


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _cache(case, n_pages, gen):
    """Keys and values as projections leave them: unit spread, some key columns far wider than the rest."""
    P, Hkv, D = case["page"], case["Hkv"], case["D"]
    s = {}
    for name in ("k", "v"):
        x = _normal((n_pages, P, Hkv, D), gen)
        if name == "k":
            x.mul_((1.0 + 3.0 * torch.rand((Hkv, D), generator=gen, device=DEV) ** 12).to(BF16))
        s[name], s[name + "_scale"] = x, None
        if case["eight"]:
            codes = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=DEV)
            scale = torch.empty((n_pages, Hkv, P), dtype=FP32, device=DEV)
            for p in range(0, n_pages, 4096):
                codes[p:p + 4096], t = _eight_bits(x[p:p + 4096])
                scale[p:p + 4096] = t.transpose(1, 2)
            s[name], s[name + "_scale"] = codes, scale
    return s


def _tables_of(case, lens, gen):
    """The requests' pages somewhere in the cache, in no order, with some pages that belong to nobody."""
    P = case["page"]
    pages = [_ceil(n, P) for n in lens]
    total = sum(pages)
    n_pages = total + 7
    perm = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((len(lens), max(max(pages), 1) + 3), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, n_pages, perm[at:]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op, B, P = case["op"], case["B"], case["page"]
    s = {"op": op, "P": P}
    lens = _lens(case)
    if op == "tables":
        new = _new(case)
        owned = [_ceil(n, P) for n in lens]
        need = [_ceil(n + m, P) - p for n, m, p in zip(lens, new, owned)]
        table, _, _ = _tables_of(case, lens, gen)
        n_pages = sum(owned) + sum(need) + 50
        wide = torch.full((B, max(p + n for p, n in zip(owned, need)) + 5), -1, dtype=torch.int32, device=DEV)
        n = min(wide.shape[1], table.shape[1])
        wide[:, :n] = table[:, :n]
        # a second numbering of all pages, so that the free ones are those no request holds
        perm = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
        held = wide >= 0
        order = torch.cumsum(held.reshape(-1), 0).reshape(held.shape) - 1
        s["table"] = torch.where(held, perm[torch.where(held, order, 0)], wide)
        s["free"] = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
        s["free"][:n_pages - sum(owned)] = perm[sum(owned):]
        s["count"] = _int32([n_pages - sum(owned)])
        s["lens"], s["keep"], s["new"] = _int32(lens), _int32(lens), _int32(new)
        s["tokens"] = sum(new)
        see = _int32([max(n + m, 1) for n, m in zip(lens, new)])[:, None]
        # an ascending selection, one position per equal stretch, -1 behind it (a request that sees less has fewer)
        j = torch.arange(case["k"], device=DEV, dtype=torch.int32)[None, :]
        take = torch.minimum(see, torch.full_like(see, case["k"]))
        s["positions"] = torch.where(j < take, (j.to(torch.int64) * see // take).to(torch.int32), torch.full_like(j, -1))
        return s
    if op == "append":
        new = _new(case)
        after = [n + m for n, m in zip(lens, new)]
        table, n_pages, _ = _tables_of(case, after, gen)
        s.update(_cache(case, n_pages, gen))
        T, Hkv, D = sum(new), case["Hkv"], case["D"]
        s["slots"] = torch.cat([table[b, torch.arange(n, n + m, device=DEV) // P].to(torch.int64) * P + torch.arange(n, n + m, device=DEV) % P
                                for b, (n, m) in enumerate(zip(lens, new))])
        # keys and values where the projection leaves them: behind the query heads of the same row
        row = _normal((T, (case["H"] + 2 * Hkv) * D), gen)
        s["new_k"] = row[:, case["H"] * D:(case["H"] + Hkv) * D].view(T, Hkv, D)
        s["new_v"] = row[:, (case["H"] + Hkv) * D:].view(T, Hkv, D)
        s["bounds"] = _normal((n_pages, Hkv, 2, D), gen)
        _with_handle(s)
        return s
    s["lens"], s["max_len"], s["scale"], s["Hkv"] = _int32(lens), max(lens), 1.0 / math.sqrt(case["D"]), case["Hkv"]
    table, n_pages, _ = _tables_of(case, lens, gen)
    s["table"] = table
    Hkv, D, steps = case["Hkv"], case["D"], case["steps"]
    s["q"] = _normal((B, steps, case["H"] + 2 * Hkv, D), gen, 1.5)[:, :, :case["H"]]
    ld = (table.shape[1] + 3) // 4 * 4
    s["pages_of"] = _int32([_ceil(n, P) for n in lens])
    if op == "scores":
        middle, half = _normal((n_pages, Hkv, 1, D), gen), _normal((n_pages, Hkv, 1, D), gen).abs() + 1
        s["bounds"] = torch.cat((middle - half, middle + half), dim=2).contiguous()
        s["out"] = torch.zeros((B * Hkv, ld), dtype=FP32, device=DEV)
        return s
    s.update(_cache(case, n_pages, gen))
    _with_handle(s)
    if op == "pages":
        s["scores"] = torch.randn((B * Hkv, ld), generator=gen, device=DEV) * 3.0 + 10.0
        at = torch.arange(ld, device=DEV)[None, :]
        n = s["pages_of"].repeat_interleave(Hkv)[:, None]
        s["scores"][(at == 0).expand_as(s["scores"]) | (at == n - 1)] = FORCED        # the first and the newest page are kept
        s["row_pages"] = n.reshape(-1).contiguous()
        s["k_pages"] = case["k"]
    return s


def _with_handle(s):
    """What a program keeps beside its cache for the library's calls."""
    if own:
        from paper_2603_12201_b200 import binding as idxc

        s["cache"] = idxc.PagedCache(s["k"], s["v"], s.get("k_scale"), s.get("v_scale"), s.get("bounds"))


# ------------------------------------------------------------------ plain forms
def _eight_bits(x):
    """[..., D] -> e4m3 codes of x / scale and the scale of every row of D."""
    x = x.to(FP32)
    top = x.abs().amax(dim=-1).clamp_min(1e-12)
    scale = top / torch.full_like(top, 448.0)
    return (x / scale[..., None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn), scale


def _values(x, scale):
    """Cache rows [..., page_size, H_kv, D] as the values they stand for, float32; scale [..., H_kv, page_size]."""
    return x.to(FP32) if scale is None else x.to(FP32) * scale.transpose(-1, -2)[..., None]


def _tables(s):
    P, table, lens, new, free = s["P"], s["table"], s["lens"].to(torch.int64), s["new"].to(torch.int64), s["free"]
    B, ld = table.shape
    T = s["tokens"]
    owned = (lens + P - 1) // P
    need = (lens + new + P - 1) // P - owned
    upto = torch.cumsum(need, 0)
    served = upto <= s["count"].to(torch.int64)
    start = torch.where(served, lens, torch.full_like(lens, -1))
    p = torch.arange(ld, device=DEV)[None, :]
    flat = (upto - need)[:, None] + p - owned[:, None]
    fresh = (p >= owned[:, None]) & (p < (owned + need)[:, None]) & served[:, None]
    top = s["count"].to(torch.int64) - 1
    after = torch.where(fresh, free[torch.where(fresh, top - flat, 0)], table)
    begin = torch.nn.functional.pad(torch.cumsum(new, 0), (1, 0))
    t = torch.arange(T, device=DEV)
    req = (t[:, None] >= begin[None, 1:]).sum(dim=1)
    at = start[req] + t - begin[req]
    slots = torch.where(start[req] >= 0, after[req, torch.where(start[req] >= 0, at, 0) // P].to(torch.int64) * P + at % P, -1)
    pos = s["positions"].to(torch.int64)
    page = torch.gather(after, 1, pos.clamp_min(0) // P).to(torch.int64)
    rows = torch.where((pos >= 0) & (page >= 0), page * P + pos % P, -1).to(torch.int32)
    # given back: what lies behind the length that is kept
    grown = torch.where(served, lens + new, lens)
    keep = torch.minimum(s["keep"].to(torch.int64), grown)
    first, last = (keep + P - 1) // P, (grown + P - 1) // P
    back = (last - first).clamp_min(0)
    count = s["count"].to(torch.int64) - torch.where(served, need, 0).sum()
    gone = (p >= first[:, None]) & (p < last[:, None])
    place = count + back.sum() - 1 - ((torch.cumsum(back, 0) - back)[:, None] + p - first[:, None])
    wide = torch.cat((free, free[:1]))                             # entries that stay go to a place of their own
    wide = wide.scatter(0, torch.where(gone, place, free.shape[0]).reshape(-1), after.reshape(-1))
    table.copy_(torch.where(gone, torch.full_like(after, -1), after))
    s["free"].copy_(wide[:-1])
    s["count"].copy_((count + back.sum()).to(torch.int32))
    s["lens"].copy_(keep)
    return {"slots": slots, "begin": begin.to(torch.int32), "start": start.to(torch.int32), "rows": rows, "table": table, "free": s["free"],
            "count": s["count"], "lens": s["lens"]}


def _append(s):
    P, slots = s["P"], s["slots"]
    page, off = slots // P, slots % P
    for name in ("k", "v"):
        if s[name + "_scale"] is None:
            s[name][page, off] = s["new_" + name]
        else:
            codes, scale = _eight_bits(s["new_" + name])
            s[name].view(torch.uint8)[page, off] = codes.view(torch.uint8)
            s[name + "_scale"][page, :, off] = scale
    n_pages = s["k"].shape[0]
    last = torch.full((n_pages,), -1, dtype=torch.int64, device=DEV).scatter_reduce(0, page, off, "amax")      # newest row of every touched page
    out = {}
    for name in ("k", "v"):
        rows = s[name].view(torch.uint8)[page, off].view(s[name].dtype) if s[name + "_scale"] is not None else s[name][page, off]
        v = rows.to(FP32) if s[name + "_scale"] is None else rows.to(FP32) * s[name + "_scale"][page, :, off][..., None]
        out[name] = v.to(BF16)
    for p0 in range(0, n_pages, 2048):
        held = _values(s["k"][p0:p0 + 2048], None if s["k_scale"] is None else s["k_scale"][p0:p0 + 2048]).to(BF16)
        inside = (torch.arange(P, device=DEV)[None, :] <= last[p0:p0 + 2048, None])[:, :, None, None]
        lo = torch.where(inside, held, float("inf")).amin(dim=1)
        hi = torch.where(inside, held, float("-inf")).amax(dim=1)
        touched = (last[p0:p0 + 2048] >= 0)[:, None, None, None]
        s["bounds"][p0:p0 + 2048] = torch.where(touched, torch.stack((lo, hi), dim=2), s["bounds"][p0:p0 + 2048])
    out["bounds"] = s["bounds"]
    return out


def _softmax_rows(q, k, v, sees, scale):
    """q [G, steps, group, D], k, v [G, n, D], sees [G, steps, n] -> out [G, steps, group, D], lse [G, steps, group], all float32."""
    G, steps, group, D = q.shape
    x = torch.matmul(q.reshape(G, steps * group, D), k.transpose(1, 2)).reshape(G, steps, group, -1) * scale
    x = x.masked_fill(~sees[:, :, None, :], float("-inf"))
    top = x.amax(dim=-1, keepdim=True)
    top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
    e = torch.exp(x - top)
    z = e.sum(dim=-1, keepdim=True)
    p = torch.where(z > 0, e / torch.where(z > 0, z, torch.ones_like(z)), torch.zeros_like(e))
    return torch.matmul(p.reshape(G, steps * group, -1), v).reshape(G, steps, group, D), (top + torch.log(z)).squeeze(-1)


def _grouped(q, Hkv):
    """[B, steps, H, D] -> [B, H_kv, steps, group, D] float32."""
    B, steps, H, D = q.shape
    return q.to(FP32).reshape(B, steps, Hkv, H // Hkv, D).permute(0, 2, 1, 3, 4)


def _attend(s):
    P, Hkv = s["P"], s["Hkv"]
    B, steps, H, D = s["q"].shape
    out = torch.empty((B, steps, H, D), dtype=BF16, device=DEV)
    lse = torch.empty((B, steps, H), dtype=FP32, device=DEV)
    n_pages = _ceil(s["max_len"], P)
    at = torch.arange(n_pages * P, device=DEV)
    q = _grouped(s["q"], Hkv)
    per = max(1, (1 << 31) // (n_pages * P * Hkv * D * 4))                # requests at a time
    for b0 in range(0, B, per):
        b1 = min(B, b0 + per)
        page = s["table"][b0:b1, :n_pages].clamp_min(0).to(torch.int64)
        k, v = [_values(s[n][page], None if s[n + "_scale"] is None else s[n + "_scale"][page]).permute(0, 3, 1, 2, 4).reshape((b1 - b0) * Hkv, n_pages * P, D)
                for n in ("k", "v")]
        inside = at[None, :] < s["lens"][b0:b1, None]
        v = torch.where(inside.repeat_interleave(Hkv, 0)[:, :, None], v, torch.zeros_like(v))
        sees = at < (s["lens"][b0:b1, None] - (steps - 1) + torch.arange(steps, device=DEV))[:, :, None]
        o, z = _softmax_rows(q[b0:b1].reshape(-1, steps, H // Hkv, D), k, v, sees.repeat_interleave(Hkv, 0), s["scale"])
        out[b0:b1] = o.reshape(b1 - b0, Hkv, steps, H // Hkv, D).permute(0, 2, 1, 3, 4).reshape(b1 - b0, steps, H, D).to(BF16)
        lse[b0:b1] = z.reshape(b1 - b0, Hkv, steps, H // Hkv).permute(0, 2, 1, 3).reshape(b1 - b0, steps, H)
    return {"out": out, "lse": lse}


def _scores(s):
    B, steps, H, D = s["q"].shape
    Hkv = s["Hkv"]
    q = _grouped(s["q"], Hkv).reshape(B, Hkv, -1, D)
    ld = s["table"].shape[1]
    p = torch.arange(ld, device=DEV)[None, :]
    n = s["pages_of"][:, None].to(torch.int64)
    for b in range(B):
        edge = s["bounds"][s["table"][b].clamp_min(0).to(torch.int64)].to(FP32).permute(1, 2, 3, 0)      # [H_kv, 2, D, pages]
        u = torch.matmul(q[b].clamp_min(0.0), edge[:, 1]) + torch.matmul(q[b].clamp_max(0.0), edge[:, 0])
        u = u.amax(dim=1) * s["scale"]
        u = torch.where((p < 1) | (p >= n[b] - 1), torch.full_like(u, FORCED), u)
        rows = s["out"][b * Hkv:(b + 1) * Hkv, :ld]
        rows.copy_(torch.where(p < n[b], u, rows))
    return {"scores": s["out"], "pages": s["pages_of"].repeat_interleave(Hkv)}


def _select(s):
    at = torch.arange(s["scores"].shape[1], device=DEV)[None, :]
    n = s["row_pages"][:, None].to(torch.int64)
    k = s["k_pages"]
    order = torch.sort(s["scores"].masked_fill(at >= n, float("-inf")), dim=1, descending=True, stable=True).indices
    order = torch.nn.functional.pad(order, (0, max(0, k - order.shape[1])), value=1 << 30)[:, :k]
    j = torch.arange(k, device=DEV)[None, :]
    kept = torch.where(j < n, order, 1 << 30).sort(dim=1).values
    return torch.where(j < n, kept, -1)


def _pages(s):
    P, Hkv = s["P"], s["Hkv"]
    B, steps, H, D = s["q"].shape
    sel = _select(s)
    pick = sel.reshape(B, Hkv, -1)
    k_pages = pick.shape[2]
    q = _grouped(s["q"], Hkv)
    head = torch.arange(Hkv, device=DEV)[None, :, None]
    out = torch.empty((B, steps, H, D), dtype=BF16, device=DEV)
    lse = torch.empty((B, steps, H), dtype=FP32, device=DEV)
    per = max(1, (1 << 31) // (k_pages * P * Hkv * D * 4))
    for b0 in range(0, B, per):
        b1 = min(B, b0 + per)
        one = pick[b0:b1]
        page = torch.gather(s["table"][b0:b1, None, :].expand(-1, Hkv, -1), 2, one.clamp_min(0)).to(torch.int64)
        pos = (one[..., None] * P + torch.arange(P, device=DEV)).reshape(b1 - b0, Hkv, -1)
        lens = s["lens"][b0:b1, None, None]
        inside = (one[..., None].expand(-1, -1, -1, P).reshape(b1 - b0, Hkv, -1) >= 0) & (pos < lens)
        kv = []
        for n in ("k", "v"):
            x = s[n].view(torch.uint8).view(s[n].shape + (-1,))[page, :, head].reshape(b1 - b0, Hkv, k_pages, P, -1).view(s[n].dtype).to(FP32)
            if s[n + "_scale"] is not None:
                x = x * s[n + "_scale"][page, head][..., None]
            kv.append(x.reshape((b1 - b0) * Hkv, k_pages * P, D))
        v = torch.where(inside.reshape(-1, k_pages * P)[:, :, None], kv[1], torch.zeros_like(kv[1]))
        sees = inside[:, :, None, :] & (pos[:, :, None, :] < lens[..., None] - (steps - 1) + torch.arange(steps, device=DEV)[None, None, :, None])
        o, z = _softmax_rows(q[b0:b1].reshape(-1, steps, H // Hkv, D), kv[0], v, sees.reshape(-1, steps, k_pages * P), s["scale"])
        out[b0:b1] = o.reshape(b1 - b0, Hkv, steps, H // Hkv, D).permute(0, 2, 1, 3, 4).reshape(b1 - b0, steps, H, D).to(BF16)
        lse[b0:b1] = z.reshape(b1 - b0, Hkv, steps, H // Hkv).permute(0, 2, 1, 3).reshape(b1 - b0, steps, H)
    return {"pages": sel.to(torch.int32), "out": out, "lse": lse}


# ------------------------------------------------------------------ the library's calls
def _run_own(s):
    from paper_2603_12201_b200 import binding as idxc

    op = s["op"]
    if op == "tables":
        B, T = s["table"].shape[0], s["tokens"]
        slots = torch.empty((T,), dtype=torch.int64, device=DEV)
        begin = torch.empty((B + 1,), dtype=torch.int32, device=DEV)
        start = torch.empty((B,), dtype=torch.int32, device=DEV)
        rows = torch.empty_like(s["positions"])
        idxc.page_tables(s["table"], s["lens"], s["new"], s["free"], s["count"], s["P"], slots, begin, start)
        idxc.page_rows(s["table"], s["positions"], s["P"], rows)
        idxc.page_release(s["table"], s["lens"], s["keep"], s["free"], s["count"], s["P"])
        return {"slots": slots, "begin": begin, "start": start, "rows": rows, "table": s["table"], "free": s["free"], "count": s["count"], "lens": s["lens"]}
    if op == "append":
        k, v = torch.empty(s["new_k"].shape, dtype=BF16, device=DEV), torch.empty(s["new_v"].shape, dtype=BF16, device=DEV)
        idxc.paged_append(s["cache"], s["new_k"], s["new_v"], s["slots"])
        idxc.paged_gather(s["cache"], s["slots"], k, v)
        return {"k": k, "v": v, "bounds": s["bounds"]}
    if op == "attend":
        out, lse = idxc.paged_attention(s["cache"], s["q"], s["table"], s["lens"], s["max_len"], s["scale"])
        return {"out": out, "lse": lse}
    if op == "scores":
        n = torch.empty((s["out"].shape[0],), dtype=torch.int32, device=DEV)
        idxc.page_scores(s["bounds"], s["q"], s["table"], s["lens"], s["P"], s["scale"], s["out"], n)
        return {"scores": s["out"], "pages": n}
    sel = torch.empty((s["scores"].shape[0], s["k_pages"]), dtype=torch.int32, device=DEV)
    idxc.topk_rows(s["scores"], s["k_pages"], sel, lens=s["row_pages"])
    out, lse = idxc.paged_attention(s["cache"], s["q"], s["table"], s["lens"], s["max_len"], s["scale"], pages=sel)
    return {"pages": sel, "out": out, "lse": lse}


def run(state):
    if own:
        return _run_own(state)
    return {"tables": _tables, "append": _append, "attend": _attend, "scores": _scores, "pages": _pages}[state["op"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op, B, P = case["op"], case["B"], case["page"]
    lens = _lens(case)
    if op == "tables":
        new = _new(case)
        need = sum(_ceil(n + m, P) - _ceil(n, P) for n, m in zip(lens, new))
        # pages taken, entered, taken out and put back; a slot per token; positions read, rows written
        return {"bytes": 16 * need + 8 * sum(new) + 8 * B * case["k"] + 24 * B, "flops": 0}
    Hkv, D, H = case["Hkv"], case["D"], case["H"]
    row = (2 * D + 8) if case.get("eight") else 4 * D          # a key and a value of one head
    if op == "append":
        new = _new(case)
        pages = sum(_ceil(n + m, P) - n // P for n, m in zip(lens, new) if m)
        old = sum(n % P for n, m in zip(lens, new) if m)
        T = sum(new)
        return {"bytes": T * Hkv * (4 * D + 2 * row + 4 * D) + 16 * T + old * Hkv * row // 2 + pages * Hkv * 4 * D, "flops": 0}
    steps = case["steps"]
    io = B * steps * H * D * 2
    if op == "scores":
        pages = sum(_ceil(n, P) for n in lens)
        return {"bytes": pages * (Hkv * (4 * D + 4) + 4) + io, "flops": 4 * D * steps * H * pages}
    io = 2 * io + 4 * B * steps * H
    if op == "attend":
        pairs = sum(max(0, n - i) for n in lens for i in range(steps)) * H
        return {"bytes": sum(lens) * Hkv * row + sum(_ceil(n, P) for n in lens) * 4 + io, "flops": 4 * D * pairs}
    picked = sum(min(n, min(case["k"], _ceil(n, P)) * P) for n in lens)
    scored = sum(_ceil(n, P) for n in lens)
    return {"bytes": picked * Hkv * row + scored * Hkv * 4 + B * Hkv * case["k"] * 8 + io, "flops": 4 * D * steps * H * picked}


# ------------------------------------------------------------------ 64 bits
def _rows64(s, name, slots, head):
    """Rows of one head at the given slots, by arithmetic on the slots, in 64 bits."""
    P = s["P"]
    page, off = torch.div(slots, P, rounding_mode="floor"), torch.remainder(slots, P)
    if s[name + "_scale"] is None:
        return s[name][page, off, head].double()
    return s[name].view(torch.uint8)[page, off, head].view(torch.float8_e4m3fn).double() * s[name + "_scale"][page, head, off].double()[:, None]


def exact(case, seed):
    s = prepare(case, seed)
    op, B, P = s["op"], case["B"], s["P"]
    lens = _lens(case)
    if op == "tables":
        new = _new(case)
        table, free, count = s["table"].cpu(), s["free"].cpu().tolist(), int(s["count"])
        before, slots, start, begin = table.clone(), [], [], [0]
        for b in range(B):                                   # one request after the other, one page after the other
            need = _ceil(lens[b] + new[b], P) - _ceil(lens[b], P)
            begin.append(begin[-1] + new[b])
            assert need <= count                             # the cases leave pages over
            for p in range(need):
                count -= 1
                table[b, _ceil(lens[b], P) + p] = free[count]
            start.append(lens[b])
            at = torch.arange(lens[b], lens[b] + new[b])
            slots.append(table[b, at // P].to(torch.int64) * P + at % P)
        pos = s["positions"].cpu().to(torch.int64)
        page = torch.gather(table, 1, pos.clamp_min(0) // P).to(torch.int64)
        rows = torch.where((pos >= 0) & (page >= 0), page * P + pos % P, -1).to(torch.int32)
        return {"slots": torch.cat(slots).to(DEV), "begin": _int32(begin), "start": _int32(start), "rows": rows.to(DEV), "table": before.to(DEV),
                "free": s["free"], "count": s["count"], "lens": _int32(lens)}
    if op == "append":
        out = {}
        slots = s["slots"]
        for name in ("k", "v"):
            x = s["new_" + name].double()
            if s[name + "_scale"] is not None:
                scale = (s["new_" + name].float().abs().amax(dim=-1).clamp_min(1e-12).double() / 448.0).float()[..., None]
                code = (s["new_" + name].float() / scale).to(torch.float8_e4m3fn).double()
                s[name + "_scale"][slots // P, :, slots % P] = scale[..., 0]
                s[name].view(torch.uint8)[slots // P, slots % P] = code.to(torch.float8_e4m3fn).view(torch.uint8)
                x = code * scale.double()
            else:
                s[name][slots // P, slots % P] = s["new_" + name]
            out[name] = x
        bounds = s["bounds"].double()
        newest = {}
        for slot in slots.tolist():
            newest[slot // P] = max(newest.get(slot // P, -1), slot % P)
        pages = torch.tensor(list(newest), device=DEV)
        upto = torch.tensor(list(newest.values()), device=DEV)
        for head in range(case["Hkv"]):
            for p0 in range(0, pages.numel(), 4096):
                pg = pages[p0:p0 + 4096]
                at = (pg[:, None] * P + torch.arange(P, device=DEV)).reshape(-1)
                rows = _rows64(s, "k", at, head).reshape(pg.numel(), P, -1)
                inside = (torch.arange(P, device=DEV)[None, :] <= upto[p0:p0 + 4096, None])[:, :, None]
                bounds[pg, head, 0] = torch.where(inside, rows, math.inf).amin(dim=1)
                bounds[pg, head, 1] = torch.where(inside, rows, -math.inf).amax(dim=1)
        out["bounds"] = bounds
        return out
    Hkv, steps, H, D = s["Hkv"], case["steps"], case["H"], case["D"]
    group = H // Hkv
    if op == "scores":
        u = s["out"].double()
        for b, n in enumerate(lens):
            pages = _ceil(n, P)
            for head in range(Hkv):
                edge = s["bounds"][s["table"][b, :pages].to(torch.int64), head].double()
                q = s["q"][b, :, head * group:(head + 1) * group].double().reshape(-1, D)
                best = torch.full((pages,), -math.inf, dtype=torch.float64, device=DEV)
                for row in q:
                    best = torch.maximum(best, torch.maximum(row * edge[:, 0], row * edge[:, 1]).sum(dim=1))
                best = best * s["scale"]
                best[0] = best[pages - 1] = torch.tensor(FORCED, dtype=FP32).double()
                u[b * Hkv + head, :pages] = best
        return {"scores": u, "pages": _int32([_ceil(n, P) for n in lens for _ in range(Hkv)])}
    out = torch.zeros((B, steps, H, D), dtype=torch.float64, device=DEV)
    lse = torch.full((B, steps, H), -math.inf, dtype=torch.float64, device=DEV)
    sel = torch.full((B * Hkv, case.get("k", 1)), -1, dtype=torch.int32, device=DEV)
    for b, n in enumerate(lens):
        for head in range(Hkv):
            if op == "pages":
                row = b * Hkv + head
                pages = _ceil(n, P)
                best = torch.argsort(-s["scores"][row, :pages].double(), stable=True)[:case["k"]].sort().values
                sel[row, :best.numel()] = best.to(torch.int32)
                pos = (best[:, None] * P + torch.arange(P, device=DEV)).reshape(-1)
                pos = pos[pos < n]
            else:
                pos = torch.arange(n, device=DEV)
            slots = s["table"][b, pos // P].to(torch.int64) * P + pos % P
            k, v = _rows64(s, "k", slots, head), _rows64(s, "v", slots, head)
            for i in range(steps):
                q = s["q"][b, i, head * group:(head + 1) * group].double()
                x = torch.where((pos < n - (steps - 1 - i))[None, :], (q @ k.T) * s["scale"], -math.inf)
                z = torch.logsumexp(x, dim=1)
                p = torch.where(torch.isfinite(z)[:, None], torch.exp(x - z[:, None]), 0.0)
                out[b, i, head * group:(head + 1) * group] = p @ v
                lse[b, i, head * group:(head + 1) * group] = z
    return {"out": out, "lse": lse} if op == "attend" else {"pages": sel, "out": out, "lse": lse}
