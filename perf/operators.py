"""The operators around a latent key/value cache under memory pressure: each in its plain form and as the library's call.

A latent cache row is 576 columns per token: 512 value columns (keys too) and 64 positional columns (keys only). Held in
bf16 a row takes 1152 bytes. Held in 4 bits it takes 416 bytes (uint8): bytes 0..255 the 512 codes, bytes 256..287 one bf16
scale per 32 columns, bytes 288..415 the 64 positional columns in bf16. A code is a nibble u = code + 8, code in -7..7; the
four bytes of columns 8g..8g+7 hold, nibble by nibble from the lowest, columns 0 2 4 6 1 3 5 7 of the eight.

  quantize   rows of bf16 -> rows of 416 bytes, written at given cache rows; returned as the values they stand for
  attend     every head of a new token over its sequence's cached rows (values = their first 512 columns); several new tokens
             of a sequence see one key more each; cache in bf16 or 4 bits
  sparse     the same over the rows that an index tensor selects, cache in 4 bits
  weights    attention probability that every cached position received, summed over heads and new tokens, added to a decayed sum
  evict      the positions of a sequence that stay (the newest, and the largest sums among the others), and the cache rows
             of those positions brought together
"""
import math

import torch

own = False

D_V, D_R, D = 512, 64, 576
GROUP = 32
ROW4 = 256 + 32 + 128
SCALE = 1.0 / 24.0
DEV = "cuda:0"


# ------------------------------------------------------------------ cases
def listed():
    return [
        # a decode step's 32 new tokens appended to the 4-bit cache: latency alone
        {"name": "quantize_append_32", "op": "quantize", "n": 32, "rows": 65536, "scatter": True},
        # a prompt's rows written at once
        {"name": "quantize_prompt_131071", "op": "quantize", "n": 131071, "rows": 131071, "scatter": False},
        # one short conversation, one new token: latency
        {"name": "attend_bf16_1x777", "op": "attend", "four": False, "B": 1, "steps": 1, "H": 128, "lo": 777, "hi": 777},
        # a serving batch of long and very ragged conversations, 128 heads
        {"name": "attend_bf16_32x16k_64k", "op": "attend", "four": False, "B": 32, "steps": 1, "H": 128, "lo": 16384, "hi": 65536},
        # 64 conversations of a few thousand tokens, one GPU's 16 heads of eight GPUs, two drafted tokens beside the new one
        {"name": "attend_bf16_64x5k_h16_s3", "op": "attend", "four": False, "B": 64, "steps": 3, "H": 16, "lo": 1000, "hi": 9001},
        # eight full 131072-token contexts in the 4-bit cache
        {"name": "attend_4bit_8x131072", "op": "attend", "four": True, "B": 8, "steps": 1, "H": 128, "lo": 131072, "hi": 131072},
        # a decode step after the indexer: 32 tokens, 2048 selected rows each
        {"name": "sparse_4bit_decode_32", "op": "sparse", "n_q": 32, "H": 128, "k_top": 2048, "n_kv": 1048576, "prefill": False},
        # a chunk of a prompt after the indexer (its first rows see fewer than 2048 keys)
        {"name": "sparse_4bit_prefill_2047", "op": "sparse", "n_q": 2047, "H": 128, "k_top": 2048, "n_kv": 3001, "prefill": True},
        # scoring the cached positions of a batch before an eviction, bf16 cache
        {"name": "weights_bf16_8x40k", "op": "weights", "four": False, "B": 8, "steps": 1, "H": 128, "lo": 20001, "hi": 60000},
        # the same for one conversation in the 4-bit cache, 16 heads, four new tokens
        {"name": "weights_4bit_1x8k_h16_s4", "op": "weights", "four": True, "B": 1, "steps": 4, "H": 16, "lo": 8191, "hi": 8191},
        # eight contexts cut to a quarter, 4-bit rows
        {"name": "evict_4bit_8x131072", "op": "evict", "four": True, "B": 8, "lo": 131072, "hi": 131072, "budget": 32768, "recent": 512},
        # ragged conversations cut to 2048 rows, bf16 rows; some are shorter than that and stay whole
        {"name": "evict_bf16_24x900_6k", "op": "evict", "four": False, "B": 24, "lo": 900, "hi": 6007, "budget": 2048, "recent": 65},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "attend", "attend", "attend", "sparse", "sparse", "weights", "evict"])
    if op == "quantize":
        n = _log_int(rng, 1, 131071)
        scatter = rng.random() < 0.5
        return {"op": op, "n": n, "rows": n + (rng.randrange(0, 5000) if scatter else 0), "scatter": scatter}
    if op == "sparse":
        n_q = _log_int(rng, 1, 1500)
        prefill = n_q >= 48 and rng.random() < 0.6
        n_kv = n_q + _log_int(rng, 1, 20000)
        return {"op": op, "n_q": n_q, "H": rng.choice([5, 16, 24, 64, 100, 128]), "k_top": rng.choice([2048, 1024, 2001, _log_int(rng, 1, 2048)]),
                "n_kv": n_kv, "prefill": prefill}
    B = _log_int(rng, 1, 64)
    hi = _log_int(rng, 1, min(131072, 1250000 // B))
    lo = max(1, int(hi * rng.random()))
    if op == "evict":
        budget = _log_int(rng, 1, hi + 100)
        return {"op": op, "four": rng.random() < 0.5, "B": B, "lo": lo, "hi": hi, "budget": budget, "recent": rng.randrange(0, min(budget, 600) + 1)}
    H = rng.choice([5, 16, 32, 64, 100, 128])
    steps = rng.choice([1, 1, 2, 4])
    while B > 1 and B * hi * H * steps > 1250000 * 128:
        B -= 1
    return {"op": op, "four": rng.random() < 0.5, "B": B, "steps": steps, "H": H, "lo": lo, "hi": hi}


def _lens(case):
    """Lengths of the case's sequences: spread between lo and hi, in no order, the longest among them."""
    B, lo, hi = case["B"], case["lo"], case["hi"]
    return [hi if b == B // 2 else lo + (hi - lo) * ((b * 7919 + 13) % 101) // 100 for b in range(B)]


def _starts(lens):
    """First cache row of every sequence: one behind the other with a few rows between."""
    out, at = [], 3
    for n in lens:
        out.append(at)
        at += n + 5
    return out, at


# ------------------------------------------------------------------ the 4-bit format
_NIBBLE_COLUMN = [0, 2, 4, 6, 1, 3, 5, 7]      # column of the eight that nibble i of a word holds


def _pack(values):
    """[n, 576] float32 -> [n, 416] uint8: groups of 32 columns share the smallest scale of 5 significant bits that holds
    their largest magnitude in 7 steps."""
    n = values.shape[0]
    x = values[:, :D_V].reshape(n, D_V // GROUP, GROUP)
    top = x.abs().amax(dim=2).clamp_min(7.0 * 2.0 ** -100)
    bits = (top / torch.full_like(top, 7.0)).view(torch.int32)      # a tensor divides; a number would multiply by its rounded inverse
    scale = ((bits + 0x7FFFF) & ~0x7FFFF).view(torch.float32)
    code = torch.round(x / scale[:, :, None]).clamp_(-7.0, 7.0).to(torch.int32) + 8
    word = code.reshape(n, D_V // 8, 8)[:, :, _NIBBLE_COLUMN]
    low, high = word[:, :, 0::2], word[:, :, 1::2]
    out = torch.empty((n, ROW4), dtype=torch.uint8, device=values.device)
    out[:, :256] = (low + 16 * high).to(torch.uint8).reshape(n, 256)
    out[:, 256:288] = scale.to(torch.bfloat16).view(torch.uint8).reshape(n, 32)
    out[:, 288:] = values[:, D_V:].to(torch.bfloat16).contiguous().view(torch.uint8).reshape(n, 128)
    return out


def _unpack(rows):
    """[..., 416] uint8 -> [..., 576] float32, the values that the rows stand for."""
    lead = rows.shape[:-1]
    b = rows[..., :256].reshape(*lead, 64, 4)
    nib = torch.stack((b & 15, b >> 4), dim=-1).reshape(*lead, 64, 8)
    back = [_NIBBLE_COLUMN.index(c) for c in range(8)]
    code = nib[..., back].reshape(*lead, D_V // GROUP, GROUP).to(torch.float32) - 8.0
    scale = rows[..., 256:288].contiguous().view(torch.bfloat16).to(torch.float32)
    rope = rows[..., 288:].contiguous().view(torch.bfloat16).to(torch.float32)
    return torch.cat(((code * scale[..., None]).reshape(*lead, D_V), rope), dim=-1)


def _read(rows):
    return _unpack(rows) if rows.dtype == torch.uint8 else rows.to(torch.float32)


# ------------------------------------------------------------------ inputs
def _normal(shape, gen, gain=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * gain).to(torch.bfloat16)


def _cache(rows, four, gen):
    """Latent rows as a normalised projection leaves them (unit spread); the 4-bit ones as the quantiser leaves them."""
    if not four:
        return _normal((rows, D), gen)
    out = torch.empty((rows, ROW4), dtype=torch.uint8, device=DEV)
    for r in range(0, rows, 131072):
        n = min(131072, rows - r)
        out[r:r + n] = _pack(torch.randn((n, D), generator=gen, device=DEV))
    return out


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op = case["op"]
    s = {"op": op}
    if op == "quantize":
        # hidden rows have a few large columns beside many small ones
        gain = 0.25 + torch.rand((1, D), generator=gen, device=DEV) ** 8 * 8.0
        s["x"] = (torch.randn((case["n"], D), generator=gen, device=DEV) * gain).to(torch.bfloat16)
        s["dst"] = torch.randperm(case["rows"], generator=gen, device=DEV)[:case["n"]].contiguous() if case["scatter"] else None
        s["cache"] = torch.zeros((case["rows"], ROW4), dtype=torch.uint8, device=DEV)
        return s
    if op == "sparse":
        n_q, k, n_kv = case["n_q"], case["k_top"], case["n_kv"]
        s["q"] = _normal((n_q, case["H"], D), gen, 2.0)
        s["kv"] = _cache(n_kv, True, gen)
        if case["prefill"]:      # queries n_kv - n_q .. n_kv - 1 of one prompt; each picks positions at or before its own
            s["base"] = None
            see = torch.arange(n_kv - n_q, n_kv, device=DEV) + 1
        else:                    # every query has its own sequence, one after the other in the cache
            each = n_kv // n_q
            s["base"] = torch.arange(n_q, device=DEV) * each
            see = torch.full((n_q,), each, device=DEV)
        # an ascending selection without repeats: one position per equal stretch of what the query sees, padded with -1
        take = torch.minimum(see, torch.full_like(see, k))
        j = torch.arange(k, device=DEV)[None, :]
        first = j * see[:, None] // take[:, None]
        last = (j + 1) * see[:, None] // take[:, None]
        u = torch.rand((n_q, k), generator=gen, device=DEV)
        pick = first + torch.minimum((u * (last - first)).to(torch.int64), last - first - 1)
        s["topk"] = torch.where(j < take[:, None], pick, torch.full_like(pick, -1)).to(torch.int32)
        return s
    lens = _lens(case)
    starts, rows = _starts(lens)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["base"] = torch.tensor(starts, dtype=torch.int64, device=DEV)
    s["max_len"] = max(lens)
    s["kv"] = _cache(rows, case["four"], gen)
    B = case["B"]
    if op in ("attend", "weights"):
        s["q"] = _normal((B, case["steps"], case["H"], D), gen, 2.0)
    if op in ("weights", "evict"):
        ld = (s["max_len"] + 3) // 4 * 4
        # sums of probabilities as they stand after some steps: a few positions hold most of them
        s["acc"] = torch.rand((B, ld), generator=gen, device=DEV) ** 12 * 4.0
    if op == "weights":
        # what the attention of the same step left: log-sum-exp per head, over the visible positions of the plain form
        s["lse"] = _scores(s)[1]
        s["out"] = torch.empty_like(s["acc"])
    if op == "evict":
        s["budget"], s["recent"] = case["budget"], case["recent"]
        s["dst_base"] = torch.arange(B, device=DEV) * case["budget"]
        s["dst"] = torch.zeros((B * case["budget"], s["kv"].shape[1]), dtype=s["kv"].dtype, device=DEV)
    return s


# ------------------------------------------------------------------ plain forms
def _rows(s):
    """The sequences' cache rows side by side, padded to the longest: [B, max_len, 576] float32."""
    at = torch.arange(s["max_len"], device=DEV)[None, :]
    inside = at < s["lens"][:, None]
    row = torch.where(inside, s["base"][:, None] + at, torch.zeros_like(at))
    return _read(s["kv"][row])


def _scores(s, rows=None):
    """Scaled scores [B, steps, H, max_len] with -inf where a new token does not see a position, and their log-sum-exp."""
    rows = _rows(s) if rows is None else rows
    B, steps, H, _ = s["q"].shape
    x = torch.matmul(s["q"].to(torch.float32).reshape(B, steps * H, D), rows.transpose(1, 2)).reshape(B, steps, H, -1) * SCALE
    sees = s["lens"][:, None] - (steps - 1) + torch.arange(steps, device=DEV)[None, :]
    x = x.masked_fill(torch.arange(x.shape[-1], device=DEV) >= sees[:, :, None, None], float("-inf"))
    top = x.amax(dim=-1, keepdim=True)
    top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
    return x, (top + torch.log(torch.exp(x - top).sum(dim=-1, keepdim=True))).squeeze(-1)


def _quantize(s):
    row = torch.arange(s["x"].shape[0], device=DEV) if s["dst"] is None else s["dst"]
    s["cache"][row] = _pack(s["x"].to(torch.float32))
    return {"values": _unpack(s["cache"][row]).to(torch.bfloat16)}


def _attend(s):
    rows = _rows(s)
    x, lse = _scores(s, rows)
    B, steps, H, n = x.shape
    shift = torch.where(lse == float("-inf"), torch.zeros_like(lse), lse)
    p = torch.exp(x - shift[..., None]).reshape(B, steps * H, n)
    return {"out": torch.matmul(p, rows[:, :, :D_V]).reshape(B, steps, H, D_V).to(torch.bfloat16), "lse": lse}


def _sparse(s):
    pick = s["topk"].to(torch.int64)
    base = 0 if s["base"] is None else s["base"][:, None]
    rows = _read(s["kv"][torch.where(pick >= 0, pick + base, torch.zeros_like(pick))])
    x = torch.matmul(s["q"].to(torch.float32), rows.transpose(1, 2)) * SCALE
    x = x.masked_fill((pick < 0)[:, None, :], float("-inf"))
    top = x.amax(dim=-1, keepdim=True)
    e = torch.exp(x - top)
    z = e.sum(dim=-1, keepdim=True)
    return {"out": torch.matmul(e / z, rows[:, :, :D_V]).to(torch.bfloat16), "lse": (top + torch.log(z)).squeeze(-1)}


def _weights(s):
    x, _ = _scores(s)
    inside = torch.arange(s["max_len"], device=DEV)[None, :] < s["lens"][:, None]
    shift = torch.where(s["lse"] == float("-inf"), torch.zeros_like(s["lse"]), s["lse"])
    p = torch.exp(x - shift[..., None]).sum(dim=(1, 2))
    s["out"].copy_(s["acc"])
    s["out"][:, :s["max_len"]] = torch.where(inside, 0.75 * s["acc"][:, :s["max_len"]] + p, s["acc"][:, :s["max_len"]])
    return {"acc": s["out"]}


def _evict(s):
    lens, budget, recent = s["lens"].to(torch.int64), s["budget"], s["recent"]
    B, ld = s["acc"].shape
    at = torch.arange(ld, device=DEV)[None, :]
    worth = s["acc"].masked_fill(at >= lens[:, None] - recent, float("inf"))
    order = torch.sort(worth.masked_fill(at >= lens[:, None], float("-inf")), dim=1, descending=True, stable=True).indices
    stay = torch.minimum(lens, torch.full_like(lens, budget))
    order = torch.nn.functional.pad(order, (0, max(0, budget - ld)), value=ld)[:, :budget]
    slot = torch.arange(budget, device=DEV)[None, :]
    kept = torch.where(slot < stay[:, None], order, torch.full_like(order, ld)).sort(dim=1).values
    used = slot < stay[:, None]
    src = torch.where(used, kept + s["base"][:, None], torch.zeros_like(kept))
    s["dst"].copy_(torch.where(used.reshape(-1, 1), s["kv"][src.reshape(-1)], s["dst"]))
    return {"keep": torch.where(used, kept, torch.full_like(kept, -1)).to(torch.int32), "lens": stay.to(torch.int32),
            "values": _read(s["dst"]).to(torch.bfloat16)}


# ------------------------------------------------------------------ the library's calls
def _run_own(s):
    from paper_2603_12201_b200 import binding as idxc

    op = s["op"]
    if op == "quantize":
        idxc.quantize_q4(s["x"], s["cache"], dst_rows=s["dst"])
        values = torch.empty_like(s["x"])
        idxc.dequantize_q4(s["cache"], values, src_rows=s["dst"])
        return {"values": values}
    if op == "attend":
        out, lse = idxc.latent_attention(s["q"], s["kv"], s["base"], s["lens"], s["max_len"], D_V, SCALE)
        return {"out": out, "lse": lse}
    if op == "sparse":
        out, lse = idxc.sparse_attention_q4(s["q"], s["kv"], s["topk"], D_V, SCALE, kv_base=s["base"])
        return {"out": out, "lse": lse}
    if op == "weights":
        s["out"].copy_(s["acc"])
        idxc.attention_weights(s["q"], s["kv"], s["lse"], s["out"], SCALE, kv_base=s["base"], lens=s["lens"], max_len=s["max_len"], beta=0.75)
        return {"acc": s["out"]}
    B = s["lens"].shape[0]
    keep = torch.empty((B, s["budget"]), dtype=torch.int32, device=DEV)
    lens = torch.empty((B,), dtype=torch.int32, device=DEV)
    idxc.evict_select(s["acc"], s["lens"], s["budget"], s["recent"], keep, lens)
    idxc.compact_rows(s["kv"], s["dst"], keep, lens, src_base=s["base"], dst_base=s["dst_base"])
    if s["dst"].dtype == torch.uint8:
        values = torch.empty((s["dst"].shape[0], D), dtype=torch.bfloat16, device=DEV)
        idxc.dequantize_q4(s["dst"], values)
        return {"keep": keep, "lens": lens, "values": values}
    return {"keep": keep, "lens": lens, "values": s["dst"]}


def run(state):
    if own:
        return _run_own(state)
    return {"quantize": _quantize, "attend": _attend, "sparse": _sparse, "weights": _weights, "evict": _evict}[state["op"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op = case["op"]
    if op == "quantize":      # rows read; their 416 bytes written and read back as values
        return {"bytes": case["n"] * (2 * D + ROW4 + 2 * D + (8 if case["scatter"] else 0)), "flops": 0}
    if op == "sparse":
        n_q, H, k, n_kv = case["n_q"], case["H"], case["k_top"], case["n_kv"]
        if case["prefill"]:
            entries = sum(min(k, t + 1) for t in range(n_kv - n_q, n_kv))
            rows = min(n_kv, entries)
        else:
            entries = rows = n_q * min(k, n_kv // n_q)
        io = n_q * (H * (2 * D + 2 * D_V + 4) + 4 * k)
        return {"bytes": rows * ROW4 + io, "flops": 2 * H * (D + D_V) * entries}
    lens = _lens(case)
    row = ROW4 if case["four"] else 2 * D
    if op == "evict":
        stay = [min(n, case["budget"]) for n in lens]
        return {"bytes": 4 * sum(lens) + 2 * row * sum(stay) + 4 * sum(stay) + (2 * D + row) * len(lens) * case["budget"] * int(case["four"]), "flops": 0}
    steps, H = case["steps"], case["H"]
    pairs = sum(max(0, n - i) for n in lens for i in range(steps)) * H
    if op == "weights":
        return {"bytes": sum(lens) * (row + 8) + case["B"] * steps * H * (2 * D + 4), "flops": 2 * D * pairs}
    return {"bytes": sum(lens) * row + case["B"] * steps * H * (2 * D + 2 * D_V + 4), "flops": 2 * (D + D_V) * pairs}


# ------------------------------------------------------------------ 64 bits
def _row64(raw):
    """One definition apart from _unpack: the value of column c of a row, from its bytes."""
    if raw.dtype != torch.uint8:
        return raw.double()
    c = torch.arange(D_V, device=raw.device)
    in8 = c % 8
    nibble = torch.where(in8 % 2 == 0, in8 // 2, 4 + in8 // 2)
    byte = raw[:, (c // 8) * 4 + nibble // 2].to(torch.int64)
    code = torch.bitwise_and(torch.bitwise_right_shift(byte, 4 * (nibble % 2)), 15) - 8
    word = raw[:, 256:].to(torch.int64)
    halves = word[:, 0::2] + 256 * word[:, 1::2]

    def bf16(h):
        sign = 1.0 - 2.0 * (h >> 15).double()
        exponent = (h >> 7) & 255
        mantissa = (h & 127).double()
        normal = (1.0 + mantissa / 128.0) * torch.pow(2.0, (exponent - 127).double())
        return sign * torch.where(exponent > 0, normal, mantissa / 128.0 * 2.0 ** -126)

    return torch.cat((code.double() * bf16(halves[:, c // GROUP]), bf16(halves[:, 16:])), dim=1)


def _soft64(q, rows, keys):
    """q [R, 576], rows [n, 576] in 64 bits, keys [R] = visible leading rows -> (out [R, 512], lse [R], p [R, n])"""
    x = (q @ rows.T) * SCALE
    x = torch.where(torch.arange(rows.shape[0], device=q.device)[None, :] < keys[:, None], x, float("-inf"))
    lse = torch.logsumexp(x, dim=1)
    p = torch.where(torch.isfinite(lse)[:, None], torch.exp(x - lse[:, None]), 0.0)
    return p @ rows[:, :D_V], lse, p


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op == "quantize":
        x = s["x"].double()
        top = x[:, :D_V].reshape(-1, 16, 32).abs().max(dim=2).values.clamp_min(7.0 * 2.0 ** -100)
        top = top / torch.full_like(top, 7.0)
        mantissa, exponent = torch.frexp(top)          # mantissa in [1/2, 1): five bits = steps of 1/32
        scale = torch.ldexp(torch.ceil(mantissa * 32.0) / 32.0, exponent)
        per = scale.repeat_interleave(32, dim=1)
        return {"values": torch.cat((torch.round(x[:, :D_V] / per).clamp(-7, 7) * per, x[:, D_V:]), dim=1)}
    if op == "sparse":
        n_q, H, _ = s["q"].shape
        out = torch.empty((n_q, H, D_V), dtype=torch.float64, device=DEV)
        lse = torch.empty((n_q, H), dtype=torch.float64, device=DEV)
        for t in range(n_q):
            pick = s["topk"][t]
            row = pick[pick >= 0].to(torch.int64) + (0 if s["base"] is None else s["base"][t])
            rows = _row64(s["kv"][row])
            out[t], lse[t], _ = _soft64(s["q"][t].double(), rows, torch.full((H,), rows.shape[0], device=DEV))
        return {"out": out, "lse": lse}
    if op in ("attend", "weights"):
        B, steps, H, _ = s["q"].shape
        out = torch.empty((B, steps, H, D_V), dtype=torch.float64, device=DEV)
        lse = torch.empty((B, steps, H), dtype=torch.float64, device=DEV)
        acc = s["acc"].double() if op == "weights" else None
        for b, n in enumerate(_lens(case)):
            rows = _row64(s["kv"][int(s["base"][b]):int(s["base"][b]) + n])
            for i in range(steps):
                q = s["q"][b, i].double()
                keys = torch.full((H,), n - (steps - 1 - i), device=DEV)
                if op == "attend":
                    out[b, i], lse[b, i], _ = _soft64(q, rows, keys)
                    continue
                x = (q @ rows.T) * SCALE - s["lse"][b, i].double()[:, None]
                p = torch.where(torch.arange(n, device=DEV)[None, :] < keys[:, None], torch.exp(x), 0.0).sum(dim=0)
                acc[b, :n] = (0.75 if i == 0 else 1.0) * acc[b, :n] + p
        return {"out": out, "lse": lse} if op == "attend" else {"acc": acc}
    budget, recent = s["budget"], s["recent"]
    keep = torch.full((case["B"], budget), -1, dtype=torch.int64, device=DEV)
    values = torch.zeros((case["B"] * budget, D), dtype=torch.float64, device=DEV)
    stay = []
    for b, n in enumerate(_lens(case)):
        stay.append(min(n, budget))
        if n <= budget:
            best = torch.arange(n, device=DEV)
        else:
            old = n - recent
            by_worth = torch.argsort(-s["acc"][b, :old].double(), stable=True)[:budget - recent]
            best = torch.cat((by_worth, torch.arange(old, n, device=DEV))).sort().values
        keep[b, :stay[b]] = best
        values[b * budget:b * budget + stay[b]] = _row64(s["kv"][best + s["base"][b]])
    return {"keep": keep.to(torch.int32), "lens": torch.tensor(stay, dtype=torch.int32, device=DEV), "values": values}
