"""Inputs and bounds for the latent-cache tests."""
import numpy as np
import torch

from oracle import latent as oracle


def bits(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


def stored(t: torch.Tensor) -> np.ndarray:
    """A cache tensor as the oracle takes it."""
    return t.detach().cpu().contiguous().numpy() if t.dtype == torch.uint8 else bits(t)


def bf16_rows(n, gen, gain=1.0):
    return (torch.randn((n, 576), generator=gen) * gain).to(torch.bfloat16)


def q4_rows(n, gen):
    """Rows of any codes (-8 included) with 5-bit scales around 1/4: drawn, not quantised."""
    out = torch.randint(0, 256, (n, 416), generator=gen, dtype=torch.int32).to(torch.uint8)
    m = torch.randint(16, 32, (n, 16), generator=gen).float() / 128.0
    out[:, 256:288] = m.to(torch.bfloat16).view(torch.uint8).reshape(n, 32)
    out[:, 288:] = torch.randn((n, 64), generator=gen).to(torch.bfloat16).view(torch.uint8).reshape(n, 128)
    return out


def cache_rows(n, four, gen):
    return q4_rows(n, gen) if four else bf16_rows(n, gen)


def score_error(reach):
    """How far a score may be off: the products are exact in fp32 and 576 of them are summed in fp32 in some order; with a
    relative error of at most 2^-22 a step and 576 / 16 = 36 steps of the matrix instruction (576 / 32 + 5 in the plain
    kernel), the sum is within 36 * 2^-22 < 2^-16 of the sum of magnitudes; scaling and the change to base 2 add 2^-22."""
    return 2.0 ** -16 * reach


def check_attention(out, lse, o_out, o_lse, spread, reach, what=""):
    """out [R, 512] bf16 and lse [R] against the oracle. A probability p is off by a factor within exp(+-2e) from the scores
    (e = score_error: its own score and the normaliser), 2^-8 from rounding p to bf16, and 2^-20 from exp2 and the fp32 sums
    of up to 2^13 terms per split; the output is then rounded to bf16, half a step of which is 2^-8."""
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    empty = np.isneginf(o_lse)
    assert np.array_equal(np.isneginf(lse), empty), f"{what}: rows that see nothing"
    assert np.all(out[empty] == 0), f"{what}: rows that see nothing"
    e = score_error(reach)[:, None]
    bound = spread * (2.0 ** -8 + 2 * e + 2.0 ** -20) * (1 + 2.0 ** -7) + np.abs(o_out) * 2.0 ** -8
    err = np.abs(out - o_out)
    assert np.all(err <= bound), f"{what}: out off by {(err / np.maximum(bound, 1e-300)).max():.2f} bounds"
    ok = ~empty
    lerr = np.abs(lse[ok] - o_lse[ok])
    assert np.all(lerr <= score_error(reach)[ok] + 2.0 ** -20 * (1 + np.abs(o_lse[ok]))), f"{what}: lse off by {lerr.max() if lerr.size else 0}"


def oracle_sequence(q, kv, base, n, n_step, scale, n_kv=None):
    """The oracle over one sequence: q [n_step, H, 576] tensor, its rows kv[base : base + n]; rows outside the cache take no part."""
    H = q.shape[1]
    total = kv.shape[0]
    idx = np.arange(base, base + n)
    inside = (idx >= 0) & (idx < total)
    rows = stored(kv[torch.as_tensor(np.clip(idx, 0, max(total - 1, 0)), dtype=torch.int64, device=kv.device)]) if total else np.zeros((0, 576), np.uint16)
    keys = np.repeat(n - (n_step - 1 - np.arange(n_step)), H)
    mask = (np.arange(n)[None, :] < keys[:, None]) & inside[None, :]
    return oracle.attention(bits(q).reshape(n_step * H, 576), rows, scale, mask)
