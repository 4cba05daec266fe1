"""Python binding of the idxc C-ABI library: argument marshalling only.

Every step of the path (scoring, selection, schedule bookkeeping) runs inside
``libidxc.so``; torch is used for device memory and streams. There is no CPU or
eager fallback: if the library is missing or a call fails, an exception is raised.
Function names mirror ``include/idxc.h``.
"""
from __future__ import annotations

import contextlib
import ctypes
from pathlib import Path

import torch

_LIB_PATH = Path(__file__).resolve().parent / "libidxc.so"

OK = 0
ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_PATTERN, ERR_CUDA, ERR_DEVICE_TIMEOUT = 1, 2, 3, 4, 5, 6
BF16, FP8_E4M3 = 0, 1
LATENT_BF16, LATENT_Q4 = 0, 1
Q4_ROW_BYTES = 416
FLAG_COPY_SHARED = 0x1
FLAG_SIMT_SCORER = 0x2
FLAG_FILL_MASKED = 0x4
FLAG_STREAM_TOPK = 0x8

EXPORTED_SYMBOLS = [
    "idxc_status_string", "idxc_prefill_workspace_bytes", "idxc_indexer_prefill", "idxc_decode_workspace_bytes",
    "idxc_indexer_decode", "idxc_topk_rows", "idxc_schedule_create", "idxc_schedule_destroy",
    "idxc_schedule_begin_pass", "idxc_schedule_source", "idxc_schedule_stats", "idxc_schedule_prefill_layer",
    "idxc_schedule_decode_layer", "idxc_poll_device_status", "idxc_launch_count", "idxc_indexer_decode_noalloc",
    "idxc_selftest_bounded_wait", "idxc_selftest_tmem_readout", "idxc_selftest_tmem_readout_under_mma", "idxc_selftest_issue_rates", "idxc_quantize_e4m3", "idxc_topk_overlap", "idxc_pattern_search_dp",
    "idxc_pattern_search_greedy", "idxc_distill_kl", "idxc_sparse_attention_workspace_bytes", "idxc_sparse_attention",
    "idxc_quantize_q4", "idxc_dequantize_q4", "idxc_latent_attention_workspace_bytes", "idxc_latent_attention", "idxc_sparse_attention_q4",
    "idxc_attention_weights", "idxc_evict_select", "idxc_compact_rows",
    "idxc_page_tables", "idxc_page_release", "idxc_page_rows", "idxc_paged_append", "idxc_paged_gather", "idxc_paged_attention_workspace_bytes",
    "idxc_paged_attention", "idxc_page_scores",
]
NOALLOC_SCRATCH_BYTES = 16 << 20


EVAL_LOSS_FN = ctypes.CFUNCTYPE(ctypes.c_double, ctypes.c_char_p, ctypes.c_int, ctypes.c_void_p)


class IdxcError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library; raises if it has not been built (run paper_2603_12201_b200/build.py)."""
    global _lib
    if _lib is None:
        if not _LIB_PATH.exists():
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2603_12201_b200.build` "
                               "(there is no fallback path)")
        L = ctypes.CDLL(str(_LIB_PATH))
        vp, i64, i32, u32, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_uint32, ctypes.c_size_t
        L.idxc_status_string.restype = ctypes.c_char_p
        L.idxc_status_string.argtypes = [i32]
        L.idxc_launch_count.restype = i64
        L.idxc_prefill_workspace_bytes.restype = sz
        L.idxc_prefill_workspace_bytes.argtypes = [i64, i64, i32, i32, i32, i32, u32]
        L.idxc_decode_workspace_bytes.restype = sz
        L.idxc_decode_workspace_bytes.argtypes = [i32, i64, i32, i32, i32, i32, u32]
        prefill_args = [vp, vp, vp, vp, vp, i64, i64, i64, i32, i32, i32, i32, vp, i64, vp, vp, sz, u32, vp]
        decode_args = [vp, vp, i64, vp, vp, vp, vp, vp, i32, i64, i32, i32, i32, i32, vp, i64, vp, vp, sz, u32, vp]
        L.idxc_indexer_prefill.restype = i32
        L.idxc_indexer_prefill.argtypes = prefill_args
        L.idxc_indexer_decode.restype = i32
        L.idxc_indexer_decode.argtypes = decode_args
        L.idxc_indexer_decode_noalloc.restype = i32
        L.idxc_indexer_decode_noalloc.argtypes = [vp, vp, i64, vp, vp, vp, vp, vp, i32, i64, i32, i32, i32, i32, vp, u32, vp]
        L.idxc_topk_rows.restype = i32
        L.idxc_topk_rows.argtypes = [vp, i64, i64, i64, i64, vp, i32, vp, vp]
        L.idxc_schedule_create.restype = i32
        L.idxc_schedule_create.argtypes = [ctypes.c_char_p, i32, ctypes.POINTER(vp)]
        L.idxc_schedule_destroy.restype = None
        L.idxc_schedule_destroy.argtypes = [vp]
        L.idxc_schedule_begin_pass.restype = i32
        L.idxc_schedule_begin_pass.argtypes = [vp]
        L.idxc_schedule_source.restype = i32
        L.idxc_schedule_source.argtypes = [vp, i32, ctypes.POINTER(i32)]
        L.idxc_schedule_stats.restype = i32
        L.idxc_schedule_stats.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32), ctypes.POINTER(i64)]
        L.idxc_schedule_prefill_layer.restype = i32
        L.idxc_schedule_prefill_layer.argtypes = [vp, i32] + prefill_args + [ctypes.POINTER(vp)]
        L.idxc_schedule_decode_layer.restype = i32
        L.idxc_schedule_decode_layer.argtypes = [vp, i32] + decode_args + [ctypes.POINTER(vp)]
        L.idxc_topk_overlap.restype = i32
        L.idxc_topk_overlap.argtypes = [vp, vp, i32, i64, i32, vp, vp, vp]
        L.idxc_pattern_search_dp.restype = i32
        L.idxc_pattern_search_dp.argtypes = [vp, i32, i32, ctypes.c_char_p, ctypes.POINTER(ctypes.c_double)]
        L.idxc_pattern_search_greedy.restype = i32
        L.idxc_pattern_search_greedy.argtypes = [i32, i32, EVAL_LOSS_FN, vp, ctypes.c_char_p, ctypes.POINTER(i32),
                                                 ctypes.POINTER(ctypes.c_double), ctypes.POINTER(i64)]
        L.idxc_distill_kl.restype = i32
        L.idxc_distill_kl.argtypes = [vp, i64, i64, i64, i64, ctypes.POINTER(vp), i32, vp, i32, vp, vp, vp]
        L.idxc_sparse_attention_workspace_bytes.restype = sz
        L.idxc_sparse_attention_workspace_bytes.argtypes = [i64, i32]
        L.idxc_sparse_attention.restype = i32
        L.idxc_sparse_attention.argtypes = [vp, vp, vp, vp, i64, i64, i32, i32, i32, i32, ctypes.c_float, vp, vp, vp, sz, vp]
        L.idxc_quantize_e4m3.restype = i32
        L.idxc_quantize_e4m3.argtypes = [vp, i64, i32, vp, vp, vp, vp]
        L.idxc_quantize_q4.restype = i32
        L.idxc_quantize_q4.argtypes = [vp, i64, vp, i64, vp, vp]
        L.idxc_dequantize_q4.restype = i32
        L.idxc_dequantize_q4.argtypes = [vp, i64, vp, i64, vp, vp]
        L.idxc_latent_attention_workspace_bytes.restype = sz
        L.idxc_latent_attention_workspace_bytes.argtypes = [i64, i32, i64, i32]
        L.idxc_latent_attention.restype = i32
        L.idxc_latent_attention.argtypes = [vp, vp, i32, i64, vp, vp, i64, i32, i64, i32, i32, i32, ctypes.c_float, vp, vp, vp, sz, vp]
        L.idxc_sparse_attention_q4.restype = i32
        L.idxc_sparse_attention_q4.argtypes = [vp, vp, vp, vp, i64, i64, i32, i32, i32, i32, ctypes.c_float, vp, vp, vp, sz, vp]
        L.idxc_attention_weights.restype = i32
        L.idxc_attention_weights.argtypes = [vp, vp, i32, i64, vp, vp, vp, i32, i64, i32, i64, i32, i32, ctypes.c_float, vp, ctypes.c_float,
                                             vp, i64, vp]
        L.idxc_evict_select.restype = i32
        L.idxc_evict_select.argtypes = [vp, i64, vp, i64, i32, i32, vp, vp, vp]
        L.idxc_compact_rows.restype = i32
        L.idxc_compact_rows.argtypes = [vp, vp, i32, i64, i64, vp, vp, vp, i32, vp, i64, vp]
        f32 = ctypes.c_float
        L.idxc_page_tables.restype = i32
        L.idxc_page_tables.argtypes = [vp, i64, vp, vp, i64, i32, vp, i64, vp, vp, vp, vp, i64, vp, vp]
        L.idxc_page_release.restype = i32
        L.idxc_page_release.argtypes = [vp, i64, vp, vp, i64, i32, vp, i64, vp, vp]
        L.idxc_page_rows.restype = i32
        L.idxc_page_rows.argtypes = [vp, i64, i64, vp, vp, i64, i32, i32, vp, vp]
        L.idxc_paged_append.restype = i32
        L.idxc_paged_append.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp]
        L.idxc_paged_gather.restype = i32
        L.idxc_paged_gather.argtypes = [vp, vp, i64, vp, vp, vp]
        L.idxc_paged_attention_workspace_bytes.restype = sz
        L.idxc_paged_attention_workspace_bytes.argtypes = [i32, i32, i32, i32]
        L.idxc_paged_attention.restype = i32
        L.idxc_paged_attention.argtypes = [vp, vp, i64, vp, i64, vp, i64, i32, i64, i32, vp, i32, f32, vp, vp, vp, sz, vp]
        L.idxc_page_scores.restype = i32
        L.idxc_page_scores.argtypes = [vp, i64, i32, i32, i32, vp, i64, vp, i64, vp, i64, i32, i32, i32, i32, f32, vp, i64, vp, vp]
        L.idxc_selftest_bounded_wait.restype = i32
        L.idxc_selftest_bounded_wait.argtypes = [u32, vp]
        L.idxc_selftest_tmem_readout.restype = i32
        L.idxc_selftest_tmem_readout.argtypes = [u32, ctypes.POINTER(i64), vp]
        L.idxc_selftest_tmem_readout_under_mma.restype = i32
        L.idxc_selftest_tmem_readout_under_mma.argtypes = [u32, ctypes.c_int, ctypes.POINTER(i64), vp, vp]
        L.idxc_selftest_issue_rates.restype = i32
        L.idxc_selftest_issue_rates.argtypes = [u32, vp, vp]
        L.idxc_poll_device_status.restype = i32
        L.idxc_poll_device_status.argtypes = [vp]
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().idxc_status_string(int(status)).decode()


def launch_count() -> int:
    return int(lib().idxc_launch_count())


def _check(status: int, where: str):
    if status != OK:
        raise IdxcError(status, where)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _dtype_of(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float8_e4m3fn:
        return FP8_E4M3
    raise TypeError(f"q/k must be bfloat16 or float8_e4m3fn, got {t.dtype}")


def _dev(t: torch.Tensor, name: str, dtype=None):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must live on a CUDA device (this library has no CPU path)")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    return t


def prefill_workspace_bytes(q_len, L_k, H, d, k_top, dt=BF16, flags=0) -> int:
    return int(lib().idxc_prefill_workspace_bytes(q_len, L_k, H, d, k_top, dt, flags))


def decode_workspace_bytes(B, max_len, H, d, k_top, dt=BF16, flags=0) -> int:
    return int(lib().idxc_decode_workspace_bytes(B, max_len, H, d, k_top, dt, flags))


def alloc_workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _prefill_marshal(q, k, w, q_scale, k_scale, q_begin, k_top, scores_out, topk_out, workspace, flags, stream):
    _dev(q, "q"); _dev(k, "k"); _dev(w, "w", torch.float32)
    _dev(q_scale, "q_scale", torch.float32); _dev(k_scale, "k_scale", torch.float32)
    _dev(scores_out, "scores_out", torch.float32); _dev(topk_out, "topk_out", torch.int32); _dev(workspace, "workspace")
    dt = _dtype_of(q)
    if k.dtype != q.dtype:
        raise TypeError("q and k must have the same dtype")
    q_len, H, d = q.shape
    L_k = k.shape[0]
    if k.shape[1] != d or tuple(w.shape) != (q_len, H):
        raise ValueError("shape mismatch between q, k and w")
    ld = 0
    if scores_out is not None:
        if scores_out.dim() != 2 or scores_out.shape[0] != q_len:
            raise ValueError("scores_out must be [q_len, ld]")
        ld = scores_out.shape[1]
    if topk_out is not None and tuple(topk_out.shape) != (q_len, k_top):
        raise ValueError("topk_out must be [q_len, k_top]")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    return [_ptr(q), _ptr(k), _ptr(w), _ptr(q_scale), _ptr(k_scale), int(q_begin), q_len, L_k, H, d, int(k_top), dt,
            _ptr(scores_out), ld, _ptr(topk_out), _ptr(workspace), ws_bytes, int(flags), _stream(stream)]


def indexer_prefill(q, k, w, k_top, q_scale=None, k_scale=None, q_begin=0, scores_out=None, topk_out=None,
                    workspace=None, flags=0, stream=None):
    """idxc_indexer_prefill. Writes into scores_out / topk_out (either may be None, not both)."""
    args = _prefill_marshal(q, k, w, q_scale, k_scale, q_begin, k_top, scores_out, topk_out, workspace, flags, stream)
    _check(lib().idxc_indexer_prefill(*args), "idxc_indexer_prefill")


def _decode_marshal(q_step, k_cache, w, q_scale, k_scale, k_offsets, lens, max_len, k_top, scores_out, topk_out,
                    workspace, flags, stream):
    _dev(q_step, "q_step"); _dev(k_cache, "k_cache"); _dev(w, "w", torch.float32)
    _dev(q_scale, "q_scale", torch.float32); _dev(k_scale, "k_scale", torch.float32)
    _dev(k_offsets, "k_offsets", torch.int64); _dev(lens, "lens", torch.int32)
    _dev(scores_out, "scores_out", torch.float32); _dev(topk_out, "topk_out", torch.int32); _dev(workspace, "workspace")
    dt = _dtype_of(q_step)
    if k_cache.dtype != q_step.dtype:
        raise TypeError("q_step and k_cache must have the same dtype")
    B, H, d = q_step.shape
    if k_cache.shape[1] != d or tuple(w.shape) != (B, H) or k_offsets.shape[0] != B or lens.shape[0] != B:
        raise ValueError("shape mismatch between q_step, k_cache, w, k_offsets and lens")
    ld = 0
    if scores_out is not None:
        if scores_out.dim() != 2 or scores_out.shape[0] != B:
            raise ValueError("scores_out must be [B, ld]")
        ld = scores_out.shape[1]
    if topk_out is not None and tuple(topk_out.shape) != (B, k_top):
        raise ValueError("topk_out must be [B, k_top]")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    return [_ptr(q_step), _ptr(k_cache), k_cache.shape[0], _ptr(w), _ptr(q_scale), _ptr(k_scale), _ptr(k_offsets),
            _ptr(lens), B, int(max_len), H, d, int(k_top), dt, _ptr(scores_out), ld, _ptr(topk_out), _ptr(workspace),
            ws_bytes, int(flags), _stream(stream)]


def indexer_decode(q_step, k_cache, w, k_offsets, lens, max_len, k_top, q_scale=None, k_scale=None, scores_out=None,
                   topk_out=None, workspace=None, flags=0, stream=None):
    """idxc_indexer_decode. ``max_len`` is a host upper bound on ``lens``."""
    args = _decode_marshal(q_step, k_cache, w, q_scale, k_scale, k_offsets, lens, max_len, k_top, scores_out,
                           topk_out, workspace, flags, stream)
    _check(lib().idxc_indexer_decode(*args), "idxc_indexer_decode")


def indexer_decode_noalloc(q_step, k_cache, w, k_offsets, lens, max_len, k_top, topk_out, q_scale=None, k_scale=None,
                           flags=0, stream=None):
    """idxc_indexer_decode_noalloc: the decode step with the score scratch kept in an array
    built into the library, for hosts that cannot hand over (or allocate) a workspace. The
    step's scores, B * round_up(max_len, 32) * 4 bytes, must fit NOALLOC_SCRATCH_BYTES;
    calls that may overlap on the GPU share that array and race."""
    a = _decode_marshal(q_step, k_cache, w, q_scale, k_scale, k_offsets, lens, max_len, k_top, None, topk_out,
                        None, flags, stream)
    # same leading arguments as idxc_indexer_decode, without scores_out/ld and workspace/size
    args = a[:14] + [a[16], a[19], a[20]]
    _check(lib().idxc_indexer_decode_noalloc(*args), "idxc_indexer_decode_noalloc")


def topk_rows(scores, k_top, topk_out, first_len=0, len_step=0, lens=None, stream=None):
    """idxc_topk_rows on a [n_rows, ld] fp32 tensor."""
    _dev(scores, "scores", torch.float32); _dev(topk_out, "topk_out", torch.int32); _dev(lens, "lens", torch.int32)
    n_rows, ld = scores.shape
    if tuple(topk_out.shape) != (n_rows, k_top):
        raise ValueError("topk_out must be [n_rows, k_top]")
    _check(lib().idxc_topk_rows(_ptr(scores), ld, n_rows, int(first_len), int(len_step), _ptr(lens), int(k_top),
                                _ptr(topk_out), _stream(stream)), "idxc_topk_rows")


def quantize_e4m3(x, codes_out, scale_out, dst_rows=None, stream=None):
    """idxc_quantize_e4m3: x [n_tokens, ...] bf16 -> e4m3 codes (float8_e4m3fn or uint8 tensor with the same
    trailing shape) and one fp32 scale per token, written at row r or at row dst_rows[r]."""
    _dev(x, "x", torch.bfloat16); _dev(codes_out, "codes_out"); _dev(scale_out, "scale_out", torch.float32)
    _dev(dst_rows, "dst_rows", torch.int64)
    if codes_out.element_size() != 1:
        raise TypeError("codes_out must be an 8-bit tensor")
    n = x.shape[0]
    row = x.numel() // n if n else int(torch.tensor(x.shape[1:]).prod())
    if codes_out.numel() // max(codes_out.shape[0], 1) != row or scale_out.shape[0] != codes_out.shape[0]:
        raise ValueError("codes_out / scale_out rows do not match x")
    if dst_rows is None and codes_out.shape[0] < n:
        raise ValueError("codes_out has fewer rows than x")
    _check(lib().idxc_quantize_e4m3(_ptr(x), n, row, _ptr(codes_out), _ptr(scale_out), _ptr(dst_rows), _stream(stream)),
           "idxc_quantize_e4m3")


def topk_overlap(layers, pairs=None, want_rows=False, stream=None):
    """idxc_topk_overlap. layers: list of [rows, k_top] int32 index tensors; pairs: list of (a, b) layer
    indices (default: every pair a < b). Returns a [n_pairs] float64 tensor of MEAN row ratios (and, with
    want_rows and a single pair, the per-row ratios)."""
    for t in layers:
        _dev(t, "layer", torch.int32)
    rows, k_top = layers[0].shape
    if pairs is None:
        pairs = [(a, b) for a in range(len(layers)) for b in range(a + 1, len(layers))]
    dev = layers[0].device
    ptrs = torch.tensor([t.data_ptr() for t in layers], dtype=torch.int64, device=dev)
    pr = torch.tensor(pairs, dtype=torch.int32, device=dev).reshape(-1)
    mean = torch.empty((len(pairs),), dtype=torch.float64, device=dev)
    row_out = torch.empty((rows,), dtype=torch.float32, device=dev) if want_rows else None
    _check(lib().idxc_topk_overlap(_ptr(ptrs), _ptr(pr), len(pairs), rows, k_top, _ptr(mean), _ptr(row_out), _stream(stream)),
           "idxc_topk_overlap")
    return (mean, row_out) if want_rows else mean


def pattern_search_dp(S, M: int):
    """idxc_pattern_search_dp on a host [N, N] similarity matrix. Returns (pattern, value)."""
    import numpy as np
    S = np.ascontiguousarray(S, dtype=np.float64)
    N = S.shape[0]
    buf = ctypes.create_string_buffer(N)
    val = ctypes.c_double()
    _check(lib().idxc_pattern_search_dp(S.ctypes.data_as(ctypes.c_void_p), N, int(M), buf, ctypes.byref(val)),
           "idxc_pattern_search_dp")
    return buf.raw[:N].decode(), val.value


def pattern_search_greedy(N: int, K: int, eval_loss, want_losses: bool = False):
    """idxc_pattern_search_greedy (Algorithm 1). eval_loss(pattern: str) -> float.
    Returns (pattern, order of flipped layers, number of evaluations[, loss after each step])."""
    cb = EVAL_LOSS_FN(lambda p, n, user: float(eval_loss(p[:n].decode())))
    buf = ctypes.create_string_buffer(N)
    order = (ctypes.c_int * max(K, 1))()
    losses = (ctypes.c_double * max(K, 1))()
    evals = ctypes.c_int64()
    _check(lib().idxc_pattern_search_greedy(N, K, cb, None, buf, order, losses, ctypes.byref(evals)), "idxc_pattern_search_greedy")
    out = (buf.raw[:N].decode(), list(order)[:K], evals.value)
    return out + (list(losses)[:K],) if want_losses else out


def distill_kl(scores, targets, first_len=1, len_step=1, topk=None, want_rows=False, stream=None):
    """idxc_distill_kl: the multi-layer distillation loss (Eq. 1). scores [rows, ld] fp32; targets: list of
    [rows, ld] fp32 distributions; topk: optional [rows, k] int32. Returns the loss as a 1-element float64 device
    tensor (and the per-row values with want_rows)."""
    _dev(scores, "scores", torch.float32); _dev(topk, "topk", torch.int32)
    rows, ld = scores.shape
    for t in targets:
        _dev(t, "target", torch.float32)
        if tuple(t.shape) != (rows, ld):
            raise ValueError("targets must have the shape of scores")
    ptrs = (ctypes.c_void_p * len(targets))(*[t.data_ptr() for t in targets])
    loss = torch.empty((1,), dtype=torch.float64, device=scores.device)
    row_out = torch.empty((rows,), dtype=torch.float32, device=scores.device) if want_rows else None
    k_top = 0 if topk is None else topk.shape[1]
    _check(lib().idxc_distill_kl(_ptr(scores), ld, rows, int(first_len), int(len_step), ptrs, len(targets), _ptr(topk), k_top,
                                 _ptr(loss), _ptr(row_out), _stream(stream)), "idxc_distill_kl")
    return (loss, row_out) if want_rows else loss


def sparse_attention(q, kv, topk, d_v, scale, kv_base=None, want_lse=True, out=None, workspace=None, stream=None):
    """idxc_sparse_attention: attention of q [n_q, H, d_qk] bf16 over the rows of kv [n_kv, d_qk] bf16 named by
    topk [n_q, k_top] int32 (entries < 0 skipped); values are the leading d_v columns of the same rows.
    Returns (out [n_q, H, d_v] bf16, lse [n_q, H] fp32 or None)."""
    _dev(q, "q", torch.bfloat16); _dev(kv, "kv", torch.bfloat16); _dev(topk, "topk", torch.int32)
    _dev(kv_base, "kv_base", torch.int64)
    n_q, H, d_qk = q.shape
    n_kv = kv.shape[0]
    if kv.shape[1] != d_qk or topk.shape[0] != n_q:
        raise ValueError("kv must be [n_kv, d_qk] and topk [n_q, k_top]")
    if out is None:
        out = torch.empty((n_q, H, d_v), dtype=torch.bfloat16, device=q.device)
    lse = torch.empty((n_q, H), dtype=torch.float32, device=q.device) if want_lse else None
    need = int(lib().idxc_sparse_attention_workspace_bytes(n_q, topk.shape[1]))
    if workspace is None:
        workspace = alloc_workspace(max(need, 256), q.device)
    _check(lib().idxc_sparse_attention(_ptr(q), _ptr(kv), _ptr(topk), _ptr(kv_base), n_q, n_kv, H, d_qk, int(d_v), topk.shape[1],
                                       ctypes.c_float(scale), _ptr(out), _ptr(lse), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                       _stream(stream)), "idxc_sparse_attention")
    return out, lse


# ------------------------------------------------------------------ latent cache: 4-bit rows, dense attention, eviction
_NO_GUARD = contextlib.nullcontext()


def _launch_on(stream, **tensors):
    """Checks that the tensors (None allowed, not the first) are contiguous CUDA tensors of one device and returns (guard, raw
    stream): inside the guard that device is current and so is the stream, which is the device's current one unless given."""
    index = None
    for name, t in tensors.items():
        if t is None:
            continue
        if index is None:
            index = t.get_device()                               # (-1: not on a GPU)
        if index < 0 or t.get_device() != index or not t.is_contiguous():
            _dev(t, name)
            raise ValueError(f"{name} is on {t.device}, the other tensors are on cuda:{index}")
    if stream is not None:
        if stream.device.index != index:
            raise ValueError(f"the stream is on {stream.device}, the tensors are on cuda:{index}")
        return torch.cuda.stream(stream), stream.cuda_stream
    raw = torch._C._cuda_getCurrentRawStream(index)              # (torch.cuda.current_stream builds an object: 2 us a call)
    return (_NO_GUARD if torch.cuda.current_device() == index else torch.cuda.device(index)), raw


def _new3(a, b, c, dtype, device):
    """torch.empty((a, b, c)), a microsecond faster."""
    return torch.empty_strided((a, b, c), (b * c, c, 1), dtype=dtype, device=device)


def _at(t):
    """The address of a tensor for a pointer argument."""
    return None if t is None else t.data_ptr()


def _typed(t, name, dtype, shape=None):
    if t is None:
        return
    if t.dtype is not dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")


def _latent_format(kv) -> int:
    if kv.dim() == 2 and kv.dtype == torch.bfloat16 and kv.shape[1] == 576:
        return LATENT_BF16
    if kv.dim() == 2 and kv.dtype == torch.uint8 and kv.shape[1] == Q4_ROW_BYTES:
        return LATENT_Q4
    raise ValueError(f"kv must be [n_kv, 576] bfloat16 or [n_kv, {Q4_ROW_BYTES}] uint8, got {list(kv.shape)} {kv.dtype}")


def quantize_q4(x, cache_out, dst_rows=None, stream=None):
    """idxc_quantize_q4: x [n, 576] bf16 -> rows of cache_out [rows, 416] uint8, row r or row dst_rows[r] (int64)."""
    guard, stream = _launch_on(stream, x=x, cache_out=cache_out, dst_rows=dst_rows)
    if x.dim() != 2 or cache_out.dim() != 2:
        raise ValueError("x must be [n, 576] and cache_out [rows, 416]")
    n = x.shape[0]
    _typed(x, "x", torch.bfloat16, (n, 576)); _typed(cache_out, "cache_out", torch.uint8, (cache_out.shape[0], Q4_ROW_BYTES))
    _typed(dst_rows, "dst_rows", torch.int64, (n,))
    with guard:
        _check(lib().idxc_quantize_q4(_at(x), n, _at(cache_out), cache_out.shape[0], _at(dst_rows), stream), "idxc_quantize_q4")


def dequantize_q4(cache, out, src_rows=None, stream=None):
    """idxc_dequantize_q4: out [n, 576] bf16, row r = the values of cache row r, or of row src_rows[r] (int64)."""
    guard, stream = _launch_on(stream, cache=cache, out=out, src_rows=src_rows)
    if cache.dim() != 2 or out.dim() != 2:
        raise ValueError("cache must be [rows, 416] and out [n, 576]")
    n = out.shape[0]
    _typed(out, "out", torch.bfloat16, (n, 576)); _typed(cache, "cache", torch.uint8, (cache.shape[0], Q4_ROW_BYTES))
    _typed(src_rows, "src_rows", torch.int64, (n,))
    with guard:
        _check(lib().idxc_dequantize_q4(_at(cache), cache.shape[0], _at(src_rows), n, _at(out), stream), "idxc_dequantize_q4")


def latent_attention_workspace_bytes(B, n_step, max_len, H) -> int:
    return lib().idxc_latent_attention_workspace_bytes(int(B), int(n_step), int(max_len), int(H))


def _latent_workspace(workspace, B, n_step, max_len, H, device):
    if workspace is None:
        workspace = torch.empty_strided((max(latent_attention_workspace_bytes(B, n_step, max_len, H), 256),), (1,), dtype=torch.uint8, device=device)
    return workspace


def latent_attention(q, kv, kv_base, lens, max_len, d_v, scale, want_lse=True, out=None, workspace=None, stream=None):
    """idxc_latent_attention: q [B, n_step, H, 576] bf16 over each sequence's rows of kv ([n_kv, 576] bf16 or [n_kv, 416] uint8
    4-bit rows), rows kv_base[b] .. kv_base[b] + lens[b] - 1 (kv_base None: 0). The n_step new tokens are the last rows; token i
    sees lens[b] - (n_step - 1 - i) of them. ``max_len`` is a host upper bound on lens.
    Returns (out [B, n_step, H, d_v] bf16, lse [B, n_step, H] fp32 or None)."""
    guard, stream = _launch_on(stream, q=q, kv=kv, kv_base=kv_base, lens=lens, out=out, workspace=workspace)
    if q.dim() != 4:
        raise ValueError("q must be [B, n_step, H, 576]")
    fmt = _latent_format(kv)
    B, n_step, H, d_qk = q.shape
    _typed(q, "q", torch.bfloat16); _typed(kv_base, "kv_base", torch.int64, (B,)); _typed(lens, "lens", torch.int32, (B,))
    _typed(out, "out", torch.bfloat16, (B, n_step, H, d_v))
    with guard:
        if out is None:
            out = torch.empty_strided((B, n_step, H, d_v), (n_step * H * d_v, H * d_v, d_v, 1), dtype=torch.bfloat16, device=q.device)
        lse = _new3(B, n_step, H, torch.float32, q.device) if want_lse else None
        workspace = _latent_workspace(workspace, B, n_step, max_len, H, q.device)
        _check(lib().idxc_latent_attention(_at(q), _at(kv), fmt, kv.shape[0], _at(kv_base), _at(lens), B, n_step, int(max_len), H, d_qk,
                                           int(d_v), float(scale), _at(out), _at(lse), _at(workspace), workspace.nbytes,
                                           stream), "idxc_latent_attention")
    return out, lse


def sparse_attention_q4(q, kv, topk, d_v, scale, kv_base=None, want_lse=True, out=None, workspace=None, stream=None):
    """idxc_sparse_attention_q4: sparse_attention over a cache of 4-bit rows, kv [n_kv, 416] uint8.
    Returns (out [n_q, H, d_v] bf16, lse [n_q, H] fp32 or None)."""
    guard, stream = _launch_on(stream, q=q, kv=kv, topk=topk, kv_base=kv_base, out=out, workspace=workspace)
    if q.dim() != 3 or topk.dim() != 2 or _latent_format(kv) != LATENT_Q4:
        raise ValueError("q must be [n_q, H, 576], topk [n_q, k_top] and kv [n_kv, 416] uint8")
    n_q, H, d_qk = q.shape
    k_top = topk.shape[1]
    _typed(q, "q", torch.bfloat16); _typed(topk, "topk", torch.int32, (n_q, k_top)); _typed(kv_base, "kv_base", torch.int64, (n_q,))
    _typed(out, "out", torch.bfloat16, (n_q, H, d_v))
    with guard:
        if out is None:
            out = _new3(n_q, H, d_v, torch.bfloat16, q.device)
        lse = torch.empty_strided((n_q, H), (H, 1), dtype=torch.float32, device=q.device) if want_lse else None
        workspace = _latent_workspace(workspace, n_q, 1, k_top, H, q.device)
        _check(lib().idxc_sparse_attention_q4(_at(q), _at(kv), _at(topk), _at(kv_base), n_q, kv.shape[0], H, d_qk, int(d_v), k_top,
                                              float(scale), _at(out), _at(lse), _at(workspace), workspace.nbytes,
                                              stream), "idxc_sparse_attention_q4")
    return out, lse


def attention_weights(q, kv, lse, acc, scale, kv_base=None, lens=None, max_len=None, topk=None, beta=1.0, stream=None):
    """idxc_attention_weights: adds to acc [B, ld] fp32, in place, the probability every cached position received from
    q [B, n_step, H, 576] (or [B, H, 576] for n_step = 1), given the attention's lse. Dense: lens and max_len; acc is scaled by beta first, over each sequence's own
    positions. Selected: topk [B, k_top] int32, beta = 1."""
    guard, stream = _launch_on(stream, q=q, kv=kv, lse=lse, acc=acc, kv_base=kv_base, lens=lens, topk=topk)
    if q.dim() == 3:
        q, lse = q.unsqueeze(1), lse.unsqueeze(1)
    if q.dim() != 4 or acc.dim() != 2 or (topk is not None and topk.dim() != 2):
        raise ValueError("q must be [B, n_step, H, 576], acc [B, ld] and topk [B, k_top]")
    if (lens is None) == (topk is None) or (lens is not None and max_len is None):
        raise ValueError("give either lens and max_len, or topk")
    fmt = _latent_format(kv)
    B, n_step, H, d_qk = q.shape
    _typed(q, "q", torch.bfloat16); _typed(kv_base, "kv_base", torch.int64, (B,)); _typed(lens, "lens", torch.int32, (B,))
    _typed(lse, "lse", torch.float32, (B, n_step, H)); _typed(acc, "acc", torch.float32, (B, acc.shape[1]))
    k_top = 0 if topk is None else topk.shape[1]
    _typed(topk, "topk", torch.int32, (B, k_top))
    with guard:
        _check(lib().idxc_attention_weights(_at(q), _at(kv), fmt, kv.shape[0], _at(kv_base), _at(lens), _at(topk), k_top, B, n_step,
                                            0 if max_len is None else int(max_len), H, d_qk, float(scale), _at(lse),
                                            float(beta), _at(acc), acc.shape[1], stream), "idxc_attention_weights")


def evict_select(acc, lens, budget, recent, keep_out, new_lens_out, stream=None):
    """idxc_evict_select: acc [B, ld] fp32, lens [B] int32 -> keep_out [B, budget] int32 (ascending, -1 padded), new_lens_out [B]."""
    guard, stream = _launch_on(stream, acc=acc, lens=lens, keep_out=keep_out, new_lens_out=new_lens_out)
    if acc.dim() != 2:
        raise ValueError("acc must be [B, ld]")
    B, ld = acc.shape
    _typed(acc, "acc", torch.float32); _typed(lens, "lens", torch.int32, (B,)); _typed(new_lens_out, "new_lens_out", torch.int32, (B,))
    _typed(keep_out, "keep_out", torch.int32, (B, budget))
    with guard:
        _check(lib().idxc_evict_select(_at(acc), ld, _at(lens), B, int(budget), int(recent), _at(keep_out), _at(new_lens_out),
                                       stream), "idxc_evict_select")


def compact_rows(src, dst, keep, n_keep, src_base, dst_base=None, stream=None):
    """idxc_compact_rows: row dst_base[b] + j of dst <- row src_base[b] + keep[b, j] of src, j < n_keep[b]. dst may be src
    itself (in place; dst_base must then be left out or be src_base)."""
    if dst_base is None:
        dst_base = src_base
    guard, stream = _launch_on(stream, src=src, dst=dst, keep=keep, n_keep=n_keep, src_base=src_base, dst_base=dst_base)
    if keep.dim() != 2:
        raise ValueError("keep must be [B, ld_keep]")
    B, ld_keep = keep.shape
    if src.dtype != dst.dtype or src.shape[1:] != dst.shape[1:]:
        raise ValueError("src and dst must have rows of the same type and shape")
    row_bytes = src.element_size()
    for n in src.shape[1:]:
        row_bytes *= n
    _typed(keep, "keep", torch.int32); _typed(n_keep, "n_keep", torch.int32, (B,))
    _typed(src_base, "src_base", torch.int64, (B,)); _typed(dst_base, "dst_base", torch.int64, (B,))
    with guard:
        _check(lib().idxc_compact_rows(_at(src), _at(dst), row_bytes, src.shape[0], dst.shape[0], _at(src_base), _at(dst_base), _at(keep),
                                       ld_keep, _at(n_keep), B, stream), "idxc_compact_rows")


# ------------------------------------------------------------------ paged key/value cache
def page_tables(table, lens, new_tokens, free_pages, free_count, page_size, slots_out, token_begin_out, start_out, seq_out=None, stream=None):
    """idxc_page_tables: pages for new_tokens[b] more positions of every request, taken from the stack free_pages[:free_count]. table [B, ld]
    int32, lens [B] int32 and free_count [1] int32 are brought up to date in place; slots_out [n] int64 (and seq_out [n] int32) get one
    entry per new token, requests one after the other, -1 behind the last; token_begin_out [B + 1] int32; start_out [B] int32: a request's length
    before, or -1 if it is refused (the stack, the table or slots_out too small for it and those in front of it)."""
    guard, stream = _launch_on(stream, table=table, lens=lens, new_tokens=new_tokens, free_pages=free_pages, free_count=free_count, slots_out=slots_out,
                               token_begin_out=token_begin_out, start_out=start_out, seq_out=seq_out)
    if table.dim() != 2 or free_pages.dim() != 1 or slots_out.dim() != 1:
        raise ValueError("table must be [B, ld], free_pages [capacity] and slots_out [n]")
    B, ld = table.shape
    n = slots_out.shape[0]
    _typed(table, "table", torch.int32); _typed(lens, "lens", torch.int32, (B,)); _typed(new_tokens, "new_tokens", torch.int32, (B,))
    _typed(free_pages, "free_pages", torch.int32); _typed(free_count, "free_count", torch.int32, (1,)); _typed(slots_out, "slots_out", torch.int64)
    _typed(token_begin_out, "token_begin_out", torch.int32, (B + 1,)); _typed(start_out, "start_out", torch.int32, (B,))
    _typed(seq_out, "seq_out", torch.int32, (n,))
    with guard:
        _check(lib().idxc_page_tables(_at(table), ld, _at(lens), _at(new_tokens), B, int(page_size), _at(free_pages), free_pages.shape[0], _at(free_count),
                                      _at(token_begin_out), _at(start_out), _at(slots_out), n, _at(seq_out), stream), "idxc_page_tables")


def page_release(table, lens, keep_lens, free_pages, free_count, page_size, stream=None):
    """idxc_page_release: every request cut to its first keep_lens[b] positions (None: 0); pages that hold none of them go back to the stack.
    table, lens, free_pages and free_count change in place."""
    guard, stream = _launch_on(stream, table=table, lens=lens, keep_lens=keep_lens, free_pages=free_pages, free_count=free_count)
    if table.dim() != 2 or free_pages.dim() != 1:
        raise ValueError("table must be [B, ld] and free_pages [capacity]")
    B, ld = table.shape
    _typed(table, "table", torch.int32); _typed(lens, "lens", torch.int32, (B,)); _typed(keep_lens, "keep_lens", torch.int32, (B,))
    _typed(free_pages, "free_pages", torch.int32); _typed(free_count, "free_count", torch.int32, (1,))
    with guard:
        _check(lib().idxc_page_release(_at(table), ld, _at(lens), _at(keep_lens), B, int(page_size), _at(free_pages), free_pages.shape[0], _at(free_count),
                                       stream), "idxc_page_release")


def page_rows(table, positions, page_size, out, seq=None, stream=None):
    """idxc_page_rows: out [n, k] int32 = rows of a paged cache for positions [n, k] int32 of request seq[r] (None: r); -1 stays -1. With it
    sparse_attention and sparse_attention_q4 read paged latent caches: topk = out, kv_base = None."""
    guard, stream = _launch_on(stream, table=table, positions=positions, out=out, seq=seq)
    if table.dim() != 2 or positions.dim() != 2:
        raise ValueError("table must be [B, ld] and positions [n, k]")
    n, k = positions.shape
    _typed(table, "table", torch.int32); _typed(positions, "positions", torch.int32); _typed(out, "out", torch.int32, (n, k))
    _typed(seq, "seq", torch.int32, (n,))
    with guard:
        _check(lib().idxc_page_rows(_at(table), table.shape[1], table.shape[0], _at(seq), _at(positions), n, k, int(page_size), _at(out), stream),
               "idxc_page_rows")


class _PagedCacheStruct(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("bounds", ctypes.c_void_p),
                ("n_pages", ctypes.c_int64), ("page_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("page_size", ctypes.c_int32), ("H_kv", ctypes.c_int32), ("d", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class PagedCache:
    """idxc_paged_cache: keys and values [n_pages, page_size, H_kv, d] of one paged cache, bf16, or float8_e4m3fn with k_scale and v_scale
    [n_pages, H_kv, page_size] fp32; optionally the pages' bounds [n_pages, H_kv, 2, d] bf16. k and v may be strided views with the same strides
    (heads in front of tokens, keys and values interleaved), as long as the d columns lie side by side. Holds the tensors, copies nothing."""

    def __init__(self, k, v, k_scale=None, v_scale=None, bounds=None):
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype:
            raise ValueError("k and v must be [n_pages, page_size, H_kv, d] of one type")
        dt = _dtype_of(k)
        n_pages, page_size, H_kv, d = k.shape
        if not k.is_cuda:
            raise ValueError("k must live on a CUDA device (this library has no CPU path)")
        for name, t in (("v", v), ("k_scale", k_scale), ("v_scale", v_scale), ("bounds", bounds)):
            if t is not None and t.device != k.device:
                raise ValueError(f"{name} is on {t.device}, k is on {k.device}")
        strides = []
        for t in (k, v):
            row, own = d, list(t.stride())
            if own[3] != 1 and d > 1:
                raise ValueError("the columns of k and v must lie side by side")
            for axis in (2, 1, 0):              # an axis of length 1 may have any stride: it gets the one it would have without gaps
                if t.shape[axis] == 1:
                    own[axis] = row
                row = max(row, own[axis] * t.shape[axis])
            strides.append(own)
        if strides[0] != strides[1]:
            raise ValueError(f"k and v must have the same strides, got {k.stride()} and {v.stride()}")
        if (dt == FP8_E4M3) != (k_scale is not None) or (k_scale is None) != (v_scale is None):
            raise ValueError("float8_e4m3fn rows need k_scale and v_scale, bf16 rows have none")
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
            _typed(t, name, torch.float32, (n_pages, H_kv, page_size))
        _typed(bounds, "bounds", torch.bfloat16, (n_pages, H_kv, 2, d))
        for name, t in (("k_scale", k_scale), ("v_scale", v_scale), ("bounds", bounds)):
            if t is not None and not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous")
        self.k, self.v, self.k_scale, self.v_scale, self.bounds = k, v, k_scale, v_scale, bounds
        self.n_pages, self.page_size, self.H_kv, self.d = n_pages, page_size, H_kv, d
        self.device, self.device_index = k.device, k.get_device()
        self._workspace_bytes = {}               # by (n_step, H)
        self._c = _PagedCacheStruct(_at(k), _at(v), _at(k_scale), _at(v_scale), _at(bounds), n_pages, *strides[0][:3], page_size, H_kv, d, dt)
        self._p = ctypes.addressof(self._c)


def _token_stride(t, name, heads, d, index):
    """Checks that t [..., heads, d] is bf16 on the device, with heads and columns side by side and one stride for all its tokens, and returns that stride."""
    if t.dtype is not torch.bfloat16:
        raise TypeError(f"{name}: expected {torch.bfloat16}, got {t.dtype}")
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, the cache is on cuda:{index}")
    shape, stride = t.shape, t.stride()
    if shape[-2:] != (heads, d):
        raise ValueError(f"{name} must be [..., {heads}, {d}], got {list(shape)}")
    if t.is_contiguous():
        return heads * d
    if stride[-1] != 1 or (heads > 1 and stride[-2] != d):
        raise ValueError(f"the heads and columns of {name} must lie side by side")
    step, n = heads * d, 1                                      # tokens of the inner axes so far, and their stride
    for axis in range(t.dim() - 3, -1, -1):
        if shape[axis] == 1:
            continue
        if n == 1:
            step = stride[axis]
        elif stride[axis] != step * n:
            raise ValueError(f"the tokens of {name} must be one stride apart")
        n *= shape[axis]
    return step if n > 1 else max(step, heads * d)


def _on_cache(cache, stream, **tensors):
    """_launch_on for calls whose device is the cache's."""
    index = cache.device_index
    for t in tensors.values():
        if t is not None and (t.get_device() != index or not t.is_contiguous()):
            for name, t in tensors.items():
                _dev(t, name)
                if t is not None and t.get_device() != index:
                    raise ValueError(f"{name} is on {t.device}, the cache is on cuda:{index}")
    if stream is not None:
        if stream.device.index != index:
            raise ValueError(f"the stream is on {stream.device}, the cache is on cuda:{index}")
        return torch.cuda.stream(stream), stream.cuda_stream
    raw = torch._C._cuda_getCurrentRawStream(index)
    return (_NO_GUARD if torch.cuda.current_device() == index else torch.cuda.device(index)), raw


def paged_append(cache, k, v, slots, stream=None):
    """idxc_paged_append: k, v [n, H_kv, d] bf16 (tokens any stride apart) written to slots [n] int64 of a PagedCache, in 8 bits with their scales; the
    bounds of the pages written to are brought up to date if the cache has them. Slots outside the cache are skipped."""
    guard, stream = _on_cache(cache, stream, slots=slots)
    n = slots.shape[0]
    _typed(slots, "slots", torch.int64, (n,))
    if k.dim() != 3 or v.dim() != 3 or k.shape[0] != n or v.shape[0] != n:
        raise ValueError(f"k and v must be [{n}, {cache.H_kv}, {cache.d}]")
    k_stride = _token_stride(k, "k", cache.H_kv, cache.d, cache.device_index)
    v_stride = _token_stride(v, "v", cache.H_kv, cache.d, cache.device_index)
    with guard:
        _check(lib().idxc_paged_append(cache._p, _at(k), k_stride, _at(v), v_stride, _at(slots), n, stream), "idxc_paged_append")


def paged_gather(cache, slots, k_out, v_out, stream=None):
    """idxc_paged_gather: rows slots [n] int64 of a PagedCache read into k_out, v_out [n, H_kv, d] bf16; zeros for slots outside the cache."""
    guard, stream = _on_cache(cache, stream, slots=slots, k_out=k_out, v_out=v_out)
    n = slots.shape[0]
    _typed(slots, "slots", torch.int64, (n,))
    _typed(k_out, "k_out", torch.bfloat16, (n, cache.H_kv, cache.d)); _typed(v_out, "v_out", torch.bfloat16, (n, cache.H_kv, cache.d))
    with guard:
        _check(lib().idxc_paged_gather(cache._p, _at(slots), n, _at(k_out), _at(v_out), stream), "idxc_paged_gather")


def paged_attention_workspace_bytes(n_step, H, H_kv, d) -> int:
    return lib().idxc_paged_attention_workspace_bytes(int(n_step), int(H), int(H_kv), int(d))


def paged_attention(cache, q, table, lens, max_len, scale, pages=None, want_lse=True, out=None, workspace=None, stream=None):
    """idxc_paged_attention: q [B, n_step, H, d] bf16 (tokens any one stride apart) over the requests' pages of a PagedCache, H / H_kv query heads to a
    key head; the n_step new tokens are the last positions, and token i sees lens[b] - (n_step - 1 - i) of them. table [B, ld] int32, lens [B] int32,
    ``max_len`` a host bound on lens. pages [B, H_kv, n_sel] (or [B * H_kv, n_sel]) int32: only the positions of these logical pages.
    Returns (out [B, n_step, H, d] bf16, lse [B, n_step, H] fp32 or None)."""
    guard, stream = _on_cache(cache, stream, table=table, lens=lens, pages=pages, out=out, workspace=workspace)
    if q.dim() != 4 or table.dim() != 2:
        raise ValueError("q must be [B, n_step, H, d] and table [B, ld]")
    B, n_step, H, d = q.shape
    q_stride = _token_stride(q, "q", H, cache.d, cache.device_index)
    ld = table.shape[1]
    _typed(table, "table", torch.int32, (B, ld)); _typed(lens, "lens", torch.int32, (B,)); _typed(out, "out", torch.bfloat16, (B, n_step, H, d))
    n_sel = 0
    if pages is not None:
        n_sel = pages.shape[-1]
        _typed(pages, "pages", torch.int32, (B, cache.H_kv, n_sel) if pages.dim() == 3 else (B * cache.H_kv, n_sel))
    with guard:
        if out is None:
            out = torch.empty_strided((B, n_step, H, d), (n_step * H * d, H * d, d, 1), dtype=torch.bfloat16, device=cache.device)
        lse = _new3(B, n_step, H, torch.float32, cache.device) if want_lse else None
        if workspace is None:
            need = cache._workspace_bytes.get((n_step, H))
            if need is None:
                need = cache._workspace_bytes[n_step, H] = max(paged_attention_workspace_bytes(n_step, H, cache.H_kv, d), 256)
            workspace = torch.empty_strided((need,), (1,), dtype=torch.uint8, device=cache.device)
        else:
            need = workspace.nbytes
        _check(lib().idxc_paged_attention(cache._p, _at(q), q_stride, _at(table), ld, _at(lens), B, n_step, int(max_len), H, _at(pages), n_sel, float(scale),
                                          _at(out), _at(lse), _at(workspace), need, stream), "idxc_paged_attention")
    return out, lse


def page_scores(bounds, q, table, lens, page_size, scale, scores_out, n_pages_out, keep_first=1, keep_last=1, stream=None):
    """idxc_page_scores: the largest score that a key between a page's bounds could reach, for every page of every request and key head. bounds
    [n_pages, H_kv, 2, d] bf16, q [B, n_step, H, d] bf16 -> scores_out [B * H_kv, ld] fp32, n_pages_out [B * H_kv] int32, which topk_rows takes as
    scores and lens; its selection is paged_attention's pages. The first keep_first and last keep_last pages score 3e38."""
    guard, stream = _launch_on(stream, bounds=bounds, table=table, lens=lens, scores_out=scores_out, n_pages_out=n_pages_out)
    if q.dim() != 4 or table.dim() != 2 or bounds.dim() != 4 or scores_out.dim() != 2:
        raise ValueError("bounds must be [n_pages, H_kv, 2, d], q [B, n_step, H, d], table [B, ld] and scores_out [B * H_kv, ld]")
    n_pages, H_kv, _, d = bounds.shape
    B, n_step, H, _ = q.shape
    _typed(bounds, "bounds", torch.bfloat16, (n_pages, H_kv, 2, d))
    q_stride = _token_stride(q, "q", H, d, bounds.get_device())
    _typed(table, "table", torch.int32, (B, table.shape[1])); _typed(lens, "lens", torch.int32, (B,))
    _typed(scores_out, "scores_out", torch.float32, (B * H_kv, scores_out.shape[1])); _typed(n_pages_out, "n_pages_out", torch.int32, (B * H_kv,))
    with guard:
        _check(lib().idxc_page_scores(_at(bounds), n_pages, int(page_size), H_kv, d, _at(q), q_stride, _at(table), table.shape[1], _at(lens), B, n_step, H,
                                      int(keep_first), int(keep_last), float(scale), _at(scores_out), scores_out.shape[1], _at(n_pages_out), stream),
               "idxc_page_scores")


def selftest_bounded_wait(wait_cycles: int = 1_000_000, stream=None):
    """idxc_selftest_bounded_wait: enqueue a kernel whose wait can never be satisfied; the next
    poll_device_status() must raise IdxcError(ERR_DEVICE_TIMEOUT)."""
    _check(lib().idxc_selftest_bounded_wait(int(wait_cycles), _stream(stream)), "idxc_selftest_bounded_wait")


def selftest_tmem_readout(accumulators_per_warp: int, stream=None) -> int:
    """idxc_selftest_tmem_readout: enqueue the tensor-memory read-out measurement kernel; returns the accumulator bytes
    the launch reads over all SMs (time the call with CUDA events)."""
    nbytes = ctypes.c_int64()
    _check(lib().idxc_selftest_tmem_readout(int(accumulators_per_warp), ctypes.byref(nbytes), _stream(stream)),
           "idxc_selftest_tmem_readout")
    return int(nbytes.value)


def selftest_tmem_readout_under_mma(accumulators_per_warp: int, fp8: bool, counters, stream=None) -> int:
    """idxc_selftest_tmem_readout_under_mma: the read-out measurement with MMAs running beside it; counters is a device
    int64 tensor of two entries (accumulator fills completed, cycles of the slowest reader). Returns the bytes read."""
    _dev(counters, "counters", torch.int64)
    nbytes = ctypes.c_int64()
    _check(lib().idxc_selftest_tmem_readout_under_mma(int(accumulators_per_warp), int(bool(fp8)), ctypes.byref(nbytes),
                                                      _ptr(counters), _stream(stream)), "idxc_selftest_tmem_readout_under_mma")
    return int(nbytes.value)


ISSUE_RATE_KINDS = ("fmnmx", "fadd_abs", "ffma", "ffma2_packed", "fsetp_sel_pair", "lop3", "shfl")


def selftest_issue_rates(rounds: int = 4096, stream=None) -> dict:
    """idxc_selftest_issue_rates: scheduler cycles per warp instruction for seven instruction kinds (two warps per
    scheduler). Synchronises the stream to read the counters back."""
    s = torch.cuda.current_stream() if stream is None else stream
    cycles = torch.zeros(len(ISSUE_RATE_KINDS), dtype=torch.int64, device=f"cuda:{torch.cuda.current_device()}")
    _check(lib().idxc_selftest_issue_rates(int(rounds), _ptr(cycles), _stream(s)), "idxc_selftest_issue_rates")
    s.synchronize()
    c = cycles.tolist()
    return {name: c[i] / (rounds * (8 if name == "ffma2_packed" else 16) * 2.0) for i, name in enumerate(ISSUE_RATE_KINDS)}


def poll_device_status(stream=None):
    """Synchronises the stream and raises if a kernel recorded a bounded-wait timeout."""
    _check(lib().idxc_poll_device_status(_stream(stream)), "idxc_poll_device_status")


class Schedule:
    """idxc_schedule: the Full/Shared layer pattern and the cached index tensor (host state)."""

    def __init__(self, pattern: str):
        self._h = ctypes.c_void_p()
        self.pattern = pattern
        raw = pattern.encode("ascii", errors="replace")
        _check(lib().idxc_schedule_create(raw, len(raw), ctypes.byref(self._h)), "idxc_schedule_create")
        self._keep = {}          # topk buffers by data_ptr, so a returned alias can be mapped back to its tensor

    def close(self):
        if self._h:
            lib().idxc_schedule_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def begin_pass(self):
        self._keep.clear()
        _check(lib().idxc_schedule_begin_pass(self._h), "idxc_schedule_begin_pass")

    def source(self, layer: int) -> int:
        out = ctypes.c_int()
        _check(lib().idxc_schedule_source(self._h, layer, ctypes.byref(out)), "idxc_schedule_source")
        return out.value

    def stats(self):
        nf, ns, calls = ctypes.c_int(), ctypes.c_int(), ctypes.c_int64()
        _check(lib().idxc_schedule_stats(self._h, ctypes.byref(nf), ctypes.byref(ns), ctypes.byref(calls)),
               "idxc_schedule_stats")
        return nf.value, ns.value, calls.value

    def _result(self, res_ptr, topk_buf):
        if topk_buf is not None:
            self._keep[topk_buf.data_ptr()] = topk_buf
        t = self._keep.get(res_ptr.value)
        if t is None:
            raise RuntimeError("schedule returned a pointer to a buffer this object has not seen")
        return t

    def prefill_layer(self, layer, q=None, k=None, w=None, k_top=0, q_scale=None, k_scale=None, q_begin=0, q_len=None,
                      scores_out=None, topk_buf=None, workspace=None, flags=0, stream=None):
        """One layer of a prefill pass. S layers need only k_top and q_len (inputs may be None).
        Returns the tensor holding this layer's indices (the F layer's buffer on S layers)."""
        res = ctypes.c_void_p()
        if q is None:
            if q_len is None:
                raise ValueError("q_len is required when q is None")
            args = [None, None, None, None, None, int(q_begin), int(q_len), 0, 0, 0, int(k_top), BF16, None, 0,
                    _ptr(_dev(topk_buf, "topk_buf", torch.int32)), None, 0, int(flags), _stream(stream)]
        else:
            args = _prefill_marshal(q, k, w, q_scale, k_scale, q_begin, k_top, scores_out, topk_buf, workspace, flags, stream)
        _check(lib().idxc_schedule_prefill_layer(self._h, layer, *args, ctypes.byref(res)), "idxc_schedule_prefill_layer")
        return self._result(res, topk_buf)

    def decode_layer(self, layer, q_step=None, k_cache=None, w=None, k_offsets=None, lens=None, max_len=0, k_top=0,
                     q_scale=None, k_scale=None, B=None, scores_out=None, topk_buf=None, workspace=None, flags=0,
                     stream=None):
        res = ctypes.c_void_p()
        if q_step is None:
            if B is None:
                raise ValueError("B is required when q_step is None")
            args = [None, None, 0, None, None, None, None, None, int(B), int(max_len), 0, 0, int(k_top), BF16, None, 0,
                    _ptr(_dev(topk_buf, "topk_buf", torch.int32)), None, 0, int(flags), _stream(stream)]
        else:
            args = _decode_marshal(q_step, k_cache, w, q_scale, k_scale, k_offsets, lens, max_len, k_top, scores_out,
                                   topk_buf, workspace, flags, stream)
        _check(lib().idxc_schedule_decode_layer(self._h, layer, *args, ctypes.byref(res)), "idxc_schedule_decode_layer")
        return self._result(res, topk_buf)
