"""Thin Python binding of libatts (ctypes): argument marshalling only.

Every function takes torch CUDA tensors, passes their device pointers and the current
CUDA stream to the C entry point of the same name (include/atts.h), and raises
:class:`AttsError` on a non-zero status.  Nothing is computed here, and there is no
fallback: if the CUDA library cannot be loaded, loading raises.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_void_p, c_char_p, POINTER, c_uint32

from . import build as _build

EXPORTS = (
    "atts_strerror", "atts_version", "atts_score_workspace_bytes", "atts_score_logprob",
    "atts_conformal_rank", "atts_classify", "atts_calib_workspace_bytes", "atts_calib_update",
    "atts_last_device_status", "atts_profile_begin", "atts_profile_end",
    "atts_calib_update_static", "atts_rank_classify", "atts_score_logprob_scaled", "atts_rms_inv",
    "atts_threshold", "atts_classify_threshold", "atts_conformal_rank_conditional", "atts_classify_conditional",
    "atts_debug_score_plan", "atts_debug_score_unit", "atts_score_slice", "atts_score_combine",
    "atts_calib_index_bytes", "atts_calib_index_build", "atts_calib_update_indexed", "atts_rank_classify_indexed",
    "atts_takeover_ids_workspace_bytes", "atts_takeover_ids", "atts_debug_set_wait", "atts_debug_score_form",
    "atts_tree_plan", "atts_rope_append", "atts_tree_attention_workspace_bytes", "atts_tree_attention",
    "atts_cache_weights", "atts_cache_select", "atts_cache_gather",
)

STAGE_DRAFT, STAGE_ACCEPTED, STAGE_TARGET = 1, 2, 3
DEV_TOKEN_ID_RANGE, DEV_WAIT_EXPIRED, DEV_GROUP_ID_RANGE, DEV_INDEX_STALE = 1, 2, 4, 8
DEV_PAGE_RANGE, DEV_SEQ_RANGE = 16, 32

_lib = None


class AttsError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} (status {status})")


def load(rebuild_if_stale: bool = True) -> ctypes.CDLL:
    """Load libatts.so from the package directory (building it first if the sources are newer)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB_PATH
    if rebuild_if_stale and _build.is_stale():
        # A library older than its sources is never loaded: if it cannot be rebuilt (no nvcc, or the sources no
        # longer compile) this raises, so that nothing runs on a binary that does not match the tree.
        _build.build_library()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2509_15148_b200.build`")
    lib = ctypes.CDLL(path)
    lib.atts_strerror.restype = c_char_p
    lib.atts_strerror.argtypes = [c_int]
    lib.atts_version.restype = c_int
    lib.atts_score_workspace_bytes.argtypes = [c_int64, c_int64, c_int64, c_int64, POINTER(c_size_t)]
    lib.atts_score_logprob.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int64, c_int64, c_int64,
                                       c_int32, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.atts_conformal_rank.argtypes = [c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p, c_void_p]
    lib.atts_classify.argtypes = [c_void_p, c_int64, c_int64, c_double, c_void_p, c_void_p, c_void_p]
    lib.atts_rank_classify.argtypes = [c_void_p, c_int64, c_void_p, c_int64, POINTER(c_double), c_int32, c_void_p, c_void_p,
                                       c_void_p, c_void_p, c_void_p]
    lib.atts_score_logprob_scaled.argtypes = [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int64, c_int64,
                                              c_int64, c_int32, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.atts_score_slice.argtypes = [c_void_p, c_void_p, c_void_p, c_int64, c_int64, c_int64, c_int64, c_void_p, c_void_p,
                                     c_size_t, c_void_p]
    lib.atts_score_combine.argtypes = [c_void_p, c_int64, c_void_p, c_int64, c_int64, c_int32, c_void_p, c_void_p, c_void_p,
                                       c_size_t, c_void_p]
    lib.atts_rms_inv.argtypes = [c_void_p, c_int64, c_int64, ctypes.c_float, c_void_p, c_void_p]
    lib.atts_threshold.argtypes = [c_void_p, c_int64, c_double, c_void_p, c_void_p]
    lib.atts_classify_threshold.argtypes = [c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_void_p]
    lib.atts_conformal_rank_conditional.argtypes = [c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64,
                                                    c_void_p, c_void_p, c_void_p, c_void_p]
    lib.atts_classify_conditional.argtypes = [c_void_p, c_void_p, c_int64, c_double, c_void_p, c_void_p, c_void_p]
    lib.atts_debug_score_plan.argtypes = [c_int64, c_int64, c_int64, c_int32, c_int32, POINTER(c_int32)]
    lib.atts_debug_score_unit.argtypes = [c_int64, c_int64, c_int64, c_int32, c_int32, c_int32, POINTER(c_int32)]
    lib.atts_calib_workspace_bytes.argtypes = [c_int64, c_int64, POINTER(c_size_t)]
    lib.atts_calib_update.argtypes = [c_void_p, c_int64, c_int64, c_void_p, c_int64, POINTER(c_int64), c_void_p,
                                      c_size_t, c_void_p]
    lib.atts_last_device_status.argtypes = [c_void_p, POINTER(c_uint32)]
    lib.atts_calib_update_static.argtypes = [c_void_p, c_int64, c_int64, c_void_p, c_int64, POINTER(c_int64), c_void_p]
    lib.atts_calib_index_bytes.argtypes = [c_int64, POINTER(c_size_t)]
    lib.atts_calib_index_build.argtypes = [c_void_p, c_int64, c_void_p, c_size_t, c_void_p]
    lib.atts_calib_update_indexed.argtypes = [c_void_p, c_int64, c_int64, c_void_p, c_int64, POINTER(c_int64), c_void_p,
                                              c_size_t, c_void_p, c_size_t, c_void_p]
    lib.atts_rank_classify_indexed.argtypes = [c_void_p, c_int64, c_void_p, c_int64, c_void_p, POINTER(c_double), c_int32,
                                               c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]
    lib.atts_takeover_ids_workspace_bytes.argtypes = [c_int64, POINTER(c_size_t)]
    lib.atts_takeover_ids.argtypes = [c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.atts_debug_set_wait.argtypes = [c_int64, c_int32]
    lib.atts_debug_score_form.argtypes = [c_int64, c_int64, c_int64, POINTER(c_int32)]
    lib.atts_tree_plan.argtypes = [c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_void_p]
    rows = [c_void_p, c_int64, c_int64]
    lib.atts_rope_append.argtypes = rows * 3 + [c_void_p, c_void_p, c_int32, c_float, c_int32, c_void_p, c_void_p, c_void_p,
                                                c_int64, c_int32, c_int64] + rows + [c_void_p]
    lib.atts_tree_attention_workspace_bytes.argtypes = [c_int64, c_int64, c_int32, c_int32, c_int32, c_int64, c_int64,
                                                        POINTER(c_size_t)]
    lib.atts_tree_attention.argtypes = rows + [c_void_p] * 5 + [c_int64, c_int32, c_int64, c_int64, c_float] + rows + [
        c_void_p, c_void_p, c_size_t, c_void_p]
    lib.atts_cache_weights.argtypes = rows + [c_void_p] * 6 + [c_int64, c_int32, c_int64, c_int64, c_float, c_void_p, c_void_p,
                                                                c_int64, c_void_p]
    lib.atts_cache_select.argtypes = [c_void_p, c_int64, c_void_p, c_int64, c_int32, c_int64, c_int64, c_int64, c_void_p,
                                      c_void_p, c_void_p]
    lib.atts_cache_gather.argtypes = [c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_int64, c_void_p, c_void_p]
    lib.atts_profile_begin.argtypes = [c_int]
    lib.atts_profile_end.argtypes = [POINTER(ctypes.c_float), c_int, POINTER(c_int)]
    for name in EXPORTS[2:]:
        getattr(lib, name).restype = c_int
    _lib = lib
    return lib


def strerror(status: int) -> str:
    return load().atts_strerror(int(status)).decode()


def version() -> int:
    return load().atts_version()


def _check(status: int, where: str) -> None:
    if status != 0:
        raise AttsError(status, where)


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _stream() -> int:
    """The current stream of the current device (the raw handle where torch hands it out directly: 0.1 against 3.3 us)."""
    global _raw_stream, _current_device
    if _raw_stream is None:
        import torch
        get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        _raw_stream = (lambda: torch.cuda.current_stream().cuda_stream) if get is None else (lambda: get(_current_device()))
        torch.cuda.current_device()       # the first use brings the device up
    return _raw_stream()


_raw_stream = _current_device = None


def score_workspace_bytes(M: int, d: int, V: int, S: int) -> int:
    out = c_size_t(0)
    _check(load().atts_score_workspace_bytes(M, d, V, S, ctypes.byref(out)), "atts_score_workspace_bytes")
    return out.value


def score_logprob(hidden, lm_head, token_ids, seg_offsets, token_logprob, sample_score, workspace,
                  score_mode: int = 0) -> None:
    """hidden [M,d] bf16, lm_head [V,d] bf16, token_ids [M] i32, seg_offsets [S+1] i32 ->
    token_logprob [M] f32 (or None), sample_score [S] f32; workspace: uint8 tensor."""
    M, d = hidden.shape
    V = lm_head.shape[0]
    S = seg_offsets.numel() - 1
    _check(load().atts_score_logprob(_ptr(hidden), _ptr(lm_head), _ptr(token_ids), _ptr(seg_offsets), M, d, V, S,
                                     score_mode, _ptr(token_logprob), _ptr(sample_score), _ptr(workspace),
                                     workspace.numel() * workspace.element_size(), _stream()), "atts_score_logprob")


def score_logprob_scaled(hidden, lm_head, token_ids, row_scale, seg_offsets, token_logprob, sample_score, workspace,
                         score_mode: int = 0) -> None:
    """score_logprob with logits of row i multiplied by row_scale[i] (f32 [M], finite and > 0)."""
    M, d = hidden.shape
    V = lm_head.shape[0]
    S = seg_offsets.numel() - 1
    _check(load().atts_score_logprob_scaled(_ptr(hidden), _ptr(lm_head), _ptr(token_ids), _ptr(row_scale),
                                            _ptr(seg_offsets), M, d, V, S, score_mode, _ptr(token_logprob),
                                            _ptr(sample_score), _ptr(workspace),
                                            workspace.numel() * workspace.element_size(), _stream()),
           "atts_score_logprob_scaled")


def score_slice(hidden, lm_head_slice, token_ids, vocab_offset: int, slice_stats, workspace) -> None:
    """Per-token (max, sum exp, token logit or -inf) over one vocabulary slice: slice_stats [M, 3] f32."""
    M, d = hidden.shape
    _check(load().atts_score_slice(_ptr(hidden), _ptr(lm_head_slice), _ptr(token_ids), M, d, lm_head_slice.shape[0],
                                   int(vocab_offset), _ptr(slice_stats), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream()), "atts_score_slice")


def score_combine(slice_stats, seg_offsets, token_logprob, sample_score, workspace, score_mode: int = 0) -> None:
    """Merge slice_stats [G, M, 3] (all ranks' blocks in rank order) into token log-probs and sample scores."""
    G, M = slice_stats.shape[0], slice_stats.shape[1]
    S = seg_offsets.numel() - 1
    _check(load().atts_score_combine(_ptr(slice_stats), G, _ptr(seg_offsets), M, S, score_mode, _ptr(token_logprob),
                                     _ptr(sample_score), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                     _stream()), "atts_score_combine")


def rms_inv(hidden, eps: float, row_scale) -> None:
    """row_scale[i] = 1 / sqrt(mean(hidden[i]^2) + eps)."""
    M, d = hidden.shape
    _check(load().atts_rms_inv(_ptr(hidden), M, d, float(eps), _ptr(row_scale), _stream()), "atts_rms_inv")


def threshold(calib_sorted, n: int, alpha: float, tau) -> None:
    """tau[0] = the floor(alpha (n + 1))-th largest of the first n calibration scores (+inf if that is 0)."""
    _check(load().atts_threshold(_ptr(calib_sorted), n, float(alpha), _ptr(tau), _stream()), "atts_threshold")


def classify_threshold(scores, tau, stage, stage_counts=None) -> None:
    """Stage per sample from s > tau[0]; stage_counts [3] or None."""
    _check(load().atts_classify_threshold(_ptr(scores), scores.numel(), _ptr(tau), _ptr(stage), _ptr(stage_counts),
                                          _stream()), "atts_classify_threshold")


def takeover_ids_workspace_bytes(Nc: int) -> int:
    out = c_size_t(0)
    _check(load().atts_takeover_ids_workspace_bytes(Nc, ctypes.byref(out)), "atts_takeover_ids_workspace_bytes")
    return out.value


def takeover_ids(stage, ids, count, workspace) -> None:
    """Positions (ascending, int32) of the samples in stage 3 into ids (as many as fit), their number into count[0]."""
    _check(load().atts_takeover_ids(_ptr(stage), stage.numel(), _ptr(ids), 0 if ids is None else ids.numel(), _ptr(count),
                                    _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
                                    _stream()), "atts_takeover_ids")


def conformal_rank_conditional(scores, group_ids, calib_segments, seg_offsets, numer, denom, pvalue=None) -> None:
    """Rank each score against the ascending calibration segment of its own group."""
    _check(load().atts_conformal_rank_conditional(_ptr(scores), _ptr(group_ids), scores.numel(), _ptr(calib_segments),
                                                  calib_segments.numel(), _ptr(seg_offsets), seg_offsets.numel() - 1,
                                                  _ptr(numer), _ptr(denom), _ptr(pvalue), _stream()),
           "atts_conformal_rank_conditional")


def classify_conditional(numer, denom, alpha: float, stage, stage_counts=None) -> None:
    _check(load().atts_classify_conditional(_ptr(numer), _ptr(denom), numer.numel(), float(alpha), _ptr(stage),
                                            _ptr(stage_counts), _stream()), "atts_classify_conditional")


def conformal_rank(scores, calib_sorted, n: int, numer, pvalue=None) -> None:
    """scores [Nc] f32, calib_sorted (first n entries used) -> numer [Nc] u32 (int32 storage), pvalue [Nc] f32."""
    _check(load().atts_conformal_rank(_ptr(scores), scores.numel(), _ptr(calib_sorted), n, _ptr(numer), _ptr(pvalue),
                                      _stream()), "atts_conformal_rank")


def classify(numer, n: int, alpha: float, stage, stage_counts=None) -> None:
    """numer [Nc] u32 -> stage [Nc] u8, stage_counts [3] u32 (int32 storage) or None."""
    _check(load().atts_classify(_ptr(numer), numer.numel(), n, float(alpha), _ptr(stage), _ptr(stage_counts),
                                _stream()), "atts_classify")


def rank_classify(scores, calib_sorted, n: int, alphas, numer, pvalue, stage, stage_counts=None) -> None:
    """Rank and threshold at up to four alphas in one launch: stage [len(alphas), Nc] u8, stage_counts [len(alphas), 3]."""
    arr = (c_double * len(alphas))(*[float(a) for a in alphas])
    _check(load().atts_rank_classify(_ptr(scores), scores.numel(), _ptr(calib_sorted), n, arr, len(alphas), _ptr(numer),
                                     _ptr(pvalue), _ptr(stage), _ptr(stage_counts), _stream()), "atts_rank_classify")


def calib_workspace_bytes(n: int, k: int) -> int:
    out = c_size_t(0)
    _check(load().atts_calib_workspace_bytes(n, k, ctypes.byref(out)), "atts_calib_workspace_bytes")
    return out.value


def calib_update(calib, n: int, new_scores, workspace) -> int:
    """calib: f32 buffer of capacity calib.numel() whose first n entries are sorted; inserts new_scores in place.
    Returns the new fill n + k."""
    n_out = c_int64(0)
    k = 0 if new_scores is None else new_scores.numel()
    _check(load().atts_calib_update(_ptr(calib), n, calib.numel(), _ptr(new_scores), k, ctypes.byref(n_out),
                                    _ptr(workspace), 0 if workspace is None else workspace.numel() * workspace.element_size(),
                                    _stream()), "atts_calib_update")
    return n_out.value


def _nbytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def calib_index_bytes(cap: int) -> int:
    out = c_size_t(0)
    _check(load().atts_calib_index_bytes(cap, ctypes.byref(out)), "atts_calib_index_bytes")
    return out.value


def calib_index_build(calib_sorted, n: int, index) -> None:
    """Write into `index` (uint8 tensor) the search index of the first n entries of calib_sorted."""
    _check(load().atts_calib_index_build(_ptr(calib_sorted), n, _ptr(index), _nbytes(index), _stream()),
           "atts_calib_index_build")


def calib_update_indexed(calib, n: int, new_scores, index, workspace) -> int:
    """:func:`calib_update` that also leaves in `index` the search index of the updated buffer. Returns n + k."""
    n_out = c_int64(0)
    k = 0 if new_scores is None else new_scores.numel()
    _check(load().atts_calib_update_indexed(_ptr(calib), n, calib.numel(), _ptr(new_scores), k, ctypes.byref(n_out),
                                            _ptr(index), _nbytes(index), _ptr(workspace), _nbytes(workspace), _stream()),
           "atts_calib_update_indexed")
    return n_out.value


def rank_classify_indexed(scores, calib_sorted, n: int, index, alphas, numer, pvalue=None, stage=None,
                          stage_counts=None) -> None:
    """:func:`rank_classify` with the buffer's search index; alphas may be empty (ranks and p-values only)."""
    arr = (c_double * max(len(alphas), 1))(*[float(a) for a in alphas])
    _check(load().atts_rank_classify_indexed(_ptr(scores), scores.numel(), _ptr(calib_sorted), n, _ptr(index), arr,
                                             len(alphas), _ptr(numer), _ptr(pvalue), _ptr(stage), _ptr(stage_counts),
                                             _stream()), "atts_rank_classify_indexed")


STATIC_MAX_TOTAL, STATIC_MAX_NEW = 65536, 16384


def calib_update_static(calib, n: int, new_scores) -> int:
    """Same as :func:`calib_update` without a workspace, for callers that cannot allocate device memory (an engine
    plug-in left with no free HBM, a loop that must not pay cudaMalloc's device-wide synchronisation): the scratch is
    a fixed array inside the library, so n + k <= STATIC_MAX_TOTAL and k <= STATIC_MAX_NEW (status 10 otherwise).
    All calls on a device share that array: keep them on one stream or order them, overlapping calls race.
    Make the first call on a device at start-up (it looks up the array's address). Returns n + k."""
    n_out = c_int64(0)
    k = 0 if new_scores is None else new_scores.numel()
    _check(load().atts_calib_update_static(_ptr(calib), n, calib.numel(), _ptr(new_scores), k, ctypes.byref(n_out),
                                           _stream()), "atts_calib_update_static")
    return n_out.value


def last_device_status() -> int:
    """Synchronises the current stream; returns and clears the device status bits. Raises on an expired wait or a
    stale calibration index."""
    bits = c_uint32(0)
    st = load().atts_last_device_status(_stream(), ctypes.byref(bits))
    if st != 0:
        raise AttsError(st, "atts_last_device_status")
    return bits.value


def debug_set_wait(limit_cycles: int = 0, withhold_loads: bool = False) -> None:
    """Bound (SM cycles; <= 0 restores the default) of the scoring kernel's pipeline waits for later calls, and the
    diagnostic switch that makes its producer issue no loads so that the first wait for data runs out."""
    _check(load().atts_debug_set_wait(int(limit_cycles), 1 if withhold_loads else 0), "atts_debug_set_wait")


def debug_score_form(M: int, d: int, V: int) -> int:
    """1 if score_logprob runs this shape on single CTAs on the current device, 2 if on CTA pairs."""
    out = c_int32(0)
    _check(load().atts_debug_score_form(M, d, V, ctypes.byref(out)), "atts_debug_score_form")
    return out.value


def profile_begin(max_records: int = 1024) -> None:
    """Start recording CUDA-event pairs around the fused scoring kernel of every score_logprob call."""
    _check(load().atts_profile_begin(int(max_records)), "atts_profile_begin")


def profile_end(cap: int = 4096) -> list[float]:
    """Stop recording; returns the fused kernel's durations in milliseconds, one per recorded call."""
    buf = (ctypes.c_float * cap)()
    cnt = c_int(0)
    _check(load().atts_profile_end(buf, cap, ctypes.byref(cnt)), "atts_profile_end")
    return [float(buf[i]) for i in range(min(cnt.value, cap))]


def debug_score_plan(M: int, d: int, V: int, workers: int, ctas: int) -> dict:
    """The fused kernel's static schedule for a shape (no device needed)."""
    out = (c_int32 * 8)()
    _check(load().atts_debug_score_plan(M, d, V, workers, ctas, out), "atts_debug_score_plan")
    return dict(zip(("RB", "NT", "KB", "C", "Gr", "units", "M_pad", "ctas"), list(out)))


def debug_score_unit(M: int, d: int, V: int, workers: int, ctas: int, u: int) -> tuple:
    """(row block, chunk, first tile, one past the last tile) of unit u of that schedule."""
    out = (c_int32 * 4)()
    _check(load().atts_debug_score_unit(M, d, V, workers, ctas, u, out), "atts_debug_score_unit")
    return tuple(out)


# ---------------------------------------------------------------------------------------------------------------------
# Attention of drafted tokens over a paged cache
# ---------------------------------------------------------------------------------------------------------------------
class _KvCache(ctypes.Structure):
    _fields_ = [("k", c_void_p), ("v", c_void_p), ("block_table", c_void_p), ("num_seqs", c_int64), ("table_cols", c_int64),
                ("table_stride", c_int64), ("num_pages", c_int64), ("page_size", c_int64), ("page_stride", c_int64),
                ("slot_stride", c_int64), ("head_stride", c_int64), ("heads", c_int32), ("head_dim", c_int32),
                ("dtype", c_int32), ("reserved", c_int32)]


class PagedCache:
    """Description of a paged key/value cache, made once and passed to every call (it holds pointers, not contents).

    k, v: [num_pages, page_size, heads, head_dim] bf16 or fp16 (any strides that are multiples of 8 elements, the same for
    both; head_dim contiguous; a head-major cache is passed as a transposed view); block_table: int32 [num_seqs, pages]."""

    def __init__(self, k, v, block_table):
        import torch
        if k.dtype not in (torch.bfloat16, torch.float16) or v.dtype != k.dtype:
            raise ValueError("k and v have to be bfloat16 or float16, both the same")
        if k.dim() != 4 or k.shape != v.shape or k.stride() != v.stride() or (k.numel() and k.stride(3) != 1):
            raise ValueError("k and v: [num_pages, page_size, heads, head_dim] with equal strides, head_dim contiguous")
        if block_table.dtype != torch.int32 or block_table.dim() != 2 or (block_table.shape[1] > 1 and block_table.stride(1) != 1):
            raise ValueError("block_table: int32 [num_seqs, pages], rows contiguous")
        if not (k.is_cuda and v.device == k.device and block_table.device == k.device):
            raise ValueError("k, v and block_table have to be on one CUDA device")
        self.k, self.v, self.block_table = k, v, block_table
        self.num_pages, self.page_size, self.heads, self.head_dim = k.shape
        self.num_seqs, self.dtype, self.device = block_table.shape[0], k.dtype, k.device
        # a dimension of one entry has a stride that means nothing
        ps, ss, hs = (k.stride(i) if k.shape[i] > 1 else 0 for i in range(3))
        self._c = _KvCache(_ptr(k), _ptr(v), _ptr(block_table), self.num_seqs, block_table.shape[1],
                           block_table.stride(0) if self.num_seqs > 1 else block_table.shape[1], self.num_pages,
                           self.page_size, ps, ss, hs, self.heads, self.head_dim, 0 if k.dtype == torch.bfloat16 else 1, 0)
        self._ref = ctypes.addressof(self._c)


def _rows(t, name: str, M: int, heads: int, cache: PagedCache):
    """(pointer, token stride, head stride) of a [M, heads, head_dim] tensor of the cache's type."""
    if t.shape != (M, heads, cache.head_dim) or t.dtype is not cache.dtype or t.device != cache.device:
        raise ValueError(f"{name}: has to be [{M}, {heads}, {cache.head_dim}], {cache.dtype}, on {cache.device} like the cache; got "
                         f"{list(t.shape)}, {t.dtype}, on {t.device}")
    token, head, channel = t.stride()
    if channel != 1 and t.numel():
        raise ValueError(f"{name}: head_dim has to be contiguous")
    return t.data_ptr(), token if M > 1 else 0, head if heads > 1 else 0


def _stream_on(device) -> int:
    """The current stream, provided that `device`, where the call's tensors are, is the current one: kernels run there."""
    stream = _stream()
    if device.index != _current_device():      # (None for the host)
        raise ValueError(f"the tensors are on {device}, the current device is cuda:{_current_device()}")
    return stream


def _vec(t, name: str, dtype, n: int, device):
    """Pointer of a contiguous tensor of n entries."""
    if t.dtype is not dtype or t.numel() != n or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name}: has to be a contiguous {dtype} tensor of {n} entries on {device}")
    return t.data_ptr()


def tree_plan(parent, cu_tokens):
    """Preorder numbers of draft trees (host): parent [M] int32 per token (index within its sequence, -1: continues the
    cache, -2: padding), cu_tokens [num_seqs + 1] int32, both CPU tensors or arrays -> (pre, end, depth) int32 CPU tensors:
    token j is an ancestor of i, or i itself, iff pre[j] <= pre[i] < end[j]."""
    import torch
    parent = torch.as_tensor(parent, dtype=torch.int32).contiguous()
    cu = torch.as_tensor(cu_tokens, dtype=torch.int32).contiguous()
    if parent.device.type != "cpu" or cu.device.type != "cpu":
        raise ValueError("parent and cu_tokens have to be on the host")
    if cu.numel() < 1 or int(cu[-1]) != parent.numel():
        raise ValueError("cu_tokens has to end at the number of tokens")
    pre, end, depth = (torch.empty_like(parent) for _ in range(3))
    _check(load().atts_tree_plan(_ptr(parent), _ptr(cu), cu.numel() - 1, _ptr(pre), _ptr(end), _ptr(depth)), "atts_tree_plan")
    return pre, end, depth


def rope_freqs(rotary_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, original_length: int = 8192,
               low: float = 1.0, high: float = 4.0, fast: float = 32.0, slow: float = 1.0):
    """Rotations of rotary positions: (float64 CPU tensor [rotary_dim / 2] of radians per position, factor on cos and sin).

    f_i = base ** (-2 i / rotary_dim), then for long contexts
      "linear"  f / factor (positions stretched)
      "bands"   pairs that turn more than `high` times over original_length keep f, those below `low` turns get f / factor,
                a straight line in the number of turns in between
      "ramp"    the same between the pairs that turn `fast` and `slow` times, a straight line in the pair's number, and
                cosine and sine grow by 0.1 ln(factor) + 1"""
    import math
    import torch
    if rotary_dim < 0 or rotary_dim % 2 or not base > 0 or not factor > 0 or original_length < 1:
        raise ValueError("rotary_dim has to be even and >= 0, base, factor and original_length positive")
    i = torch.arange(0, rotary_dim, 2, dtype=torch.float64)
    f = base ** (-i / max(rotary_dim, 1))
    if scaling == "none":
        return f, 1.0
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "bands":
        if not high > low:
            raise ValueError("bands: high has to be above low")
        keep = ((original_length * f / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        return f * keep + f / factor * (1 - keep), 1.0
    if scaling == "ramp":
        def pair(turns):   # where original_length positions make that many turns, in channels
            return rotary_dim * math.log(original_length / (turns * 2 * math.pi)) / (2 * math.log(base))
        first, last = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), max(rotary_dim - 1, 0))
        ramp = ((torch.arange(rotary_dim // 2, dtype=torch.float64) - first) / max(last - first, 1e-3)).clamp(0.0, 1.0)
        return f * (1 - ramp) + f / factor * ramp, (0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0)
    raise ValueError(f"scaling: one of none, linear, bands, ramp, not {scaling!r}")


def rope_append(q, k, v, positions, freqs, cache: PagedCache, ctx_lens, cu_tokens, max_tokens: int, q_out, interleaved: bool = False,
                mscale: float = 1.0) -> None:
    """Rotate q [M, Hq, D] into q_out (may be q) and k [M, heads, D] into the cache's slots ctx_lens[b] + t, copy v beside
    it. positions int32 [M], freqs float64 [pairs] on the device (:func:`rope_freqs`). q and q_out None: append only."""
    import torch
    M, dev, B = k.shape[0], cache.device, cache.num_seqs
    kr, vr = _rows(k, "k", M, cache.heads, cache), _rows(v, "v", M, cache.heads, cache)
    Hq = 0 if q is None else q.shape[1]
    qr, outr = ((0, 0, 0), (0, 0, 0)) if q is None else (_rows(q, "q", M, Hq, cache), _rows(q_out, "q_out", M, Hq, cache))
    n = freqs.numel()
    _check(load().atts_rope_append(*qr, *kr, *vr, _vec(positions, "positions", torch.int32, M, dev),
                                   _vec(freqs, "freqs", torch.float64, n, dev), n, mscale, 1 if interleaved else 0, cache._ref,
                                   _vec(ctx_lens, "ctx_lens", torch.int32, B, dev),
                                   _vec(cu_tokens, "cu_tokens", torch.int32, B + 1, dev), M, Hq, max_tokens, *outr, _stream_on(dev)),
           "atts_rope_append")


def tree_attention_workspace_bytes(num_seqs: int, M: int, Hq: int, heads: int, head_dim: int, max_tokens: int, max_len: int) -> int:
    """Bytes that tree_attention needs for these sizes. Ask for every batch: a smaller one may need more (more chunks)."""
    out = c_size_t(0)
    _check(load().atts_tree_attention_workspace_bytes(num_seqs, M, Hq, heads, head_dim, max_tokens, max_len, ctypes.byref(out)),
           "atts_tree_attention_workspace_bytes")
    return out.value


def tree_attention(q, cache: PagedCache, ctx_lens, cu_tokens, pre, end, max_tokens: int, max_len: int, scale: float, out, lse,
                   workspace) -> None:
    """Attention of q [M, Hq, D] over each sequence's cached slots and its own drafted ancestors -> out [M, Hq, D],
    lse [M, Hq] f32 (or None). pre, end int32 [M] (:func:`tree_plan`), both None: chains."""
    import torch
    M, Hq = q.shape[0], q.shape[1]
    dev, B, i32 = cache.device, cache.num_seqs, torch.int32
    if workspace.device != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace: has to be contiguous, on {dev}")
    _check(load().atts_tree_attention(*_rows(q, "q", M, Hq, cache), cache._ref, _vec(ctx_lens, "ctx_lens", i32, B, dev),
                                      _vec(cu_tokens, "cu_tokens", i32, B + 1, dev), None if pre is None else _vec(pre, "pre", i32, M, dev),
                                      None if end is None else _vec(end, "end", i32, M, dev), M, Hq, max_tokens, max_len, scale,
                                      *_rows(out, "out", M, Hq, cache), None if lse is None else _vec(lse, "lse", torch.float32, M * Hq, dev),
                                      _ptr(workspace), _nbytes(workspace), _stream_on(dev)), "atts_tree_attention")


def cache_weights(q, cache: PagedCache, lse, ctx_lens, cu_tokens, pre, end, max_tokens: int, max_len: int, scale: float, weights_in,
                  weights_out) -> None:
    """weights_out[b, h, s] = weights_in[b, h, s] (None: 0) + the attention that slot s of key head h receives in this batch
    (lse as tree_attention wrote it); [num_seqs, heads, cols] f32 contiguous, weights_in may be weights_out."""
    import torch
    M, Hq = q.shape[0], q.shape[1]
    dev, B, i32 = cache.device, cache.num_seqs, torch.int32
    cols = weights_out.shape[-1]
    n = B * cache.heads * cols
    _check(load().atts_cache_weights(*_rows(q, "q", M, Hq, cache), cache._ref, _vec(lse, "lse", torch.float32, M * Hq, dev),
                                     _vec(ctx_lens, "ctx_lens", i32, B, dev), _vec(cu_tokens, "cu_tokens", i32, B + 1, dev),
                                     None if pre is None else _vec(pre, "pre", i32, M, dev), None if end is None else _vec(end, "end", i32, M, dev),
                                     M, Hq, max_tokens, max_len, scale,
                                     None if weights_in is None else _vec(weights_in, "weights_in", torch.float32, n, dev),
                                     _vec(weights_out, "weights_out", torch.float32, n, dev), cols, _stream_on(dev)), "atts_cache_weights")


def cache_select(weights, lens, budget: int, sinks: int, recent: int, kept, counts) -> None:
    """kept [num_seqs, heads, budget] i32: the slots to keep, ascending (the first `sinks`, the last `recent`, then the
    largest of weights [num_seqs, heads, cols] f32; ties: the lowest), -1 behind; counts [num_seqs] i32 = min(lens, budget)."""
    import torch
    B, heads, cols = weights.shape
    dev = weights.device
    _check(load().atts_cache_select(_vec(weights, "weights", torch.float32, B * heads * cols, dev), cols,
                                    _vec(lens, "lens", torch.int32, B, dev), B, heads, budget, sinks, recent,
                                    _vec(kept, "kept", torch.int32, B * heads * budget, dev),
                                    _vec(counts, "counts", torch.int32, B, dev), _stream_on(dev)), "atts_cache_select")


def cache_gather(src: PagedCache, kept, counts, dst: PagedCache, weights_in=None, weights_out=None) -> None:
    """Slot c of every sequence and head in dst gets key and value of slot kept[b, h, c] of src (c < counts[b]; dst's pages
    must not be src's), weights_out [num_seqs, heads, cols] the kept slots' weights."""
    import torch
    dev = src.device
    if dst.device != dev:
        raise ValueError(f"dst: has to be on {dev} like src, not on {dst.device}")
    cols = kept.shape[-1]
    n = src.num_seqs * src.heads * cols
    in_cols = 0 if weights_in is None else weights_in.shape[-1]
    _check(load().atts_cache_gather(src._ref, _vec(kept, "kept", torch.int32, n, dev), cols,
                                    _vec(counts, "counts", torch.int32, src.num_seqs, dev), dst._ref,
                                    None if weights_in is None else _vec(weights_in, "weights_in", torch.float32, src.num_seqs * src.heads * in_cols, dev),
                                    in_cols, None if weights_out is None else _vec(weights_out, "weights_out", torch.float32, n, dev),
                                    _stream_on(dev)), "atts_cache_gather")
