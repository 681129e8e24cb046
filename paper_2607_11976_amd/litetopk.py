"""Python binding of the C ABI in include/litetopk.h (argument marshalling only).

Every computation runs in the HIP library liblitetopk.so built next to this
file (``python -m paper_2607_11976_amd.build``). torch is used for device
memory and streams: tensors hand over their device pointers and the current
HIP stream. There is no CPU fallback: if the library is missing or no GPU is
visible, the calls raise.

Two layers:
  * the raw entry points with the C names (``lt_indexer_topk`` ...), taking
    integers for pointers, exactly as declared in the header;
  * convenience wrappers (``indexer_topk``, ``topk_select``, ...) that check
    tensor shapes, allocate outputs and workspace with torch and call them.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import NamedTuple, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# LT_LIBRARY names another build of the same library (the host-sanitizer
# build that tests/test_abi_sanitized.py makes); default: the in-tree build
LIB_PATH = os.environ.get("LT_LIBRARY") or os.path.join(_HERE, "liblitetopk.so")

LT_OK, LT_EINVAL, LT_EUNSUPPORTED, LT_EWORKSPACE, LT_EHIP, LT_ESCRATCH = 0, -1, -2, -3, -4, -5
LT_F32, LT_BF16, LT_FP8_E4M3FN = 0, 1, 2
LT_SCORE_DSA, LT_SCORE_IP = 0, 1
LT_SORTED_OUTPUT, LT_FORCE_FALLBACK = 1, 2
LT_K_MAX = 8192
LT_SAMPLE_LIST_MAX = 32768
LT_UNION_MAX = 32768
LT_ROW_STATS = 12
LT_STATIC_SCRATCH_BYTES = 256 << 20
LT_NUM_STAGE_EVENTS = 6
LT_MAX_PAGE_SIZE = 4096
LT_PLAN_MAX_REQUESTS = 16384
LT_CACHE4_MAX_HEADS = 1024
LT_LOGPROB_MAX_TOP = 64
LT_LOGPROB_MAX_VOCAB = 1 << 30
LT_LOGPROB_MAX_ROWS = 0xFFFFFF
LT_ROTARY_INTERLEAVED, LT_ROTARY_INVERSE = 1, 2
LT_ROTARY_MAX_DIM = 1024
LT_ROTARY_MAX_HEADS = 1 << 20
LT_BEAM_MAX_TOP = 64
LT_BEAM_MAX_BEAMS = 1024
LT_REORDER_MAX_GROUP = 64
STAGES = ("sample", "range", "filter", "select", "fallback")

EXPORTED = (
    "lt_options_default", "lt_indexer_topk_workspace_size", "lt_indexer_topk", "lt_indexer_topk_static",
    "lt_indexer_scores",
    "lt_topk_select_workspace_size", "lt_topk_select", "lt_topk_radix",
    "lt_sample_from_topk_workspace_size", "lt_sample_from_topk", "lt_dsa_union",
    "lt_paged_plan", "lt_cache4_append", "lt_cache4_read", "lt_cache4_attention_workspace_size",
    "lt_cache4_attention", "lt_token_logprobs_workspace_size", "lt_token_logprobs", "lt_token_logprobs_backward",
    "lt_rotary", "lt_rotary_fp8", "lt_cache4_append_rotary", "lt_beam_select_workspace_size", "lt_beam_select",
    "lt_paged_reorder_workspace_size", "lt_paged_reorder", "lt_cache4_copy",
    "lt_event_create",
    "lt_event_destroy", "lt_event_record", "lt_event_elapsed_ms", "lt_strerror",
)


class LtOptions(ctypes.Structure):
    _fields_ = [
        ("num_bins", ctypes.c_int32),
        ("sample_size", ctypes.c_int32),
        ("capacity", ctypes.c_int32),
        ("key_splits", ctypes.c_int32),
        ("flags", ctypes.c_uint32),
        ("seed", ctypes.c_uint64),
        ("stage_events", ctypes.c_void_p),
        ("row_stats", ctypes.c_void_p),
        ("sample_keys", ctypes.c_void_p),
        ("visible_start", ctypes.c_void_p),
    ]


class LiteTopKError(RuntimeError):
    pass


_lib = None
_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_I64 = ctypes.c_int64
_SZ = ctypes.c_size_t
_F32 = ctypes.c_float
_F64 = ctypes.c_double
_U32 = ctypes.c_uint32


def load(path: str = LIB_PATH):
    """Load the shared library (once) and declare the C signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise LiteTopKError("HIP library not built: %s (run python -m paper_2607_11976_amd.build)" % path)
    lib = ctypes.CDLL(path)
    lib.lt_options_default.argtypes = [ctypes.POINTER(LtOptions)]
    lib.lt_options_default.restype = None
    lib.lt_indexer_topk_workspace_size.argtypes = [_I32, _I32, _I32, _I32, ctypes.c_int, ctypes.c_int, _I32,
                                                   ctypes.POINTER(LtOptions)]
    lib.lt_indexer_topk_workspace_size.restype = _SZ
    lib.lt_indexer_topk.argtypes = [_P, _P, _P, _P, _P, ctypes.c_int, ctypes.c_int, _I32, _I32, _I32, _I32, _I32,
                                    _P, _P, _P, _P, _SZ, ctypes.POINTER(LtOptions), _P]
    lib.lt_indexer_topk.restype = ctypes.c_int
    lib.lt_indexer_topk_static.argtypes = [_P, _P, _P, _P, _P, ctypes.c_int, ctypes.c_int, _I32, _I32, _I32, _I32,
                                           _I32, _P, _P, _P, ctypes.POINTER(LtOptions), _P]
    lib.lt_indexer_topk_static.restype = ctypes.c_int
    lib.lt_indexer_scores.argtypes = [_P, _P, _P, _P, _P, ctypes.c_int, ctypes.c_int, _I32, _I32, _I32, _I32,
                                      _P, _I64, _P]
    lib.lt_indexer_scores.restype = ctypes.c_int
    lib.lt_topk_select_workspace_size.argtypes = [_I32, _I32, _I32, ctypes.POINTER(LtOptions)]
    lib.lt_topk_select_workspace_size.restype = _SZ
    lib.lt_topk_select.argtypes = [_P, _I64, _I32, _I32, _I32, _P, _P, _P, _P, _SZ, ctypes.POINTER(LtOptions), _P]
    lib.lt_topk_select.restype = ctypes.c_int
    lib.lt_topk_radix.argtypes = [_P, _I64, _I32, _I32, _I32, _P, _P, _P, ctypes.c_uint32, _P]
    lib.lt_topk_radix.restype = ctypes.c_int
    lib.lt_sample_from_topk_workspace_size.argtypes = [_I32]
    lib.lt_sample_from_topk_workspace_size.restype = _SZ
    lib.lt_sample_from_topk.argtypes = [_P, _I64, _I32, _I32, _I32, _I32, _P, _P, _SZ, _P]
    lib.lt_sample_from_topk.restype = ctypes.c_int
    lib.lt_dsa_union.argtypes = [_P, _I64, _I32, _I32, _I32, _P, _P, _P, _P]
    lib.lt_dsa_union.restype = ctypes.c_int
    lib.lt_paged_plan.argtypes = [_P, _P, _I32, _I32, _P, _I64, _I32, _P, _I32, _P, _I32, _P, _P, _P, _P, _P, _P, _P]
    lib.lt_paged_plan.restype = ctypes.c_int
    lib.lt_cache4_append.argtypes = [_P, _P, ctypes.c_int, _I64, _I64, _I64, _P, _P, _I64, _I32, _I32, _I32, _P, _P]
    lib.lt_cache4_append.restype = ctypes.c_int
    lib.lt_cache4_read.argtypes = [_P, _P, _I64, _I32, _I32, _I32, _P, _I64, _P, _P, _P]
    lib.lt_cache4_read.restype = ctypes.c_int
    lib.lt_cache4_attention_workspace_size.argtypes = [_I32, _I32, _I32, _I32, _I32, _I32]
    lib.lt_cache4_attention_workspace_size.restype = _SZ
    lib.lt_cache4_attention.argtypes = [_P, _I64, _I32, _I32, _I32, _P, _P, _I64, _I32, _I32, _P, _I64, _I32, _P, _P,
                                        _I32, _P, _P, _P, _I64, _I32, _P, _F32, _P, _P, _P, _SZ, _P]
    lib.lt_cache4_attention.restype = ctypes.c_int
    lib.lt_token_logprobs_workspace_size.argtypes = [ctypes.c_int, _I32, _I32, _I32]
    lib.lt_token_logprobs_workspace_size.restype = _SZ
    lib.lt_token_logprobs.argtypes = [_P, ctypes.c_int, _I64, _I32, _I32, _P, _F32, _I32, _P, _P, _P, _P, _P, _P, _SZ,
                                      _P]
    lib.lt_token_logprobs.restype = ctypes.c_int
    lib.lt_token_logprobs_backward.argtypes = [_P, ctypes.c_int, _I64, _I32, _I32, _P, _F32, _P, _P, _P, _P, _P, _I64,
                                               _P]
    lib.lt_token_logprobs_backward.restype = ctypes.c_int
    lib.lt_rotary.argtypes = [_P, ctypes.c_int, _I64, _I64, _I32, _I32, _I32, _P, _P, _I32, _I32, _F64, _U32, _P,
                              ctypes.c_int, _I64, _I64, _P]
    lib.lt_rotary.restype = ctypes.c_int
    lib.lt_rotary_fp8.argtypes = [_P, ctypes.c_int, _I64, _I64, _I32, _I32, _I32, _P, _P, _I32, _I32, _F64, _U32, _P,
                                  _P, _P]
    lib.lt_rotary_fp8.restype = ctypes.c_int
    lib.lt_cache4_append_rotary.argtypes = [_P, _P, ctypes.c_int, _I64, _I64, _I64, _P, _P, _I64, _I32, _I32, _I32, _P,
                                            _P, _P, _I32, _I32, _F64, _U32, _P, _I64, _I32, _P, _P]
    lib.lt_cache4_append_rotary.restype = ctypes.c_int
    lib.lt_beam_select_workspace_size.argtypes = [ctypes.c_int, _I32, _I32, _I32, _I32]
    lib.lt_beam_select_workspace_size.restype = _SZ
    lib.lt_beam_select.argtypes = [_P, ctypes.c_int, _I64, _I32, _I32, _I32, _P, _F64, _I32, _P, _P, _P, _P, _SZ, _P]
    lib.lt_beam_select.restype = ctypes.c_int
    lib.lt_paged_reorder_workspace_size.argtypes = [_I32]
    lib.lt_paged_reorder_workspace_size.restype = _SZ
    lib.lt_paged_reorder.argtypes = [_P, _I64, _I32, _P, _P, _I32, _I32, _I32, _P, _P, _I32, _P, _P, _I64, _P, _P, _P,
                                     _P, _P, _SZ, _P]
    lib.lt_paged_reorder.restype = ctypes.c_int
    lib.lt_cache4_copy.argtypes = [_P, _P, _I64, _I32, _I32, _I32, _P, _I32, _P]
    lib.lt_cache4_copy.restype = ctypes.c_int
    lib.lt_event_create.argtypes = [ctypes.POINTER(ctypes.c_void_p)]
    lib.lt_event_create.restype = ctypes.c_int
    lib.lt_event_destroy.argtypes = [_P]
    lib.lt_event_destroy.restype = ctypes.c_int
    lib.lt_event_record.argtypes = [_P, _P]
    lib.lt_event_record.restype = ctypes.c_int
    lib.lt_event_elapsed_ms.argtypes = [_P, _P, ctypes.POINTER(ctypes.c_float)]
    lib.lt_event_elapsed_ms.restype = ctypes.c_int
    lib.lt_strerror.argtypes = [ctypes.c_int]
    lib.lt_strerror.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(status: int, what: str):
    if status != LT_OK:
        msg = load().lt_strerror(status).decode()
        raise LiteTopKError("%s failed: %s (%d)" % (what, msg, status))


# ---------------------------------------------------------------------------
# raw entry points (same names and argument order as the header)
# ---------------------------------------------------------------------------

def lt_options_default() -> LtOptions:
    o = LtOptions()
    load().lt_options_default(ctypes.byref(o))
    return o


def lt_indexer_topk_workspace_size(nq, nk, h, d, dtype, mode, k, opts: Optional[LtOptions] = None) -> int:
    return load().lt_indexer_topk_workspace_size(nq, nk, h, d, dtype, mode, k,
                                                 ctypes.byref(opts) if opts is not None else None)


def lt_indexer_topk(q, q_scale, w, keys, k_scale, dtype, mode, nq, nk, h, d, k, causal_offsets, out_idx,
                    out_scores, workspace, workspace_bytes, opts, stream) -> int:
    return load().lt_indexer_topk(q, q_scale, w, keys, k_scale, dtype, mode, nq, nk, h, d, k, causal_offsets,
                                  out_idx, out_scores, workspace, workspace_bytes,
                                  ctypes.byref(opts) if opts is not None else None, stream)


def lt_indexer_topk_static(q, q_scale, w, keys, k_scale, dtype, mode, nq, nk, h, d, k, causal_offsets, out_idx,
                           out_scores, opts, stream) -> int:
    return load().lt_indexer_topk_static(q, q_scale, w, keys, k_scale, dtype, mode, nq, nk, h, d, k,
                                         causal_offsets, out_idx, out_scores,
                                         ctypes.byref(opts) if opts is not None else None, stream)


def lt_indexer_scores(q, q_scale, w, keys, k_scale, dtype, mode, nq, nk, h, d, scores, ld, stream) -> int:
    return load().lt_indexer_scores(q, q_scale, w, keys, k_scale, dtype, mode, nq, nk, h, d, scores, ld, stream)


def lt_topk_select_workspace_size(nq, nk, k, opts: Optional[LtOptions] = None) -> int:
    return load().lt_topk_select_workspace_size(nq, nk, k, ctypes.byref(opts) if opts is not None else None)


def lt_topk_select(scores, row_stride, nq, nk, k, causal_offsets, out_idx, out_scores, workspace,
                   workspace_bytes, opts, stream) -> int:
    return load().lt_topk_select(scores, row_stride, nq, nk, k, causal_offsets, out_idx, out_scores, workspace,
                                 workspace_bytes, ctypes.byref(opts) if opts is not None else None, stream)


def lt_topk_radix(scores, row_stride, nq, nk, k, causal_offsets, out_idx, out_scores, flags, stream) -> int:
    return load().lt_topk_radix(scores, row_stride, nq, nk, k, causal_offsets, out_idx, out_scores, flags, stream)


def lt_sample_from_topk_workspace_size(nk) -> int:
    return load().lt_sample_from_topk_workspace_size(nk)


def lt_sample_from_topk(prev_idx, ld, prev_rows, prev_k, nk, sample_size, sample_keys, workspace, workspace_bytes,
                        stream) -> int:
    return load().lt_sample_from_topk(prev_idx, ld, prev_rows, prev_k, nk, sample_size, sample_keys, workspace,
                                      workspace_bytes, stream)


def lt_dsa_union(topk_idx, ld, nq, k, group, union_idx, union_count, member_mask, stream) -> int:
    return load().lt_dsa_union(topk_idx, ld, nq, k, group, union_idx, union_count, member_mask, stream)


def lt_paged_plan(*args) -> int:
    return load().lt_paged_plan(*args)


def lt_cache4_append(*args) -> int:
    return load().lt_cache4_append(*args)


def lt_cache4_read(*args) -> int:
    return load().lt_cache4_read(*args)


def lt_cache4_attention_workspace_size(tokens, requests, heads, kv_heads, head_dim, selected_k=0) -> int:
    return load().lt_cache4_attention_workspace_size(tokens, requests, heads, kv_heads, head_dim, selected_k)


def lt_cache4_attention(*args) -> int:
    return load().lt_cache4_attention(*args)


def lt_token_logprobs_workspace_size(dtype, rows, vocab, top) -> int:
    return load().lt_token_logprobs_workspace_size(dtype, rows, vocab, top)


def lt_token_logprobs(*args) -> int:
    return load().lt_token_logprobs(*args)


def lt_token_logprobs_backward(*args) -> int:
    return load().lt_token_logprobs_backward(*args)


def lt_rotary(*args) -> int:
    return load().lt_rotary(*args)


def lt_rotary_fp8(*args) -> int:
    return load().lt_rotary_fp8(*args)


def lt_cache4_append_rotary(*args) -> int:
    return load().lt_cache4_append_rotary(*args)


def lt_beam_select_workspace_size(dtype, batch, beams, vocab, top) -> int:
    return load().lt_beam_select_workspace_size(dtype, batch, beams, vocab, top)


def lt_beam_select(*args) -> int:
    return load().lt_beam_select(*args)


def lt_paged_reorder_workspace_size(rows) -> int:
    return load().lt_paged_reorder_workspace_size(rows)


def lt_paged_reorder(*args) -> int:
    return load().lt_paged_reorder(*args)


def lt_cache4_copy(*args) -> int:
    return load().lt_cache4_copy(*args)


def lt_strerror(status: int) -> str:
    return load().lt_strerror(status).decode()


# ---------------------------------------------------------------------------
# tensor helpers
# ---------------------------------------------------------------------------

def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return LT_F32
    if t.dtype == torch.bfloat16:
        return LT_BF16
    if t.dtype in (torch.uint8, torch.float8_e4m3fn):
        return LT_FP8_E4M3FN
    raise LiteTopKError("unsupported storage dtype %s" % t.dtype)


def _need(cond: bool, msg: str):
    if not cond:
        raise LiteTopKError(msg)


def _on_gpu(*ts):
    for t in ts:
        if t is not None:
            _need(t.is_cuda, "tensors must be on the GPU")
            _need(t.is_contiguous(), "tensors must be contiguous")


def make_options(num_bins=None, sample_size=None, capacity=None, key_splits=None,
                 sorted_output=False, force_fallback=False, seed=None, stage_events=None,
                 row_stats: Optional[torch.Tensor] = None,
                 sample_keys: Optional[torch.Tensor] = None,
                 visible_start: Optional[torch.Tensor] = None) -> LtOptions:
    """lt_options from keyword arguments. sample_keys: a GPU int32 list used
    as the sample (its length becomes sample_size); the tensor must stay
    alive until the call that uses these options has run."""
    o = lt_options_default()
    if num_bins is not None:
        o.num_bins = num_bins
    if sample_size is not None:
        o.sample_size = sample_size
    if capacity is not None:
        o.capacity = capacity
    if key_splits is not None:
        o.key_splits = key_splits
    o.flags = (LT_SORTED_OUTPUT if sorted_output else 0) | (LT_FORCE_FALLBACK if force_fallback else 0)
    if seed is not None:
        o.seed = seed
    if stage_events is not None:
        o.stage_events = ctypes.cast(stage_events.array, ctypes.c_void_p)
    if row_stats is not None:
        _on_gpu(row_stats)
        _need(row_stats.dtype == torch.int32 and row_stats.dim() == 2 and row_stats.shape[1] == LT_ROW_STATS,
              "row_stats must be an int32 [Nq, LT_ROW_STATS] GPU tensor")
        o.row_stats = row_stats.data_ptr()
        o.row_stats_rows = row_stats.shape[0]
    if sample_keys is not None:
        _on_gpu(sample_keys)
        _need(sample_keys.dtype == torch.int32 and sample_keys.dim() == 1, "sample_keys must be int32 [n]")
        o.sample_keys = sample_keys.data_ptr()
        o.sample_size = sample_keys.numel()
    if visible_start is not None:
        _on_gpu(visible_start)
        _need(visible_start.dtype == torch.int32 and visible_start.dim() == 1, "visible_start must be int32 [Nq]")
        o.visible_start = visible_start.data_ptr()
    return o


class StageEvents:
    """LT_NUM_STAGE_EVENTS HIP events for lt_options.stage_events."""

    def __init__(self):
        lib = load()
        self.array = (ctypes.c_void_p * LT_NUM_STAGE_EVENTS)()
        for i in range(LT_NUM_STAGE_EVENTS):
            h = ctypes.c_void_p()
            _check(lib.lt_event_create(ctypes.byref(h)), "lt_event_create")
            self.array[i] = h.value

    def stage_ms(self):
        """Device milliseconds of each stage of the last call (synchronises)."""
        lib = load()
        out = {}
        for i, name in enumerate(STAGES):
            ms = ctypes.c_float()
            _check(lib.lt_event_elapsed_ms(self.array[i], self.array[i + 1], ctypes.byref(ms)), "elapsed")
            out[name] = ms.value
        return out

    def close(self):
        lib = load()
        for i in range(LT_NUM_STAGE_EVENTS):
            if self.array[i]:
                lib.lt_event_destroy(self.array[i])
                self.array[i] = None


def _check_rows(nq: int, causal_offsets: Optional[torch.Tensor], options: Optional[LtOptions]):
    """Per-row arguments: causal_offsets int32 [Nq] on the GPU; the options'
    row_stats (checked in make_options for its shape) must cover Nq rows."""
    if causal_offsets is not None:
        _on_gpu(causal_offsets)
        _need(causal_offsets.dtype == torch.int32 and causal_offsets.numel() == nq,
              "causal_offsets must be int32 [Nq]")
    if options is not None and options.row_stats:
        n = getattr(options, "row_stats_rows", None)
        _need(n is not None and n >= nq, "row_stats must hold LT_ROW_STATS fields for each of the Nq rows "
              "(pass it through make_options)")


def _check_score_inputs(q, w, keys, causal_offsets, q_scale, k_scale, options):
    nq, h, _ = q.shape
    nk = keys.shape[0]
    if w is not None:
        _need(w.dtype == torch.float32 and tuple(w.shape) == (nq, h), "w must be float32 [Nq, H]")
    if _dtype_code(q) == LT_FP8_E4M3FN:
        _need(q_scale is not None and q_scale.dtype == torch.float32 and tuple(q_scale.shape) == (nq, h),
              "fp8: q_scale must be float32 [Nq, H]")
        _need(k_scale is not None and k_scale.dtype == torch.float32 and tuple(k_scale.shape) == (nk,),
              "fp8: k_scale must be float32 [Nk]")
    _check_rows(nq, causal_offsets, options)


def _mode_code(mode: str) -> int:
    if mode == "dsa":
        return LT_SCORE_DSA
    if mode == "ip":
        return LT_SCORE_IP
    raise LiteTopKError("mode must be 'dsa' or 'ip'")


def indexer_topk_workspace(nq, nk, h, d, dtype: int, mode: str, k: int, options: Optional[LtOptions] = None,
                           device=None) -> torch.Tensor:
    n = lt_indexer_topk_workspace_size(nq, nk, h, d, dtype, _mode_code(mode), k, options)
    _need(n > 0, "unsupported shape for lt_indexer_topk")
    return torch.empty(n, dtype=torch.uint8, device=device or "cuda")


def indexer_topk(q: torch.Tensor, w: Optional[torch.Tensor], keys: torch.Tensor, k: int,
                 causal_offsets: Optional[torch.Tensor] = None, q_scale: Optional[torch.Tensor] = None,
                 k_scale: Optional[torch.Tensor] = None, mode: str = "dsa",
                 options: Optional[LtOptions] = None, out=None, workspace: Optional[torch.Tensor] = None,
                 stream=None):
    """Exact per-row top-k of the index score. q [Nq, H, d], keys [Nk, d] in
    float32 / bfloat16 / uint8 (E4M3FN bytes, with q_scale [Nq, H] and k_scale
    [Nk]); w [Nq, H] float32 or None. Returns (idx int32 [Nq, k], scores
    float32 [Nq, k])."""
    _on_gpu(q, w, keys, causal_offsets, q_scale, k_scale)
    _need(q.dim() == 3 and keys.dim() == 2 and q.shape[2] == keys.shape[1], "q [Nq,H,d] and keys [Nk,d] required")
    dt = _dtype_code(q)
    _need(_dtype_code(keys) == dt, "q and keys must share a dtype")
    nq, h, d = q.shape
    nk = keys.shape[0]
    _check_score_inputs(q, w, keys, causal_offsets, q_scale, k_scale, options)
    if out is None:
        out = (torch.empty((nq, k), dtype=torch.int32, device=q.device),
               torch.empty((nq, k), dtype=torch.float32, device=q.device))
    if workspace is None:
        workspace = indexer_topk_workspace(nq, nk, h, d, dt, mode, k, options, q.device)
    st = lt_indexer_topk(_ptr(q), _ptr(q_scale), _ptr(w), _ptr(keys), _ptr(k_scale), dt, _mode_code(mode), nq, nk,
                         h, d, k, _ptr(causal_offsets), _ptr(out[0]), _ptr(out[1]), _ptr(workspace),
                         workspace.numel(), options, _stream(stream))
    _check(st, "lt_indexer_topk")
    return out


def indexer_topk_static(q: torch.Tensor, w: Optional[torch.Tensor], keys: torch.Tensor, k: int,
                        causal_offsets: Optional[torch.Tensor] = None, q_scale: Optional[torch.Tensor] = None,
                        k_scale: Optional[torch.Tensor] = None, mode: str = "dsa",
                        options: Optional[LtOptions] = None, out=None, stream=None):
    """indexer_topk with the library's static per-GPU workspace
    (lt_indexer_topk_static): the call allocates no device memory when `out`
    is given. Calls whose work overlaps on one GPU race."""
    _on_gpu(q, w, keys, causal_offsets, q_scale, k_scale)
    _need(q.dim() == 3 and keys.dim() == 2 and q.shape[2] == keys.shape[1], "q [Nq,H,d] and keys [Nk,d] required")
    dt = _dtype_code(q)
    _need(_dtype_code(keys) == dt, "q and keys must share a dtype")
    nq, h, d = q.shape
    nk = keys.shape[0]
    _check_score_inputs(q, w, keys, causal_offsets, q_scale, k_scale, options)
    if out is None:
        out = (torch.empty((nq, k), dtype=torch.int32, device=q.device),
               torch.empty((nq, k), dtype=torch.float32, device=q.device))
    _on_gpu(*out)
    _need(tuple(out[0].shape) == (nq, k) and out[0].dtype == torch.int32 and tuple(out[1].shape) == (nq, k)
          and out[1].dtype == torch.float32, "out must be (int32 [Nq, k], float32 [Nq, k])")
    st = lt_indexer_topk_static(_ptr(q), _ptr(q_scale), _ptr(w), _ptr(keys), _ptr(k_scale), dt, _mode_code(mode), nq,
                                nk, h, d, k, _ptr(causal_offsets), _ptr(out[0]), _ptr(out[1]), options,
                                _stream(stream))
    _check(st, "lt_indexer_topk_static")
    return out


def indexer_scores(q: torch.Tensor, w: Optional[torch.Tensor], keys: torch.Tensor,
                   q_scale: Optional[torch.Tensor] = None, k_scale: Optional[torch.Tensor] = None,
                   mode: str = "dsa", out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Dense float32 index scores [Nq, Nk] (the materialising baseline)."""
    _on_gpu(q, w, keys, q_scale, k_scale)
    _need(q.dim() == 3 and keys.dim() == 2 and q.shape[2] == keys.shape[1], "q [Nq,H,d] and keys [Nk,d] required")
    dt = _dtype_code(q)
    _need(_dtype_code(keys) == dt, "q and keys must share a dtype")
    _check_score_inputs(q, w, keys, None, q_scale, k_scale, None)
    nq, h, d = q.shape
    nk = keys.shape[0]
    if out is None:
        out = torch.empty((nq, nk), dtype=torch.float32, device=q.device)
    _need(out.dim() == 2 and out.shape[0] == nq and out.shape[1] >= nk and out.stride(1) == 1, "bad out")
    st = lt_indexer_scores(_ptr(q), _ptr(q_scale), _ptr(w), _ptr(keys), _ptr(k_scale), dt, _mode_code(mode), nq, nk,
                           h, d, _ptr(out), out.stride(0), _stream(stream))
    _check(st, "lt_indexer_scores")
    return out


def topk_select(scores: torch.Tensor, k: int, num_keys: Optional[int] = None,
                causal_offsets: Optional[torch.Tensor] = None, options: Optional[LtOptions] = None, out=None,
                workspace: Optional[torch.Tensor] = None, stream=None):
    """Exact per-row top-k of a float32 score matrix [Nq, ld] (first num_keys
    columns are keys) through the sample / filter / select pipeline."""
    _need(scores.is_cuda and scores.dtype == torch.float32 and scores.dim() == 2 and scores.stride(1) == 1,
          "scores must be a float32 [Nq, ld] GPU matrix with unit column stride")
    nq = scores.shape[0]
    nk = scores.shape[1] if num_keys is None else num_keys
    _check_rows(nq, causal_offsets, options)
    if out is None:
        out = (torch.empty((nq, k), dtype=torch.int32, device=scores.device),
               torch.empty((nq, k), dtype=torch.float32, device=scores.device))
    if workspace is None:
        n = lt_topk_select_workspace_size(nq, nk, k, options)
        _need(n > 0, "unsupported shape for lt_topk_select")
        workspace = torch.empty(n, dtype=torch.uint8, device=scores.device)
    st = lt_topk_select(_ptr(scores), scores.stride(0), nq, nk, k, _ptr(causal_offsets), _ptr(out[0]),
                        _ptr(out[1]), _ptr(workspace), workspace.numel(), options, _stream(stream))
    _check(st, "lt_topk_select")
    return out


def topk_radix(scores: torch.Tensor, k: int, num_keys: Optional[int] = None,
               causal_offsets: Optional[torch.Tensor] = None, sorted_output: bool = False, out=None, stream=None):
    """Exact per-row top-k by plain radix selection (no filter)."""
    _need(scores.is_cuda and scores.dtype == torch.float32 and scores.dim() == 2 and scores.stride(1) == 1,
          "scores must be a float32 [Nq, ld] GPU matrix with unit column stride")
    nq = scores.shape[0]
    nk = scores.shape[1] if num_keys is None else num_keys
    _check_rows(nq, causal_offsets, None)
    if out is None:
        out = (torch.empty((nq, k), dtype=torch.int32, device=scores.device),
               torch.empty((nq, k), dtype=torch.float32, device=scores.device))
    st = lt_topk_radix(_ptr(scores), scores.stride(0), nq, nk, k, _ptr(causal_offsets), _ptr(out[0]), _ptr(out[1]),
                       LT_SORTED_OUTPUT if sorted_output else 0, _stream(stream))
    _check(st, "lt_topk_radix")
    return out


def sample_from_topk(prev_idx: torch.Tensor, num_keys: int, sample_size: int, out: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The previous chunk's sample (sec. 3.2 "Sampling"): the sample_size keys
    that occur most often in prev_idx [rows, k] (int32, -1 padding ignored),
    ascending, then -1. Returns int32 [sample_size]."""
    _need(prev_idx.is_cuda and prev_idx.dtype == torch.int32 and prev_idx.dim() == 2
          and (prev_idx.numel() == 0 or prev_idx.stride(1) == 1),
          "prev_idx must be an int32 [rows, k] GPU matrix with unit column stride")
    rows, pk = prev_idx.shape
    if out is None:
        out = torch.empty(sample_size, dtype=torch.int32, device=prev_idx.device)
    _need(out.dtype == torch.int32 and out.numel() == sample_size and out.is_contiguous(), "bad out")
    if workspace is None:
        workspace = torch.empty(lt_sample_from_topk_workspace_size(num_keys), dtype=torch.uint8,
                                device=prev_idx.device)
    st = lt_sample_from_topk(_ptr(prev_idx), prev_idx.stride(0) if prev_idx.numel() else pk, rows, pk, num_keys,
                             sample_size, _ptr(out), _ptr(workspace), workspace.numel(), _stream(stream))
    _check(st, "lt_sample_from_topk")
    return out


def dsa_union(topk_idx: torch.Tensor, group: int, stream=None):
    """LiteDSA union (sec. 3.3) of each group of `group` consecutive rows of
    topk_idx [Nq, k] (int32, -1 padding). Returns (union_idx int32
    [G, group * k], union_count int32 [G], member_mask int32 [Nq, W]; the
    mask words are uint32 bit patterns, W = ceil(group * k / 32))."""
    _need(topk_idx.is_cuda and topk_idx.dtype == torch.int32 and topk_idx.dim() == 2
          and (topk_idx.numel() == 0 or topk_idx.stride(1) == 1),
          "topk_idx must be an int32 [Nq, k] GPU matrix with unit column stride")
    nq, k = topk_idx.shape
    _need(group >= 1 and k >= 1 and group * k <= LT_UNION_MAX, "need 1 <= group, group * k <= LT_UNION_MAX")
    ngroups = (nq + group - 1) // group
    words = (group * k + 31) // 32
    dev = topk_idx.device
    uidx = torch.empty((ngroups, group * k), dtype=torch.int32, device=dev)
    ucnt = torch.empty((ngroups,), dtype=torch.int32, device=dev)
    mask = torch.empty((nq, words), dtype=torch.int32, device=dev)
    st = lt_dsa_union(_ptr(topk_idx), topk_idx.stride(0) if topk_idx.numel() else k, nq, k, group, _ptr(uidx),
                      _ptr(ucnt), _ptr(mask), _stream(stream))
    _check(st, "lt_dsa_union")
    return uidx, ucnt, mask


# ---------------------------------------------------------------------------
# serving: page plan, 4-bit cache, attention over it, log probabilities
# ---------------------------------------------------------------------------

# These calls are short beside what surrounds them in a decode step, so their
# checks build no message before one is needed, and the stream handle is read
# without making a Stream object.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_of(stream, t: torch.Tensor) -> int:
    """The HIP stream to work on: `stream`, or the current one of t's device."""
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None:
        return _raw_stream(t.device.index)
    return torch.cuda.current_stream(t.device).cuda_stream


def _int32(t: Optional[torch.Tensor], n: Optional[int], name: str):
    if t is not None and not (t.is_cuda and t.dtype is torch.int32 and t.dim() == 1 and t.is_contiguous()
                              and (n is None or t.numel() == n)):
        raise LiteTopKError("%s must be a contiguous int32 vector%s on the GPU"
                            % (name, "" if n is None else " of %d entries" % n))


def _table(t: torch.Tensor, rows: int):
    """block_table int32 [rows, width] with unit column stride."""
    s = t.shape
    if not (t.is_cuda and t.dtype is torch.int32 and len(s) == 2 and s[0] == rows
            and (rows == 0 or s[1] <= 1 or t.stride(1) == 1)):
        raise LiteTopKError("block_table must be an int32 [requests, pages] GPU matrix with unit column stride")
    return t.stride(0) if rows > 1 and s[1] > 0 else s[1], s[1]


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """Memory for work on `stream`, from that stream's own: what the current
    stream's allocator hands out may still be read by work queued there."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _workspace(t: Optional[torch.Tensor], need: int, device, stream) -> torch.Tensor:
    """`need` bytes for work on `stream`, or the caller's (whose memory may belong to
    another stream; its size is checked by the call)."""
    if t is None:
        return _empty(need, torch.uint8, device, stream)
    if not (t.is_cuda and t.is_contiguous()):
        raise LiteTopKError("workspace must be contiguous memory on the GPU")
    if stream is not None:
        t.record_stream(stream)
    return t


def _used_on(stream, *ts):
    """Results on `stream`'s memory, which the caller goes on to use on the current
    stream: keep the allocator from handing them out before that work has run."""
    if stream is not None:
        now = torch.cuda.current_stream()
        if stream.cuda_stream != now.cuda_stream:
            for t in ts:
                if t is not None and t.numel():
                    t.record_stream(now)


class PagedPlan(NamedTuple):
    """What paged_plan returns; see lt_paged_plan in the header."""
    cu_tokens: torch.Tensor   # int32 [R + 1]
    seq_lens: torch.Tensor    # int32 [R]
    slots: torch.Tensor       # int64 [token_capacity]
    positions: torch.Tensor   # int32 [token_capacity]
    free_used: torch.Tensor   # int32 [1]: pages of the free list now in use
    status: torch.Tensor      # int32 [R]: 0 served, 1 table too narrow, 2 out of pages


def paged_plan(context_lens: torch.Tensor, new_lens: torch.Tensor, block_table: torch.Tensor,
               free_pages: torch.Tensor, free_used: torch.Tensor, page_size: int, token_capacity: int,
               stream=None) -> PagedPlan:
    """Block tables and slot maps of a step, built on the GPU from the
    requests' lengths (int32 [R] each): pages for the new tokens are taken from
    free_pages [free_used[0]:] in request order and entered into block_table
    [R, W] (in place), and every new token gets its slot and position. Look at
    `status` before the step goes on: the tokens of a request that was not served
    have no slots, but cache4_attention would still give them a result."""
    n = context_lens.numel()
    _int32(context_lens, None, "context_lens")
    _int32(new_lens, n, "new_lens")
    _int32(free_pages, None, "free_pages")
    _int32(free_used, 1, "free_used")
    _need(token_capacity >= 0, "token_capacity must not be negative")
    ld, width = _table(block_table, n)
    dev = context_lens.device
    # the 32-bit results in one allocation
    cu, seq, used, status, positions = _empty(3 * n + 2 + token_capacity, torch.int32, dev, stream).split_with_sizes(
        (n + 1, n, 1, n, token_capacity))
    p = PagedPlan(cu, seq, _empty(token_capacity, torch.int64, dev, stream), positions, used, status)
    st = lt_paged_plan(_ptr(context_lens), _ptr(new_lens), n, page_size, _ptr(block_table), ld, width,
                       _ptr(free_pages), free_pages.numel(), _ptr(free_used), token_capacity, _ptr(p.cu_tokens),
                       _ptr(p.seq_lens), _ptr(p.slots), _ptr(p.positions), _ptr(p.free_used), _ptr(p.status),
                       _stream_of(stream, context_lens))
    _check(st, "lt_paged_plan")
    _used_on(stream, *p)
    return p


def cache4_empty(num_pages: int, page_size: int, kv_heads: int, head_dim: int, device=None):
    """An empty 4-bit cache: (codes uint8 [pages, kv_heads, page_size, 2,
    head_dim / 2], scales uint8 [pages, kv_heads, page_size, 2, head_dim / 32])."""
    dev = device or "cuda"
    return (torch.zeros((num_pages, kv_heads, page_size, 2, head_dim // 2), dtype=torch.uint8, device=dev),
            torch.zeros((num_pages, kv_heads, page_size, 2, head_dim // 32), dtype=torch.uint8, device=dev))


def _cache4(codes: torch.Tensor, scales: torch.Tensor):
    """(pages, page size, KV heads, head dim) of a 4-bit cache."""
    _on_gpu(codes, scales)
    a, b = codes.shape, scales.shape    # each use of .shape builds it anew
    if not (codes.dtype is torch.uint8 and scales.dtype is torch.uint8 and len(a) == 5 and len(b) == 5
            and a[0] == b[0] and a[1] == b[1] and a[2] == b[2] and a[3] == b[3] == 2 and a[4] == 16 * b[4]):
        raise LiteTopKError("a cache is codes uint8 [pages, heads, page_size, 2, d / 2] and scales uint8 [pages, "
                            "heads, page_size, 2, d / 32]")
    return a[0], a[2], a[1], 2 * a[4]


def _rows_of(t: torch.Tensor, heads: int, d: int, name: str) -> int:
    """Stride between the rows of a [rows, heads, d] tensor whose rows are contiguous."""
    s = t.shape
    whole = t.is_contiguous()
    if not (t.is_cuda and len(s) == 3 and s[1] == heads and s[2] == d
            and (whole or (t.stride(2) == 1 and (heads == 1 or t.stride(1) == d)))):
        raise LiteTopKError("%s must be [rows, %d, %d] on the GPU with contiguous rows" % (name, heads, d))
    return heads * d if whole or s[0] <= 1 else t.stride(0)


def cache4_append(k: torch.Tensor, v: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, slots: torch.Tensor,
                  stream=None) -> None:
    """Quantises the keys and values [rows, kv_heads, head_dim] (float32 or
    bfloat16) into the cache's slots (int64 [rows], distinct; -1 = leave out)."""
    pages, page, heads, d = _cache4(codes, scales)
    ks, vs = _rows_of(k, heads, d, "k"), _rows_of(v, heads, d, "v")
    _need(k.dtype == v.dtype and k.dtype in (torch.float32, torch.bfloat16) and k.shape[0] == v.shape[0],
          "k and v must have as many rows of one type, float32 or bfloat16")
    _on_gpu(slots)
    _need(slots.dtype == torch.int64 and slots.dim() == 1 and slots.numel() == k.shape[0],
          "slots must be int64 [rows]")
    st = lt_cache4_append(_ptr(k), _ptr(v), _dtype_code(k), ks, vs, k.shape[0], _ptr(codes), _ptr(scales), pages,
                          page, heads, d, _ptr(slots), _stream_of(stream, k))
    _check(st, "lt_cache4_append")


def cache4_read(codes: torch.Tensor, scales: torch.Tensor, slots: torch.Tensor, stream=None):
    """The (keys, values) that slots (int64 [rows]) hold, bfloat16 [rows,
    kv_heads, head_dim] each; zeros for slots outside the cache."""
    pages, page, heads, d = _cache4(codes, scales)
    _on_gpu(slots)
    _need(slots.dtype == torch.int64 and slots.dim() == 1, "slots must be int64 [rows]")
    n = slots.numel()
    k = _empty((n, heads, d), torch.bfloat16, slots.device, stream)
    v = _empty((n, heads, d), torch.bfloat16, slots.device, stream)
    st = lt_cache4_read(_ptr(codes), _ptr(scales), pages, page, heads, d, _ptr(slots), n, _ptr(k), _ptr(v),
                        _stream_of(stream, slots))
    _check(st, "lt_cache4_read")
    _used_on(stream, k, v)
    return k, v


def cache4_attention(q: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, block_table: torch.Tensor,
                     cu_tokens: torch.Tensor, seq_lens: torch.Tensor, scale: Optional[float] = None,
                     visible_start: Optional[torch.Tensor] = None, visible_end: Optional[torch.Tensor] = None,
                     selected: Optional[torch.Tensor] = None, selected_start: Optional[torch.Tensor] = None,
                     return_lse: bool = True, workspace: Optional[torch.Tensor] = None, stream=None):
    """Attention of q [T, heads, head_dim] (bfloat16) over the 4-bit cache:
    tokens [cu_tokens[r], cu_tokens[r + 1]) belong to request r, which has
    seq_lens[r] cached keys on the pages of block_table[r]. Token t sees the keys
    [visible_start[t], visible_end[t]) (defaults: 0, and causal), and with
    `selected` int32 [T, k] only those on its list (indexer_topk's result; minus
    selected_start[t] for sequences packed into one key array). Scale defaults to
    head_dim ** -0.5. Returns (out bfloat16 like q, lse float32 [T, heads] or
    None)."""
    pages, page, hkv, d = _cache4(codes, scales)
    shape = q.shape
    _need(len(shape) == 3 and q.dtype is torch.bfloat16, "q must be bfloat16 [T, heads, head_dim]")
    tokens, hq = shape[0], shape[1]
    qs = _rows_of(q, hq, d, "q")
    _int32(seq_lens, None, "seq_lens")
    n = seq_lens.numel()
    _int32(cu_tokens, n + 1, "cu_tokens")
    _int32(visible_start, tokens, "visible_start")
    _int32(visible_end, tokens, "visible_end")
    _int32(selected_start, tokens, "selected_start")
    ld, width = _table(block_table, n)
    k, sel_ld = 0, 0
    if selected is not None:
        _need(selected.is_cuda and selected.dtype == torch.int32 and selected.dim() == 2
              and selected.shape[0] == tokens and selected.shape[1] >= 1
              and (selected.shape[1] == 1 or selected.stride(1) == 1 or tokens == 0),
              "selected must be an int32 [T, k] GPU matrix with unit column stride")
        k = selected.shape[1]
        sel_ld = selected.stride(0) if tokens > 1 else k
    out = _empty((tokens, hq, d), torch.bfloat16, q.device, stream)
    lse = _empty((tokens, hq), torch.float32, q.device, stream) if return_lse else None
    need = lt_cache4_attention_workspace_size(tokens, n, hq, hkv, d, k)
    _need(need > 0, "unsupported shape for lt_cache4_attention")
    workspace = _workspace(workspace, need, q.device, stream)
    st = lt_cache4_attention(_ptr(q), qs, tokens, hq, d, _ptr(codes), _ptr(scales), pages, page, hkv,
                             _ptr(block_table), ld, width, _ptr(cu_tokens), _ptr(seq_lens), n, _ptr(visible_start),
                             _ptr(visible_end), _ptr(selected), sel_ld, k, _ptr(selected_start),
                             d ** -0.5 if scale is None else scale, _ptr(out), _ptr(lse), _ptr(workspace),
                             workspace.numel(), _stream_of(stream, q))
    _check(st, "lt_cache4_attention")
    _used_on(stream, out, lse)
    return out, lse


class TokenLogprobs(NamedTuple):
    """What token_logprobs returns; see lt_token_logprobs in the header."""
    logprob: torch.Tensor      # float32 [rows]
    entropy: torch.Tensor      # float32 [rows]
    lse: torch.Tensor          # float32 [rows]
    top_index: torch.Tensor    # int32 [rows, top]
    top_logprob: torch.Tensor  # float32 [rows, top]


def _logits(logits: torch.Tensor, tokens: torch.Tensor) -> int:
    _need(logits.is_cuda and logits.dim() == 2 and logits.dtype in (torch.float32, torch.bfloat16)
          and (logits.numel() == 0 or logits.shape[1] == 1 or logits.stride(1) == 1),
          "logits must be a float32 or bfloat16 [rows, vocab] GPU matrix with unit column stride")
    _on_gpu(tokens)
    _need(tokens.dtype == torch.int64 and tokens.dim() == 1 and tokens.numel() == logits.shape[0],
          "tokens must be int64 [rows]")
    return logits.stride(0) if logits.shape[0] > 1 and logits.shape[1] > 0 else logits.shape[1]


def token_logprobs(logits: torch.Tensor, tokens: torch.Tensor, top: int = 0, scale: float = 1.0,
                   workspace: Optional[torch.Tensor] = None, stream=None) -> TokenLogprobs:
    """Log probability of each row's token under softmax(scale * logits), the
    row's entropy, log normaliser and `top` best alternatives with their log
    probabilities (higher logit first, equal ones by index). A token outside the
    vocabulary (-1) is not counted: its log probability is 0. The results are not
    part of an autograd graph, whether or not the logits are: their gradient is
    token_logprobs_backward's."""
    ld = _logits(logits, tokens)
    rows, vocab = logits.shape
    dt, dev = _dtype_code(logits), logits.device
    need = lt_token_logprobs_workspace_size(dt, rows, vocab, top)
    _need(need > 0, "unsupported shape for lt_token_logprobs (top must be 0..%d)" % LT_LOGPROB_MAX_TOP)
    workspace = _workspace(workspace, need, dev, stream)
    n = min(top, vocab)
    f = _empty(rows * (3 + n), torch.float32, dev, stream)
    logprob, entropy, lse, best = f.split_with_sizes((rows, rows, rows, rows * n))
    r = TokenLogprobs(logprob, entropy, lse, _empty((rows, n), torch.int32, dev, stream), best.view(rows, n))
    st = lt_token_logprobs(_ptr(logits), dt, ld, rows, vocab, _ptr(tokens), scale, n, _ptr(r.logprob),
                           _ptr(r.entropy), _ptr(r.lse), _ptr(r.top_index), _ptr(r.top_logprob), _ptr(workspace),
                           workspace.numel(), _stream_of(stream, logits))
    _check(st, "lt_token_logprobs")
    _used_on(stream, f, r.top_index)
    return r


def token_logprobs_backward(logits: torch.Tensor, tokens: torch.Tensor, lse: torch.Tensor, entropy: torch.Tensor,
                            grad_logprob: Optional[torch.Tensor] = None, grad_entropy: Optional[torch.Tensor] = None,
                            scale: float = 1.0, stream=None) -> torch.Tensor:
    """The logits' gradient (in their type) from those of token_logprobs'
    logprob and entropy (float32 [rows], None = zero) and its lse and entropy.
    For a training step pass the result on: logits.backward(gradient)."""
    ld = _logits(logits, tokens)
    rows, vocab = logits.shape
    for t in (lse, entropy, grad_logprob, grad_entropy):
        _on_gpu(t)
        _need(t is None or (t.dtype == torch.float32 and t.dim() == 1 and t.numel() == rows),
              "lse, entropy and the gradients must be float32 [rows]")
    # rows start on a line: full-width stores whatever the vocabulary's size
    pad = (vocab + 63) // 64 * 64
    out = _empty((rows, pad), logits.dtype, logits.device, stream)[:, :vocab]
    st = lt_token_logprobs_backward(_ptr(logits), _dtype_code(logits), ld, rows, vocab, _ptr(tokens), scale, _ptr(lse),
                                    _ptr(entropy), _ptr(grad_logprob), _ptr(grad_entropy), _ptr(out), pad,
                                    _stream_of(stream, logits))
    _check(st, "lt_token_logprobs_backward")
    _used_on(stream, out)
    return out


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------

class Rotary(NamedTuple):
    """How positions turn a head: `inv_freq` (float32 [pairs] on the GPU, radians a
    position) turns the values [start, start + 2 * pairs), paired (i, i + pairs) or
    interleaved (2 i, 2 i + 1); sine and cosine are multiplied by `amplitude`."""
    inv_freq: torch.Tensor
    start: int = 0
    interleaved: bool = False
    amplitude: float = 1.0


def rotary_frequencies(dim: int, base: float = 10000.0, method: str = "none", factor: float = 1.0,
                       original_length: int = 0, low: Optional[float] = None, high: Optional[float] = None,
                       start: int = 0, interleaved: bool = False, amplitude: Optional[float] = None,
                       device=None) -> Rotary:
    """The Rotary of frequencies f_i = base ** (-2 i / dim), i < dim / 2, scaled for
    contexts `factor` times as long as the `original_length` positions trained on:

    none      as they are
    linear    f_i / factor: positions are interpolated
    base      a base of base * factor ** (dim / (dim - 2)): the first frequency stays, the
              last is divided by factor
    ramp      f_i / factor below a ramp over the index i, f_i above it: the ramp ends where
              a frequency turns `low` (1) and `high` (32) times over original_length;
              amplitude 0.1 ln(factor) + 1
    turns     the same with the ramp over the number of turns, from `low` (1) to `high` (4)

    These are published methods: linear is position interpolation (Chen et al. 2023,
    arXiv 2306.15595), ramp with its amplitude and the ramp over turns are those of Peng et
    al. 2023 (YaRN, arXiv 2309.00071, which also describes the scaled base).

    amplitude overrides the method's (1 but for ramp)."""
    _need(dim >= 2 and dim % 2 == 0, "dim must be even and positive")
    _need(base > 0.0 and factor > 0.0, "base and factor must be positive")
    n = dim // 2
    two_pi = 2.0 * math.pi
    if method == "base":
        _need(dim > 2, "method 'base' needs dim > 2")
        base = base * factor ** (dim / (dim - 2.0))
    f = [base ** (-2.0 * i / dim) for i in range(n)]
    amp = 1.0
    if method == "linear":
        f = [x / factor for x in f]
    elif method in ("ramp", "turns"):
        _need(original_length > 0, "methods 'ramp' and 'turns' need original_length")
        lo = 1.0 if low is None else float(low)
        hi = (32.0 if method == "ramp" else 4.0) if high is None else float(high)
        _need(0.0 < lo < hi, "need 0 < low < high")
        if method == "turns":
            keep = [(original_length * x / two_pi - lo) / (hi - lo) for x in f]
        else:
            _need(base > 1.0, "method 'ramp' needs base > 1")
            # the (real) index whose frequency turns r times over original_length
            at = [dim * math.log(original_length / (r * two_pi)) / (2.0 * math.log(base)) for r in (hi, lo)]
            first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), dim - 1)
            keep = [1.0 - (i - first) / max(last - first, 1e-3) for i in range(n)]
            amp = 0.1 * math.log(factor) + 1.0 if factor > 1.0 else 1.0
        keep = [min(max(x, 0.0), 1.0) for x in keep]
        f = [x * k + x / factor * (1.0 - k) for x, k in zip(f, keep)]
    elif method not in ("none", "base"):
        raise LiteTopKError("method must be 'none', 'linear', 'base', 'ramp' or 'turns'")
    t = torch.tensor(f, dtype=torch.float64).float().to(device or "cuda")
    return Rotary(t, start, interleaved, amp if amplitude is None else amplitude)


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _here(*ts):
    """All tensors on one GPU, the current one (which launches go to). Its index is read
    off the tensors without making a device object of any."""
    i = ts[0].get_device()
    for t in ts:
        if t is not None and t.get_device() != i:
            raise LiteTopKError("tensors must be on one GPU")
    if i < 0:
        raise LiteTopKError("tensors must be on the GPU")
    if i != _current_device():
        raise LiteTopKError("tensors are on GPU %d, which is not the current device" % i)


def _heads(t: torch.Tensor, name: str):
    """Shape of [tokens, heads, head_dim] in float32 or bfloat16, rows contiguous."""
    s = t.shape
    if not (len(s) == 3 and (t.dtype is torch.bfloat16 or t.dtype is torch.float32)
            and (t.is_contiguous() or s[2] == 1 or t.stride(2) == 1 or t.numel() == 0)):
        raise LiteTopKError("%s must be float32 or bfloat16 [tokens, heads, head_dim] with contiguous heads" % name)
    return s


def _turn(rot: Rotary, d: int):
    f = rot.inv_freq
    if not (f.dtype is torch.float32 and f.dim() == 1 and f.is_contiguous()):
        raise LiteTopKError("inv_freq must be a contiguous float32 vector on the GPU")
    n = f.shape[0]
    if rot.start < 0 or rot.start + 2 * n > d:
        raise LiteTopKError("the rotated part [%d, %d) is not inside a head of %d" % (rot.start, rot.start + 2 * n, d))
    return n


def _rotate(x, positions, rot, out, out_dtype, flags, stream):
    t, h, d = _heads(x, "x")
    n = _turn(rot, d)
    f = rot.inv_freq
    _int32(positions, t, "positions")
    _here(x, positions, f, out)
    fresh = out is None
    kind = x.dtype
    if fresh:
        out_kind = out_dtype or kind
        out = x.new_empty((t, h, d), dtype=out_kind) if stream is None else _empty((t, h, d), out_kind, x.device, stream)
        ot, oh = h * d, d
    else:
        out_kind = out.dtype
        if not (_heads(out, "out") == x.shape and (out_dtype is None or out_dtype is out_kind)):
            raise LiteTopKError("out must have x's shape, and out_dtype if that is given")
        ot, oh = out.stride(0), out.stride(1)
    xt, xh = x.stride(0), x.stride(1)
    if out_kind is torch.bfloat16:
        out_code = LT_BF16
    else:
        out_code = _dtype_code(out)
    st = load().lt_rotary(x.data_ptr(), LT_BF16 if kind is torch.bfloat16 else LT_F32, xt, xh, t, h, d,
                          positions.data_ptr(), f.data_ptr(), n, rot.start, rot.amplitude,
                          flags | 1 if rot.interleaved else flags, out.data_ptr(), out_code, ot, oh,
                          _stream_of(stream, x))
    if st:
        _check(st, "lt_rotary")
    if fresh and stream is not None:
        _used_on(stream, out)
    return out


def rotary(x: torch.Tensor, positions: torch.Tensor, rot: Rotary, out: Optional[torch.Tensor] = None,
           out_dtype: Optional[torch.dtype] = None, stream=None) -> torch.Tensor:
    """x [T, heads, head_dim] (float32 or bfloat16, any strides between heads and
    tokens: a slice of a common projection will do) with every head turned by its
    token's position (int32 [T]; negative = padding, which becomes zeros). The result
    has x's type, or is bfloat16 (out_dtype); `out` may be x. It is not part of an
    autograd graph: its gradient is rotary_backward's."""
    return _rotate(x, positions, rot, out, out_dtype, 0, stream)


def rotary_backward(grad: torch.Tensor, positions: torch.Tensor, rot: Rotary, out: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """The gradient of rotary's x from that of its result: turned back, times the
    amplitude in the rotated part."""
    return _rotate(grad, positions, rot, out, None, LT_ROTARY_INVERSE, stream)


def rotary_fp8(x: torch.Tensor, positions: torch.Tensor, rot: Rotary, out=None, stream=None):
    """The same as fp8, for indexer_topk: (codes float8_e4m3fn [T, heads, head_dim],
    scales float32 [T, heads]); scales are powers of two. For keys (one head) view them
    as [T, head_dim] and [T]; `out` = (codes, scales) writes into an array of them."""
    t, h, d = _heads(x, "x")
    n = _turn(rot, d)
    _int32(positions, t, "positions")
    _here(x, positions, rot.inv_freq)
    if out is None:
        codes = _empty((t, h, d), torch.float8_e4m3fn, x.device, stream)
        scales = _empty((t, h), torch.float32, x.device, stream)
    else:
        codes, scales = out
        _on_gpu(codes, scales)
        _need(codes.dtype in (torch.float8_e4m3fn, torch.uint8) and codes.shape == x.shape
              and scales.dtype == torch.float32 and scales.shape == x.shape[:2],
              "out must be codes float8_e4m3fn [T, heads, head_dim] and scales float32 [T, heads]")
        _here(x, codes, scales)
    st = lt_rotary_fp8(_ptr(x), _dtype_code(x), x.stride(0), x.stride(1), t, h, d, _ptr(positions),
                       _ptr(rot.inv_freq), n, rot.start, rot.amplitude,
                       LT_ROTARY_INTERLEAVED if rot.interleaved else 0, _ptr(codes), _ptr(scales),
                       _stream_of(stream, x))
    _check(st, "lt_rotary_fp8")
    if out is None:
        _used_on(stream, codes, scales)
    return codes, scales


def cache4_append_rotary(k: torch.Tensor, v: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor,
                         slots: torch.Tensor, positions: torch.Tensor, rot: Rotary, q: Optional[torch.Tensor] = None,
                         stream=None) -> Optional[torch.Tensor]:
    """cache4_append with the keys turned by their positions (int32 [rows], as
    paged_plan gives them) on the way. With q [rows, heads, head_dim] (of k's type) the
    same launch turns the queries: returns them in bfloat16, for cache4_attention."""
    pages, page, heads, d = _cache4(codes, scales)
    ks, vs = _rows_of(k, heads, d, "k"), _rows_of(v, heads, d, "v")
    rows = k.shape[0]
    if not (k.dtype is v.dtype and k.dtype in (torch.float32, torch.bfloat16) and v.shape[0] == rows):
        raise LiteTopKError("k and v must have as many rows of one type, float32 or bfloat16")
    if not (slots.dtype is torch.int64 and slots.dim() == 1 and slots.is_contiguous() and slots.numel() == rows):
        raise LiteTopKError("slots must be a contiguous int64 [rows]")
    _int32(positions, rows, "positions")
    n = _turn(rot, d)
    _here(k, v, codes, scales, slots, positions, rot.inv_freq, q)
    hq, qs, out = 0, 0, None
    if q is not None:
        if not (q.dtype is k.dtype and q.dim() == 3 and q.shape[0] == rows and q.shape[1] >= 1):
            raise LiteTopKError("q must be [rows, heads, head_dim] of k's type")
        hq = q.shape[1]
        qs = _rows_of(q, hq, d, "q")
        out = _empty((rows, hq, d), torch.bfloat16, k.device, stream)
    st = load().lt_cache4_append_rotary(_ptr(k), _ptr(v), _dtype_code(k), ks, vs, rows, _ptr(codes), _ptr(scales), pages, page,
                                 heads, d, _ptr(slots), _ptr(positions), _ptr(rot.inv_freq), n, rot.start,
                                 rot.amplitude, LT_ROTARY_INTERLEAVED if rot.interleaved else 0,
                                 _ptr(q) if rows else None, qs, hq if rows else 0, _ptr(out), _stream_of(stream, k))
    _check(st, "lt_cache4_append_rotary")
    _used_on(stream, out)
    return out


# ---------------------------------------------------------------------------
# beam search
# ---------------------------------------------------------------------------

class BeamCandidates(NamedTuple):
    """What beam_select returns, best first; see lt_beam_select in the header."""
    score: torch.Tensor   # float32 [requests, top]; -inf behind the last candidate
    beam: torch.Tensor    # int32 [requests, top], -1 there
    token: torch.Tensor   # int32 [requests, top], -1 there


def beam_select(logits: torch.Tensor, scores: torch.Tensor, top: int, scale: float = 1.0,
                workspace: Optional[torch.Tensor] = None, stream=None) -> BeamCandidates:
    """The `top` best continuations of every request over its beams and the
    vocabulary: logits [requests * beams, vocab] (float32 or bfloat16), scores [requests,
    beams] (float32: the beams' log probabilities so far, -inf for a beam that is not
    alive, as all but one are in the first step). A program that lets beams finish asks
    for more continuations than it has beams."""
    if not (logits.dim() == 2 and (logits.dtype is torch.bfloat16 or logits.dtype is torch.float32)
            and (logits.is_contiguous() or logits.shape[1] == 1 or logits.stride(1) == 1 or logits.numel() == 0)):
        raise LiteTopKError("logits must be a float32 or bfloat16 [requests * beams, vocab] GPU matrix with unit "
                            "column stride")
    if not (scores.dim() == 2 and scores.dtype is torch.float32 and scores.is_contiguous()
            and scores.numel() == logits.shape[0]):
        raise LiteTopKError("scores must be float32 [requests, beams], contiguous")
    _here(logits, scores, workspace)
    dev = logits.device
    reqs, beams = scores.shape
    rows, vocab = logits.shape
    dt = LT_BF16 if logits.dtype is torch.bfloat16 else LT_F32
    lib = load()
    need = lib.lt_beam_select_workspace_size(dt, reqs, beams, vocab, top)
    if need == 0:
        raise LiteTopKError("unsupported shape for lt_beam_select (top must be 1..%d, beams 1..%d)"
                            % (LT_BEAM_MAX_TOP, LT_BEAM_MAX_BEAMS))
    workspace = _workspace(workspace, need, dev, stream)
    # the results in one allocation
    score, beam, token = _empty((3, reqs, top), torch.int32, dev, stream).unbind(0)
    r = BeamCandidates(score.view(torch.float32), beam, token)
    st = lib.lt_beam_select(logits.data_ptr(), dt, logits.stride(0) if rows > 1 and vocab > 0 else vocab, reqs, beams,
                            vocab, scores.data_ptr(), scale, top, score.data_ptr(), beam.data_ptr(), token.data_ptr(),
                            workspace.data_ptr(), workspace.numel(), _stream_of(stream, logits))
    if st:
        _check(st, "lt_beam_select")
    if stream is not None:
        _used_on(stream, *r)
    return r


class PagedReorder(NamedTuple):
    """What paged_reorder returns; see lt_paged_reorder in the header."""
    block_table: torch.Tensor  # int32 [rows, width]
    seq_lens: torch.Tensor     # int32 [rows]
    copies: torch.Tensor       # int32 [rows, 2]: page to copy, page to write (-1, -1: none)
    free_used: torch.Tensor    # int32 [1]
    status: torch.Tensor       # int32 [rows]: 0 goes on, 1 ended by its parent, 2 out of pages


def paged_reorder(block_table: torch.Tensor, seq_lens: torch.Tensor, parents: torch.Tensor, group: int,
                  free_pages: torch.Tensor, free_used: torch.Tensor, page_size: int,
                  keep_pages: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                  stream=None) -> PagedReorder:
    """Rows of a paged cache go on as their parents (int32 [rows], counted within each
    group of `group` rows; outside [0, group): the row ends). Full pages are shared,
    partial ones copied for all children but the first: pass `copies` to cache4_copy for
    each layer. Pages that no row holds any more go back onto free_pages (in place,
    before free_used). block_table [rows, width], seq_lens, free_pages and free_used are
    paged_plan's."""
    n = seq_lens.numel()
    for t, size, name in ((seq_lens, n, "seq_lens"), (parents, n, "parents"), (free_pages, None, "free_pages"),
                          (free_used, 1, "free_used"), (keep_pages, n, "keep_pages")):
        _int32(t, size, name)
    ld, width = _table(block_table, n)
    _here(block_table, seq_lens, parents, free_pages, free_used, keep_pages, workspace)
    dev = block_table.device
    lib = load()
    need = lib.lt_paged_reorder_workspace_size(n)
    if need == 0:
        raise LiteTopKError("at most %d rows" % LT_PLAN_MAX_REQUESTS)
    # the results in one allocation, and behind them the workspace (16 bytes a row)
    many = n * (width + 4) + 1
    if workspace is None:
        pad = -many % 64
        table, lens, copies, used, status, _, workspace = _empty(
            many + pad + need // 4, torch.int32, dev, stream).split_with_sizes((n * width, n, 2 * n, 1, n, pad, need // 4))
    else:
        workspace = _workspace(workspace, need, dev, stream)
        need = workspace.numel() * workspace.element_size()
        table, lens, copies, used, status = _empty(many, torch.int32, dev, stream).split_with_sizes(
            (n * width, n, 2 * n, 1, n))
    r = PagedReorder(table.view(n, width), lens, copies.view(n, 2), used, status)
    st = lib.lt_paged_reorder(block_table.data_ptr(), ld, width, seq_lens.data_ptr(), parents.data_ptr(), n, group,
                              page_size, _ptr(keep_pages), free_pages.data_ptr(), free_pages.numel(),
                              free_used.data_ptr(), table.data_ptr(), width, lens.data_ptr(), copies.data_ptr(),
                              used.data_ptr(), status.data_ptr(), workspace.data_ptr(), need,
                              _stream_of(stream, block_table))
    if st:
        _check(st, "lt_paged_reorder")
    if stream is not None:
        _used_on(stream, *r)
    return r


def cache4_copy(codes: torch.Tensor, scales: torch.Tensor, copies: torch.Tensor, stream=None) -> None:
    """Copies whole pages of a 4-bit cache: copies int32 [n, 2], page to copy and page
    to write, as paged_reorder gives them; pairs with a page outside the cache (-1) are
    left out."""
    pages, page, heads, d = _cache4(codes, scales)
    if not (copies.dtype is torch.int32 and copies.dim() == 2 and copies.shape[1] == 2 and copies.is_contiguous()):
        raise LiteTopKError("copies must be a contiguous int32 [n, 2] on the GPU")
    _here(codes, scales, copies)
    st = lt_cache4_copy(_ptr(codes), _ptr(scales), pages, page, heads, d, _ptr(copies), copies.shape[0],
                        _stream_of(stream, codes))
    _check(st, "lt_cache4_copy")
