"""Thin ctypes binding over ``libmsa_b200.so`` (the C ABI of ``include/msa.h``).

Argument marshalling only: tensors become device pointers, the current torch stream
becomes the stream argument, status codes become exceptions.  Every step of the path runs
in the CUDA kernels of the library.  If the library is missing this module raises; there
is no CPU fallback.
"""

from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

import torch

from .inputs import MSAConfig

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmsa_b200.so")
_lib: Optional[ctypes.CDLL] = None

c_i64, c_i32, c_vp, c_sz = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t

EXPORTS = [
    "msa_status_string", "msa_check_async_status", "msa_index_scores", "msa_index_scores_decode",
    "msa_topk_select", "msa_topk_select_decode", "msa_sparse_attn_prefill",
    "msa_sparse_attn_prefill_workspace_bytes", "msa_sparse_attn_prefill_static",
    "msa_sparse_attn_decode",
    "msa_sparse_attn_decode_workspace_bytes", "msa_index_topk_fused", "msa_index_lse_prefill",
    "msa_index_lse_prefill_workspace_bytes", "msa_prefill_forward",
    "msa_prefill_forward_workspace_bytes", "msa_prefill_forward_varlen",
    "msa_prefill_forward_varlen_workspace_bytes", "msa_prefill_forward_host",
    "msa_prefill_forward_host_workspace_bytes", "msa_decode_forward", "msa_decode_forward_host",
    "msa_launch_count", "msa_profile_begin", "msa_profile_end", "msa_index_scores_plan", "msa_debug_set_wait",
    "msa_qk_norm_rope", "msa_norm_rope_plan", "msa_qk_norm_rope_backward", "msa_qk_norm_rope_backward_workspace_bytes", "msa_paged_append",
    "msa_paged_attn", "msa_paged_attn_workspace_bytes", "msa_paged_weights", "msa_paged_weights_workspace_bytes",
    "msa_paged_keep", "msa_paged_compact", "msa_sample",
]


class MsaShape(ctypes.Structure):
    _fields_ = [("n_q_heads", c_i32), ("n_kv_heads", c_i32), ("head_dim", c_i32),
                ("idx_dim", c_i32), ("block_size", c_i32), ("top_k", c_i32),
                ("softmax_scale", ctypes.c_float), ("index_scale", ctypes.c_float),
                ("idx_fp8", c_i32), ("kv_fp8", c_i32), ("q_fp8", c_i32), ("score_runs", c_i32)]


class MsaRope(ctypes.Structure):
    _fields_ = [("freqs", c_vp), ("rot_dim", c_i32), ("interleaved", c_i32), ("mscale", ctypes.c_float)]


class MsaPagedCache(ctypes.Structure):
    _fields_ = [("k", c_vp), ("v", c_vp), ("page_table", c_vp), ("kv_lens", c_vp), ("cu_q", c_vp), ("batch", c_i32),
                ("max_pages", c_i32), ("n_pages", c_i32), ("page_size", c_i32), ("n_kv_heads", c_i32),
                ("head_dim", c_i32), ("fp8", c_i32), ("max_new", c_i32)]


class MsaSampling(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_float), ("top_k", c_i32), ("top_p", ctypes.c_float), ("min_p", ctypes.c_float),
                ("temperatures", c_vp), ("top_ks", c_vp), ("top_ps", c_vp), ("min_ps", c_vp)]


class MsaError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s failed: %s (status %d)" % (where, status_string(code), code))


def lib() -> ctypes.CDLL:
    """Loads the CUDA library; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "CUDA library %s is missing: build it with "
                "`python -m paper_2606_13392_b200.build` (needs nvcc, sm_100a)" % LIB_PATH)
        _lib = ctypes.CDLL(LIB_PATH)
        _lib.msa_status_string.restype = ctypes.c_char_p
        _lib.msa_status_string.argtypes = [c_i32]
        _lib.msa_launch_count.restype = c_i64
        for name in EXPORTS:
            if name not in ("msa_status_string", "msa_launch_count"):
                getattr(_lib, name).restype = c_i32
    return _lib


def status_string(code: int) -> str:
    return lib().msa_status_string(code).decode()


def shape_of(cfg: MSAConfig, softmax_scale: float = 0.0, index_scale: float = 0.0, score_runs: int = 0) -> MsaShape:
    return MsaShape(cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.idx_dim, cfg.block_size,
                    cfg.top_k, softmax_scale, index_scale, 1 if cfg.idx_fp8 else 0, 1 if cfg.kv_fp8 else 0,
                    1 if getattr(cfg, "q_fp8", False) else 0, score_runs)


def _ptr(t) -> c_vp:
    if t is None:
        return c_vp(0)
    assert t.is_contiguous(), "tensors passed to the C ABI must be contiguous"
    return c_vp(t.data_ptr())


def _dev(t: Optional[torch.Tensor]):
    if t is not None:
        assert t.is_cuda, "device pointer expected"
    return _ptr(t)


def _idx(shape, t: Optional[torch.Tensor], host: bool = False):
    """An index-branch operand: its element size must match the shape's idx_fp8 flag."""
    if t is not None:
        want = 1 if shape.idx_fp8 else 2
        assert t.element_size() == want, "index operand element size %d, shape expects %d" % (
            t.element_size(), want)
    return _host(t) if host else _dev(t)


def _kv(shape, t: Optional[torch.Tensor]):
    """A K or V tensor (device): its element size must match the shape's kv_fp8 flag."""
    if t is not None:
        want = 1 if shape.kv_fp8 else 2
        assert t.element_size() == want, "K/V cache element size %d, shape expects %d" % (t.element_size(), want)
    return _dev(t)


def _q(shape, t: Optional[torch.Tensor], host: bool = False):
    """The Q tensor: its element size must match the shape's q_fp8 flag."""
    if t is not None:
        want = 1 if shape.q_fp8 else 2
        assert t.element_size() == want, "Q element size %d, shape expects %d" % (t.element_size(), want)
    return _host(t) if host else _dev(t)


def _host(t: Optional[torch.Tensor]):
    if t is not None:
        assert not t.is_cuda, "host pointer expected"
    return _ptr(t)


def _stream(stream=None) -> c_vp:
    s = torch.cuda.current_stream() if stream is None else stream
    return c_vp(s.cuda_stream)


def _check(code: int, where: str) -> None:
    if code != 0:
        raise MsaError(code, where)


def launch_count() -> int:
    return int(lib().msa_launch_count())


STAGES = ["index_scores", "topk_select", "schedule", "attn_prefill", "combine",
          "index_scores_decode", "attn_decode", "combine_decode", "index_lse"]


def profile_begin() -> None:
    _check(lib().msa_profile_begin(), "msa_profile_begin")


def profile_end():
    """-> {stage: (ms, launches)} summed since profile_begin(); synchronises the device."""
    ms = (ctypes.c_float * len(STAGES))()
    n = (c_i64 * len(STAGES))()
    _check(lib().msa_profile_end(ms, n), "msa_profile_end")
    return {STAGES[i]: (float(ms[i]), int(n[i])) for i in range(len(STAGES))}


def check_async_status() -> Tuple[int, int]:
    """(status, detail) of the device-side status word; clears it.  Synchronises."""
    detail = c_i32(0)
    code = lib().msa_check_async_status(ctypes.byref(detail))
    return int(code), int(detail.value)


# ------------------------------------------------------------------ the four stages
def msa_index_scores(shape, q_idx, k_idx, q_begin, q_count, kv_len, scores, ld_scores, stream=None):
    _check(lib().msa_index_scores(ctypes.byref(shape), _idx(shape, q_idx), _idx(shape, k_idx), c_i64(q_begin),
                                  c_i64(q_count), c_i64(kv_len), _dev(scores), c_i64(ld_scores),
                                  _stream(stream)), "msa_index_scores")


def msa_index_scores_decode(shape, q_idx, k_idx_cache, seq_offsets, seq_lens, batch, max_seq_len,
                            scores, ld_scores, stream=None):
    _check(lib().msa_index_scores_decode(ctypes.byref(shape), _idx(shape, q_idx), _idx(shape, k_idx_cache),
                                         _dev(seq_offsets), _dev(seq_lens), c_i32(batch),
                                         c_i64(max_seq_len), _dev(scores), c_i64(ld_scores),
                                         _stream(stream)), "msa_index_scores_decode")


def msa_topk_select(shape, scores, ld_scores, q_begin, q_count, kv_len, block_idx, stream=None):
    _check(lib().msa_topk_select(ctypes.byref(shape), _dev(scores), c_i64(ld_scores), c_i64(q_begin),
                                 c_i64(q_count), c_i64(kv_len), _dev(block_idx), _stream(stream)),
           "msa_topk_select")


def msa_topk_select_decode(shape, scores, ld_scores, seq_lens, batch, max_seq_len, block_idx, stream=None):
    _check(lib().msa_topk_select_decode(ctypes.byref(shape), _dev(scores), c_i64(ld_scores),
                                        _dev(seq_lens), c_i32(batch), c_i64(max_seq_len), _dev(block_idx),
                                        _stream(stream)), "msa_topk_select_decode")


def msa_index_scores_plan(shape, q_count, kv_len) -> Tuple[bool, int]:
    """(runs on the tensor cores?, index heads per CTA) for msa_index_scores on the current device."""
    tc, nh = c_i32(0), c_i32(0)
    _check(lib().msa_index_scores_plan(ctypes.byref(shape), c_i64(q_count), c_i64(kv_len), ctypes.byref(tc),
                                       ctypes.byref(nh)), "msa_index_scores_plan")
    return bool(tc.value), int(nh.value)


def msa_debug_set_wait(wait_limit_cycles: int = 0, producer_delay_cycles: int = 0) -> None:
    """Test hook: shortens the device-side bounded waits (0 = the production limit) and makes the
    copy-issuing role of the tensor-core kernels start late by the given number of SM cycles."""
    _check(lib().msa_debug_set_wait(c_i64(wait_limit_cycles), c_i64(producer_delay_cycles)), "msa_debug_set_wait")


def msa_sparse_attn_prefill_workspace_bytes(shape, q_count, kv_len) -> Tuple[int, int]:
    mn, pf = c_sz(0), c_sz(0)
    _check(lib().msa_sparse_attn_prefill_workspace_bytes(ctypes.byref(shape), c_i64(q_count),
                                                         c_i64(kv_len), ctypes.byref(mn),
                                                         ctypes.byref(pf)),
           "msa_sparse_attn_prefill_workspace_bytes")
    return int(mn.value), int(pf.value)


def msa_sparse_attn_prefill(shape, q, k, v, block_idx, q_begin, q_count, kv_len, out, lse,
                            workspace, stream=None):
    _check(lib().msa_sparse_attn_prefill(ctypes.byref(shape), _q(shape, q), _kv(shape, k), _kv(shape, v),
                                         _dev(block_idx), c_i64(q_begin), c_i64(q_count),
                                         c_i64(kv_len), _dev(out), _dev(lse), _dev(workspace),
                                         c_sz(workspace.numel() * workspace.element_size()),
                                         _stream(stream)), "msa_sparse_attn_prefill")


STATIC_SCRATCH_BYTES = 64 << 20


def msa_sparse_attn_prefill_static(shape, q, k, v, block_idx, q_begin, q_count, kv_len, out, lse,
                                   stream=None):
    """Stage 3 (prefill) for callers that may not allocate device memory.

    Same inputs and outputs as :func:`msa_sparse_attn_prefill`, but no workspace argument:
    the scratch is a fixed array of ``STATIC_SCRATCH_BYTES`` inside the library's device
    image.  Meant for hosts that cannot call ``cudaMalloc`` or ask torch for a buffer at
    that point (a plug-in inside an engine that owns all device memory, code running after
    the memory pool was frozen).  Raises ``MsaError`` (workspace) when fewer than
    ``min(q_count, 16)`` queries fit the array.  Calls that overlap on the GPU race on the
    shared array; make the first call on a device outside any stream capture.
    """
    _check(lib().msa_sparse_attn_prefill_static(ctypes.byref(shape), _dev(q), _dev(k), _dev(v),
                                                _dev(block_idx), c_i64(q_begin), c_i64(q_count),
                                                c_i64(kv_len), _dev(out), _dev(lse),
                                                _stream(stream)), "msa_sparse_attn_prefill_static")


def msa_sparse_attn_decode_workspace_bytes(shape, batch) -> int:
    mn = c_sz(0)
    _check(lib().msa_sparse_attn_decode_workspace_bytes(ctypes.byref(shape), c_i32(batch),
                                                        ctypes.byref(mn)),
           "msa_sparse_attn_decode_workspace_bytes")
    return int(mn.value)


def msa_sparse_attn_decode(shape, q, k_cache, v_cache, cache_tokens, seq_offsets, seq_lens, batch,
                           block_idx, out, lse, workspace, stream=None):
    _check(lib().msa_sparse_attn_decode(ctypes.byref(shape), _dev(q), _kv(shape, k_cache), _kv(shape, v_cache),
                                        c_i64(cache_tokens), _dev(seq_offsets), _dev(seq_lens),
                                        c_i32(batch), _dev(block_idx), _dev(out), _dev(lse),
                                        _dev(workspace),
                                        c_sz(workspace.numel() * workspace.element_size()),
                                        _stream(stream)), "msa_sparse_attn_decode")


# ------------------------------------------------------------------ whole path
def msa_prefill_forward_workspace_bytes(shape, T) -> Tuple[int, int]:
    mn, pf = c_sz(0), c_sz(0)
    _check(lib().msa_prefill_forward_workspace_bytes(ctypes.byref(shape), c_i64(T), ctypes.byref(mn),
                                                     ctypes.byref(pf)),
           "msa_prefill_forward_workspace_bytes")
    return int(mn.value), int(pf.value)


def msa_prefill_forward(shape, q, k, v, q_idx, k_idx, T, out, lse, block_idx, workspace, stream=None):
    _check(lib().msa_prefill_forward(ctypes.byref(shape), _q(shape, q), _kv(shape, k), _kv(shape, v), _idx(shape, q_idx),
                                     _idx(shape, k_idx), c_i64(T), _dev(out), _dev(lse), _dev(block_idx),
                                     _dev(workspace),
                                     c_sz(workspace.numel() * workspace.element_size()),
                                     _stream(stream)), "msa_prefill_forward")


def msa_index_topk_fused(shape, q_idx, k_idx, q_begin, q_count, kv_len, block_idx, stream=None):
    _check(lib().msa_index_topk_fused(ctypes.byref(shape), _idx(shape, q_idx), _idx(shape, k_idx), c_i64(q_begin),
                                      c_i64(q_count), c_i64(kv_len), _dev(block_idx), _stream(stream)),
           "msa_index_topk_fused")


def msa_index_lse_prefill_workspace_bytes(shape, q_count, kv_len) -> Tuple[int, int]:
    mn, pf = c_sz(0), c_sz(0)
    _check(lib().msa_index_lse_prefill_workspace_bytes(ctypes.byref(shape), c_i64(q_count), c_i64(kv_len),
                                                       ctypes.byref(mn), ctypes.byref(pf)),
           "msa_index_lse_prefill_workspace_bytes")
    return int(mn.value), int(pf.value)


def msa_index_lse_prefill(shape, q_idx, k_idx, block_idx, q_begin, q_count, kv_len, lse_idx, workspace,
                          stream=None):
    _check(lib().msa_index_lse_prefill(ctypes.byref(shape), _idx(shape, q_idx), _idx(shape, k_idx), _dev(block_idx),
                                       c_i64(q_begin), c_i64(q_count), c_i64(kv_len), _dev(lse_idx),
                                       _dev(workspace), c_sz(workspace.numel() * workspace.element_size()),
                                       _stream(stream)), "msa_index_lse_prefill")


def _cu_array(cu_seqlens):
    cu = [int(c) for c in cu_seqlens]
    return (c_i64 * len(cu))(*cu), len(cu) - 1


def msa_prefill_forward_varlen_workspace_bytes(shape, cu_seqlens) -> Tuple[int, int]:
    arr, n = _cu_array(cu_seqlens)
    mn, pf = c_sz(0), c_sz(0)
    _check(lib().msa_prefill_forward_varlen_workspace_bytes(ctypes.byref(shape), arr, c_i32(n),
                                                            ctypes.byref(mn), ctypes.byref(pf)),
           "msa_prefill_forward_varlen_workspace_bytes")
    return int(mn.value), int(pf.value)


def msa_prefill_forward_varlen(shape, q, k, v, q_idx, k_idx, cu_seqlens, out, lse, block_idx, workspace,
                               stream=None):
    arr, n = _cu_array(cu_seqlens)
    _check(lib().msa_prefill_forward_varlen(ctypes.byref(shape), _q(shape, q), _kv(shape, k), _kv(shape, v), _idx(shape, q_idx),
                                            _idx(shape, k_idx), arr, c_i32(n), _dev(out), _dev(lse),
                                            _dev(block_idx), _dev(workspace),
                                            c_sz(workspace.numel() * workspace.element_size()),
                                            _stream(stream)), "msa_prefill_forward_varlen")


def msa_prefill_forward_host_workspace_bytes(shape, T) -> Tuple[int, int]:
    mn, pf = c_sz(0), c_sz(0)
    _check(lib().msa_prefill_forward_host_workspace_bytes(ctypes.byref(shape), c_i64(T),
                                                          ctypes.byref(mn), ctypes.byref(pf)),
           "msa_prefill_forward_host_workspace_bytes")
    return int(mn.value), int(pf.value)


def msa_prefill_forward_host(shape, q, k, v, q_idx, k_idx, T, out, lse, block_idx, workspace,
                             stream=None):
    """q..k_idx, out, lse, block_idx are HOST tensors (pinned for full copy rate)."""
    _check(lib().msa_prefill_forward_host(ctypes.byref(shape), _q(shape, q, True), _host(k), _host(v),
                                          _idx(shape, q_idx, True), _idx(shape, k_idx, True), c_i64(T), _host(out),
                                          _host(lse), _host(block_idx), _dev(workspace),
                                          c_sz(workspace.numel() * workspace.element_size()),
                                          _stream(stream)), "msa_prefill_forward_host")


def msa_decode_forward(shape, q, q_idx, k_cache, v_cache, k_idx_cache, cache_tokens, seq_offsets,
                       seq_lens, batch, max_seq_len, scores, ld_scores, block_idx, out, lse,
                       workspace, stream=None):
    _check(lib().msa_decode_forward(ctypes.byref(shape), _dev(q), _idx(shape, q_idx), _kv(shape, k_cache),
                                    _kv(shape, v_cache), _idx(shape, k_idx_cache), c_i64(cache_tokens),
                                    _dev(seq_offsets), _dev(seq_lens), c_i32(batch),
                                    c_i64(max_seq_len), _dev(scores), c_i64(ld_scores),
                                    _dev(block_idx), _dev(out), _dev(lse), _dev(workspace),
                                    c_sz(workspace.numel() * workspace.element_size()),
                                    _stream(stream)), "msa_decode_forward")


def msa_decode_forward_host(shape, q_host, q_idx_host, q_dev, q_idx_dev, k_cache, v_cache,
                            k_idx_cache, cache_tokens, seq_offsets, seq_lens, batch, max_seq_len,
                            scores, ld_scores, block_idx, out_dev, out_host, workspace, stream=None):
    _check(lib().msa_decode_forward_host(ctypes.byref(shape), _host(q_host), _idx(shape, q_idx_host, True),
                                         _dev(q_dev), _idx(shape, q_idx_dev), _kv(shape, k_cache), _kv(shape, v_cache),
                                         _idx(shape, k_idx_cache), c_i64(cache_tokens), _dev(seq_offsets),
                                         _dev(seq_lens), c_i32(batch), c_i64(max_seq_len),
                                         _dev(scores), c_i64(ld_scores), _dev(block_idx),
                                         _dev(out_dev), _host(out_host), _dev(workspace),
                                         c_sz(workspace.numel() * workspace.element_size()),
                                         _stream(stream)), "msa_decode_forward_host")


# ------------------------------------------------------------------ around the path
# (These run in a decode step, where a call's own cost counts: checks format their message only when they fail, and
# the argument types are declared once.)
_F32 = ctypes.c_float
_ARGTYPES = {
    "msa_qk_norm_rope": [c_vp, c_vp, c_i64, c_i32, c_vp, c_vp, c_i64, c_i32, c_vp, c_i32, c_i32, _F32, c_vp, c_i64, c_vp, c_vp,
                         c_vp],
    "msa_qk_norm_rope_backward": [c_vp, c_vp, c_i64, c_vp, c_i64, c_vp, c_i64, c_i32, c_vp, c_vp, c_i64, c_i32, c_vp, c_i32,
                                  c_i32, _F32, c_vp, c_i64, c_vp, c_vp, c_vp, c_vp, c_vp, c_sz, c_vp],
    "msa_paged_attn_workspace_bytes": [c_vp, c_i32, c_vp],
    "msa_paged_attn": [c_vp, c_vp, c_i32, c_i64, _F32, c_vp, c_vp, c_vp, c_sz, c_vp],
    "msa_paged_append": [c_vp, c_vp, c_vp, c_i64, c_i32, c_vp, c_vp, c_i64, c_vp, c_vp, c_i64, c_i32, _F32, c_i64, c_vp, c_vp],
    "msa_paged_weights_workspace_bytes": [c_vp, c_i32, c_vp],
    "msa_paged_weights": [c_vp, c_vp, c_i32, c_vp, c_i64, _F32, _F32, c_vp, c_vp, c_sz, c_vp],
    "msa_paged_keep": [c_vp, c_vp, c_i32, c_i32, c_i32, c_vp, c_vp, c_vp],
    "msa_paged_compact": [c_vp, c_vp, c_i32, c_vp, c_vp],
    "msa_sample": [c_vp, c_vp, c_i32, c_i64, c_i64, c_i32, c_vp, c_vp, c_vp, c_vp],
}
_fns = {}
_POOL_TYPES = {torch.bfloat16: 0, torch.float8_e4m3fn: 1}  # msa_paged_cache_t.fp8


def _fn(name: str):
    fn = _fns.get(name)
    if fn is None:
        fn = getattr(lib(), name)
        fn.argtypes = _ARGTYPES[name]
        _fns[name] = fn
    return fn


def _launch(index: int, name: str, *args, stream=None) -> None:
    """Calls the library with the tensors' device current (whatever the caller's is), on `stream` or that device's
    current stream."""
    raw = torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream
    if index == torch.cuda.current_device():
        code = _fn(name)(*args, raw)
    else:
        with torch.cuda.device(index):
            code = _fn(name)(*args, raw)
    if code != 0:
        raise MsaError(code, name)


def _heads(t: torch.Tensor, what: str, head_dim: int, rows: int, index: int, dense: bool = False) -> int:
    """A bf16 tensor [rows, heads, head_dim] whose heads are dense; returns its row stride."""
    shape = t.shape
    if t.dtype != torch.bfloat16 or t.get_device() != index:
        raise ValueError("%s must be bf16 on cuda:%d, got %s on %s" % (what, index, t.dtype, t.device))
    if len(shape) != 3 or shape[0] != rows or shape[2] != head_dim:
        raise ValueError("%s must be [%d, heads, %d], got %s" % (what, rows, head_dim, tuple(shape)))
    s, width = t.stride(), shape[1] * head_dim
    # (strides of dimensions with fewer than two entries say nothing)
    if (head_dim > 1 and s[2] != 1) or (shape[1] > 1 and s[1] != head_dim):
        raise ValueError("the last two dimensions of %s must be dense, got strides %s" % (what, s))
    if rows < 2:
        return width
    if dense and s[0] != width:
        raise ValueError("%s must be contiguous, got strides %s" % (what, s))
    return s[0]


def _output(t: Optional[torch.Tensor], other: torch.Tensor, what: str, head_dim: int, rows: int, index: int, stream) -> torch.Tensor:
    """An output of another's shape: dense bf16, made here if there is none."""
    if t is None:
        if stream is None:
            return torch.empty_like(other, memory_format=torch.contiguous_format)
        # Memory of the stream that writes it: a block of the current stream may still be in use by work queued there, or
        # be given to such work while the call runs.  The current stream is where the caller will read it.
        current = torch.cuda.current_stream(index)
        with torch.cuda.stream(stream):
            t = torch.empty_like(other, memory_format=torch.contiguous_format)
        t.record_stream(current)
        return t
    if t.shape != other.shape:
        raise ValueError("%s must be %s, got %s" % (what, tuple(other.shape), tuple(t.shape)))
    _heads(t, what, head_dim, rows, index, dense=True)
    return t


def _weights(head_dim: int, index: int, *weights) -> int:
    """Checks the weights of the norms (None: no norm); 1 if they are fp32, 0 if bf16."""
    kind = None
    for w in weights:
        if w is None:
            continue
        if (w.dtype not in (torch.bfloat16, torch.float32) or kind not in (None, w.dtype) or w.shape != (head_dim,) or
                not w.is_contiguous() or w.get_device() != index):
            raise ValueError("norm weights must be contiguous vectors of %d values, all bf16 or all fp32, on cuda:%d"
                             % (head_dim, index))
        kind = w.dtype
    return 1 if kind == torch.float32 else 0


def _rope(freqs, interleaved, mscale, index: int):
    if freqs is None:
        return None
    if freqs.dtype != torch.float64 or freqs.dim() != 1 or not freqs.is_contiguous() or freqs.get_device() != index:
        raise ValueError("frequencies must be a contiguous fp64 vector on cuda:%d" % index)
    return MsaRope(freqs.data_ptr(), 2 * freqs.shape[0], 1 if interleaved else 0, mscale)


def _positions(positions, rows: int, index: int):
    if positions is None:
        return None
    if (positions.dtype != torch.int64 or positions.shape != (rows,) or not positions.is_contiguous() or
            positions.get_device() != index):
        raise ValueError("positions must be a contiguous int64 vector, one for each of %d rows, on cuda:%d" % (rows, index))
    return positions.data_ptr()


def _device_of(t: Optional[torch.Tensor], what: str) -> int:
    if t is None or not t.is_cuda:
        raise ValueError("%s must be a tensor on a CUDA device" % what)
    return t.get_device()


def _at(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _ref(s):
    return None if s is None else ctypes.byref(s)


def msa_qk_norm_rope(freqs, interleaved, mscale, q, q_weight, k, k_weight, eps, positions, q_out, k_out, stream=None):
    """q, k: bf16 [rows, heads, d], rows may be strided; either may be None.  freqs None: no rotation.
    -> (q_out, k_out); outputs that are not given are made."""
    x = k if q is None else q
    index = _device_of(x, "q or k")
    rows, d = x.shape[0], x.shape[-1]
    qs = ks = hq = hk = 0
    if q is not None:
        qs, hq = _heads(q, "q", d, rows, index), q.shape[1]
        q_out = _output(q_out, q, "q_out", d, rows, index, stream)
    if k is not None:
        ks, hk = _heads(k, "k", d, rows, index), k.shape[1]
        k_out = _output(k_out, k, "k_out", d, rows, index, stream)
    w32 = _weights(d, index, q_weight, k_weight)
    rope = _rope(freqs, interleaved, mscale, index)
    _launch(index, "msa_qk_norm_rope", _ref(rope), _at(q), qs, hq, _at(q_weight), _at(k), ks, hk, _at(k_weight), d, w32, eps,
            _positions(positions, rows, index), rows, _at(q_out), _at(k_out), stream=stream)
    return q_out, k_out


def msa_norm_rope_plan(head_dim: int, n_q_heads: int, n_k_heads: int, n_v_heads: int, n_tokens: int) -> Tuple[int, int, int, int]:
    """(tokens of a tile, CTAs along the tokens, CTAs along a token's heads, dynamic shared memory) of a rotation or an
    append on the current device."""
    out = [c_i32(0) for _ in range(4)]
    _check(lib().msa_norm_rope_plan(c_i32(head_dim), c_i32(n_q_heads), c_i32(n_k_heads), c_i32(n_v_heads), c_i64(n_tokens),
                                    *[ctypes.byref(o) for o in out]), "msa_norm_rope_plan")
    return tuple(int(o.value) for o in out)


def msa_qk_norm_rope_backward_workspace_bytes(head_dim: int, n_tokens: int) -> int:
    mn = c_sz(0)
    _check(lib().msa_qk_norm_rope_backward_workspace_bytes(c_i32(head_dim), c_i64(n_tokens), ctypes.byref(mn)),
           "msa_qk_norm_rope_backward_workspace_bytes")
    return int(mn.value)


def _workspace(ws: Optional[torch.Tensor], index: int) -> int:
    """Checks a workspace and returns its bytes."""
    if ws is None:
        return 0
    if not ws.is_contiguous() or ws.get_device() != index:
        raise ValueError("the workspace must be contiguous on cuda:%d" % index)
    return ws.numel() * ws.element_size()


def msa_qk_norm_rope_backward(freqs, interleaved, mscale, dq_out, dk_out, q, q_weight, k, k_weight, eps, positions, dq,
                              dk, dq_weight, dk_weight, workspace, stream=None):
    """q / k are needed where there is a weight (else None is fine); dq, dk bf16 dense, weight gradients fp32 [d].
    -> (dq, dk); those that are not given are made."""
    x = dk_out if dq_out is None else dq_out
    index = _device_of(x, "dq_out or dk_out")
    rows, d = x.shape[0], x.shape[-1]
    at, grads = [], []
    for n, dy, t, w, dx, dw in (("q", dq_out, q, q_weight, dq, dq_weight), ("k", dk_out, k, k_weight, dk, dk_weight)):
        if dy is None:
            at.append((0, 0, 0))
            grads.append(None)
            continue
        ys, ts = _heads(dy, "the gradient of %s_out" % n, d, rows, index), 0
        if t is not None:
            ts = _heads(t, n, d, rows, index)
            if t.shape != dy.shape:
                raise ValueError("%s must be %s, got %s" % (n, tuple(dy.shape), tuple(t.shape)))
        elif w is not None:
            raise ValueError("%s is needed for the gradients of its norm" % n)
        dx = _output(dx, dy, "the gradient of " + n, d, rows, index, stream)
        if dw is not None and (dw.dtype != torch.float32 or dw.shape != (d,) or not dw.is_contiguous() or dw.get_device() != index):
            raise ValueError("the gradient of %s_weight must be a contiguous fp32 vector of %d values on cuda:%d" % (n, d, index))
        at.append((ys, ts, dy.shape[1]))
        grads.append(dx)
    w32 = _weights(d, index, q_weight, k_weight)
    rope = _rope(freqs, interleaved, mscale, index)
    _launch(index, "msa_qk_norm_rope_backward", _ref(rope), _at(dq_out), at[0][0], _at(dk_out), at[1][0], _at(q), at[0][1],
            at[0][2], _at(q_weight), _at(k), at[1][1], at[1][2], _at(k_weight), d, w32, eps, _positions(positions, rows, index),
            rows, _at(grads[0]), _at(grads[1]), _at(dq_weight), _at(dk_weight), _at(workspace), _workspace(workspace, index),
            stream=stream)
    return grads[0], grads[1]


def _paged(k_pool, v_pool, page_table, kv_lens, cu_q):
    """The cache structure of checked tensors."""
    index = _device_of(k_pool, "the key pool")
    kind, shape = k_pool.dtype, k_pool.shape
    if len(shape) != 4 or kind not in _POOL_TYPES or not k_pool.is_contiguous():
        raise ValueError("the key pool must be a contiguous [pages, page size, KV heads, head_dim] tensor of bf16 or "
                         "float8_e4m3fn, got %s %s" % (kind, tuple(shape)))
    if v_pool is not None and (v_pool.shape != shape or v_pool.dtype != kind or not v_pool.is_contiguous() or
                               v_pool.get_device() != index):
        raise ValueError("the value pool must be like the key pool")
    table, lens = page_table.shape, kv_lens.shape
    if len(table) != 2 or len(lens) != 1 or table[0] != lens[0] or cu_q.shape != (lens[0] + 1,):
        raise ValueError("page_table [batch, pages], kv_lens [batch] and cu_q [batch + 1] must agree")
    for t in (page_table, kv_lens, cu_q):
        if t.dtype != torch.int32 or not t.is_contiguous() or t.get_device() != index:
            raise ValueError("page_table, kv_lens and cu_q must be contiguous int32 on cuda:%d" % index)
    return index, MsaPagedCache(k_pool.data_ptr(), _at(v_pool), page_table.data_ptr(), kv_lens.data_ptr(), cu_q.data_ptr(), lens[0],
                                table[1], *shape, _POOL_TYPES[kind])


def msa_paged_append(k_pool, v_pool, page_table, kv_lens, cu_q, freqs, interleaved, mscale, q, q_weight, k, k_weight, v,
                     eps, q_out, stream=None):
    """k, v (and q): bf16 [rows, heads, d], rows may be strided; q None: no queries; v None: a cache without values.
    -> q_out, made if it is not given."""
    index, cache = _paged(k_pool, v_pool, page_table, kv_lens, cu_q)
    d, rows = cache.head_dim, k.shape[0]
    vs = qs = hq = 0
    ks = _heads(k, "k", d, rows, index)
    if (v is None) != (v_pool is None):
        raise ValueError("values and a value pool come together")
    if v is not None:
        vs = _heads(v, "v", d, rows, index)
    if k.shape[1] != cache.n_kv_heads or (v is not None and v.shape[1] != cache.n_kv_heads):
        raise ValueError("k and v must have the cache's %d heads" % cache.n_kv_heads)
    if q is not None:
        qs, hq = _heads(q, "q", d, rows, index), q.shape[1]
        q_out = _output(q_out, q, "q_out", d, rows, index, stream)
    w32 = _weights(d, index, q_weight, k_weight)
    rope = _rope(freqs, interleaved, mscale, index)
    _launch(index, "msa_paged_append", ctypes.byref(cache), _ref(rope), _at(q), qs, hq, _at(q_weight), _at(k), ks, _at(k_weight),
            _at(v), vs, w32, eps, rows, _at(q_out), stream=stream)
    return q_out


def msa_paged_attn_workspace_bytes(k_pool, n_q_heads: int) -> int:
    pages, size, heads, d = k_pool.shape
    cache = MsaPagedCache(n_pages=pages, page_size=size, n_kv_heads=heads, head_dim=d, fp8=0 if k_pool.dtype == torch.bfloat16 else 1)
    mn = c_sz(0)
    code = _fn("msa_paged_attn_workspace_bytes")(ctypes.byref(cache), n_q_heads, ctypes.byref(mn))
    if code != 0:
        raise MsaError(code, "msa_paged_attn_workspace_bytes")
    return mn.value


def msa_paged_attn(k_pool, v_pool, page_table, kv_lens, cu_q, q, softmax_scale, out, lse, workspace, stream=None, max_new=0):
    """q, out: bf16 [rows, heads, d] dense; lse fp32 [rows, heads] or None; max_new: the most new tokens of a sequence, 0 if
    not known.  -> out, made if it is not given."""
    index, cache = _paged(k_pool, v_pool, page_table, kv_lens, cu_q)
    cache.max_new = max_new
    d, rows = cache.head_dim, q.shape[0]
    if v_pool is None:
        raise ValueError("attention needs a value pool")
    _heads(q, "q", d, rows, index, dense=True)
    out = _output(out, q, "out", d, rows, index, stream)
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous() or
                            lse.get_device() != index):
        raise ValueError("lse must be contiguous fp32 %s on cuda:%d" % (tuple(q.shape[:2]), index))
    _launch(index, "msa_paged_attn", ctypes.byref(cache), q.data_ptr(), q.shape[1], rows, softmax_scale, out.data_ptr(), _at(lse),
            _at(workspace), _workspace(workspace, index), stream=stream)
    return out


def _made(t: Optional[torch.Tensor], near: torch.Tensor, shape, dtype, what: str, index: int, stream) -> torch.Tensor:
    """A dense output of a given shape and type, made here (beside `near`, on the stream that writes it) if there is none."""
    if t is None:
        if stream is None:
            return near.new_empty(shape, dtype=dtype)
        current = torch.cuda.current_stream(index)
        with torch.cuda.stream(stream):
            t = near.new_empty(shape, dtype=dtype)
        t.record_stream(current)
        return t
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or t.get_device() != index:
        raise ValueError("%s must be contiguous %s %s on cuda:%d, got %s %s" % (what, dtype, tuple(shape), index, t.dtype, tuple(t.shape)))
    return t


def _weight_pool(t: torch.Tensor, cache: MsaPagedCache, index: int) -> int:
    want = (cache.n_pages, cache.n_kv_heads, cache.page_size)
    if t.dtype != torch.float32 or tuple(t.shape) != want or not t.is_contiguous() or t.get_device() != index:
        raise ValueError("the weights must be contiguous fp32 [pages, KV heads, page size] = %s on cuda:%d, got %s %s"
                         % (want, index, t.dtype, tuple(t.shape)))
    return t.data_ptr()


def _int32(v: int) -> int:
    """The nearest 32-bit number, for whole numbers that only bound something (ctypes would take the lowest 32 bits)."""
    return v if -0x80000000 <= v <= 0x7FFFFFFF else (0x7FFFFFFF if v > 0 else -0x80000000)


def msa_paged_weights_workspace_bytes(k_pool, n_q_heads: int) -> int:
    pages, size, heads, d = k_pool.shape
    cache = MsaPagedCache(n_pages=pages, page_size=size, n_kv_heads=heads, head_dim=d, fp8=0 if k_pool.dtype == torch.bfloat16 else 1)
    mn = c_sz(0)
    _check(_fn("msa_paged_weights_workspace_bytes")(ctypes.byref(cache), n_q_heads, ctypes.byref(mn)), "msa_paged_weights_workspace_bytes")
    return mn.value


def msa_paged_weights(k_pool, page_table, kv_lens, cu_q, q, lse, softmax_scale, decay, weights, workspace, stream=None, max_new=0):
    """q: bf16 [rows, heads, d] dense; lse: fp32 [rows, heads]; weights: fp32 [pages, KV heads, page size], updated in place."""
    index, cache = _paged(k_pool, None, page_table, kv_lens, cu_q)
    cache.max_new = max_new
    d, rows = cache.head_dim, q.shape[0]
    _heads(q, "q", d, rows, index, dense=True)
    if lse.dtype != torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous() or lse.get_device() != index:
        raise ValueError("lse must be contiguous fp32 %s on cuda:%d" % (tuple(q.shape[:2]), index))
    _launch(index, "msa_paged_weights", ctypes.byref(cache), q.data_ptr(), q.shape[1], lse.data_ptr(), rows, softmax_scale, decay,
            _weight_pool(weights, cache, index), _at(workspace), _workspace(workspace, index), stream=stream)


def msa_paged_keep(k_pool, page_table, kv_lens, cu_q, weights, budget, sinks, recent, keep=None, new_lens=None, stream=None):
    """-> (keep int32 [batch, KV heads, budget], new_lens int32 [batch]); those that are not given are made."""
    index, cache = _paged(k_pool, None, page_table, kv_lens, cu_q)
    at = _weight_pool(weights, cache, index)
    sinks, recent = _int32(sinks), _int32(recent)
    keep = _made(keep, weights, (cache.batch, cache.n_kv_heads, max(budget, 0)), torch.int32, "keep", index, stream)
    new_lens = _made(new_lens, weights, (cache.batch,), torch.int32, "new_lens", index, stream)
    _launch(index, "msa_paged_keep", ctypes.byref(cache), at, _int32(budget), sinks, recent, keep.data_ptr(), new_lens.data_ptr(), stream=stream)
    return keep, new_lens


def msa_paged_compact(k_pool, v_pool, page_table, kv_lens, cu_q, keep, weights, stream=None):
    """keep: int32 [batch, KV heads, width]; weights: fp32 [pages, KV heads, page size] or None.  Pools and weights change in place."""
    index, cache = _paged(k_pool, v_pool, page_table, kv_lens, cu_q)
    if (keep.dtype != torch.int32 or keep.dim() != 3 or tuple(keep.shape[:2]) != (cache.batch, cache.n_kv_heads) or
            not keep.is_contiguous() or keep.get_device() != index):
        raise ValueError("keep must be contiguous int32 [%d, %d, width] on cuda:%d, got %s %s"
                         % (cache.batch, cache.n_kv_heads, index, keep.dtype, tuple(keep.shape)))
    at = None if weights is None else _weight_pool(weights, cache, index)
    _launch(index, "msa_paged_compact", ctypes.byref(cache), keep.data_ptr(), keep.shape[2], at, stream=stream)


_LOGIT_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


def _setting(v, dtype, rows: int, index: int, what: str):
    """(number, device pointer) of a setting: a number for all rows or a tensor of one for every row."""
    if not isinstance(v, torch.Tensor):
        return (_int32(v) if dtype == torch.int32 else v), None
    if v.dtype != dtype or v.shape != (rows,) or not v.is_contiguous() or v.get_device() != index:
        raise ValueError("%s must be a number or a contiguous %s vector, one for each of %d rows, on cuda:%d" % (what, dtype, rows, index))
    return 0, v.data_ptr()


def msa_sample(logits, uniform, temperature, top_k, top_p, min_p, token=None, logprob=None, stream=None):
    """logits: [rows, vocabulary] of bf16, fp16 or fp32, rows may be strided; uniform: fp32 [rows]; settings: numbers, or fp32
    (top_k: int32) vectors.  -> (token int64 [rows], logprob fp32 [rows]); those that are not given are made."""
    index = _device_of(logits, "the logits")
    kind, shape, strides = _LOGIT_TYPES.get(logits.dtype), logits.shape, logits.stride()
    if kind is None or len(shape) != 2 or shape[1] < 1 or (shape[1] > 1 and strides[1] != 1):
        raise ValueError("the logits must be bf16, fp16 or fp32 [rows, vocabulary] with dense rows, got %s %s, strides %s"
                         % (logits.dtype, tuple(shape), strides))
    rows, vocab = shape
    stride = strides[0] if rows > 1 else vocab
    if stride < vocab:
        raise ValueError("rows of the logits must not overlap: %d values every %d" % (vocab, stride))
    if uniform.dtype != torch.float32 or uniform.shape != (rows,) or not uniform.is_contiguous() or uniform.get_device() != index:
        raise ValueError("the random numbers must be a contiguous fp32 vector, one for each of %d rows, on cuda:%d" % (rows, index))
    f32 = torch.float32
    (t, ts), (k, ks) = _setting(temperature, f32, rows, index, "temperature"), _setting(top_k, torch.int32, rows, index, "top_k")
    (p, ps), (m, ms) = _setting(top_p, f32, rows, index, "top_p"), _setting(min_p, f32, rows, index, "min_p")
    token = _made(token, uniform, (rows,), torch.int64, "token", index, stream)
    logprob = _made(logprob, uniform, (rows,), f32, "logprob", index, stream)
    _launch(index, "msa_sample", ctypes.byref(MsaSampling(t, k, p, m, ts, ks, ps, ms)), logits.data_ptr(), kind,
            stride, rows, vocab, uniform.data_ptr(), token.data_ptr(), logprob.data_ptr(), stream=stream)
    return token, logprob


# ------------------------------------------------------------------ allocation helpers
def score_ld(kv_len: int, block_size: int) -> int:
    """Row pitch (in floats) for a scores buffer: B rounded up to a multiple of 4."""
    return (-(-kv_len // block_size) + 3) // 4 * 4


def alloc_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
