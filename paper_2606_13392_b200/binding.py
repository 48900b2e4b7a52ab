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
    "msa_qk_norm_rope", "msa_qk_norm_rope_backward", "msa_qk_norm_rope_backward_workspace_bytes", "msa_paged_append",
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
                ("head_dim", c_i32), ("fp8", c_i32)]


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
def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _launch(device: torch.device, name: str, *args, stream=None) -> None:
    """Calls the library with `device` current (the tensors' own, whatever the caller's is) on its current stream."""
    fn = getattr(lib(), name)
    if device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            _check(fn(*args, _stream(stream)), name)
    else:
        _check(fn(*args, _stream(stream)), name)


def _heads(t: torch.Tensor, what: str, head_dim: int, rows: int, device: torch.device, dense: bool = False) -> int:
    """A bf16 tensor [rows, heads, head_dim] whose heads are dense; returns its row stride."""
    _need(t.dtype == torch.bfloat16 and t.device == device, "%s must be bf16 on %s" % (what, device))
    _need(t.dim() == 3 and t.shape[0] == rows and t.shape[2] == head_dim,
          "%s must be [%d, heads, %d], got %s" % (what, rows, head_dim, tuple(t.shape)))
    s, width = t.stride(), t.shape[1] * head_dim
    # (strides of dimensions with fewer than two entries say nothing)
    _need((t.shape[2] < 2 or s[2] == 1) and (t.shape[1] < 2 or s[1] == head_dim),
          "the last two dimensions of %s must be dense" % what)
    if rows < 2:
        return width
    _need(s[0] == width or not dense, "%s must be contiguous" % what)
    return s[0]


def _weights(head_dim: int, device: torch.device, *weights) -> int:
    """Checks the weights of the norms (None: no norm); 1 if they are fp32, 0 if bf16."""
    kinds = {w.dtype for w in weights if w is not None}
    _need(len(kinds) < 2 and kinds <= {torch.bfloat16, torch.float32}, "norm weights must be all bf16 or all fp32")
    for w in weights:
        _need(w is None or (w.shape == (head_dim,) and w.is_contiguous() and w.device == device),
              "norm weights must be contiguous vectors of head_dim values on %s" % device)
    return 1 if torch.float32 in kinds else 0


def _rope(freqs, interleaved, mscale, device: torch.device):
    if freqs is None:
        return None
    _need(freqs.dtype == torch.float64 and freqs.dim() == 1 and freqs.is_contiguous() and freqs.device == device,
          "frequencies must be a contiguous fp64 vector on %s" % device)
    return MsaRope(freqs.data_ptr(), 2 * freqs.shape[0], 1 if interleaved else 0, mscale)


def _positions(positions, rows: int, device: torch.device):
    if positions is not None:
        _need(positions.dtype == torch.int64 and positions.shape == (rows,) and positions.is_contiguous() and
              positions.device == device, "positions must be a contiguous int64 vector, one for each row, on %s" % device)
    return c_vp(None if positions is None else positions.data_ptr())


def _at(t: Optional[torch.Tensor]) -> c_vp:
    return c_vp(None if t is None else t.data_ptr())


def _ref(s):
    return None if s is None else ctypes.byref(s)


def msa_qk_norm_rope(freqs, interleaved, mscale, q, q_weight, k, k_weight, eps, positions, q_out, k_out, stream=None):
    """q, k: bf16 [rows, heads, d], rows may be strided; either may be None.  freqs None: no rotation."""
    x = q if q is not None else k
    _need(x is not None and x.is_cuda, "a tensor on a CUDA device is needed")
    dev, rows, d = x.device, x.shape[0], x.shape[2] if x.dim() == 3 else 0
    qs = ks = 0
    if q is not None:
        qs = _heads(q, "q", d, rows, dev)
        _need(q_out.shape == q.shape, "q_out must have q's shape")
        _heads(q_out, "q_out", d, rows, dev, dense=True)
    if k is not None:
        ks = _heads(k, "k", d, rows, dev)
        _need(k_out.shape == k.shape, "k_out must have k's shape")
        _heads(k_out, "k_out", d, rows, dev, dense=True)
    w32 = _weights(d, dev, q_weight, k_weight)
    rope = _rope(freqs, interleaved, mscale, dev)
    _launch(dev, "msa_qk_norm_rope", _ref(rope), _at(q), c_i64(qs), c_i32(q.shape[1] if q is not None else 0), _at(q_weight),
            _at(k), c_i64(ks), c_i32(k.shape[1] if k is not None else 0), _at(k_weight), c_i32(d), c_i32(w32),
            ctypes.c_float(eps), _positions(positions, rows, dev), c_i64(rows), _at(q_out), _at(k_out), stream=stream)


def msa_qk_norm_rope_backward_workspace_bytes(head_dim: int, n_tokens: int) -> int:
    mn = c_sz(0)
    _check(lib().msa_qk_norm_rope_backward_workspace_bytes(c_i32(head_dim), c_i64(n_tokens), ctypes.byref(mn)),
           "msa_qk_norm_rope_backward_workspace_bytes")
    return int(mn.value)


def msa_qk_norm_rope_backward(freqs, interleaved, mscale, dq_out, dk_out, q, q_weight, k, k_weight, eps, positions, dq,
                              dk, dq_weight, dk_weight, workspace, stream=None):
    """q / k are needed where there is a weight (else None is fine); dq, dk bf16 dense, weight gradients fp32 [d]."""
    x = dq_out if dq_out is not None else dk_out
    _need(x is not None and x.is_cuda, "a tensor on a CUDA device is needed")
    dev, rows, d = x.device, x.shape[0], x.shape[2] if x.dim() == 3 else 0
    strides = []
    for n, dy, t, w, dx, dw in (("q", dq_out, q, q_weight, dq, dq_weight), ("k", dk_out, k, k_weight, dk, dk_weight)):
        if dy is None:
            strides += [0, 0]
            continue
        strides.append(_heads(dy, "d%s_out" % n, d, rows, dev))
        _need(w is None or t is not None, "%s is needed for the gradients of its norm" % n)
        strides.append(0 if t is None else _heads(t, n, d, rows, dev))
        _need((t is None or t.shape == dy.shape) and dx.shape == dy.shape, "%s and its gradients must have one shape" % n)
        _heads(dx, "d%s" % n, d, rows, dev, dense=True)
        _need(dw is None or (dw.dtype == torch.float32 and dw.shape == (d,) and dw.is_contiguous() and dw.device == dev),
              "d%s_weight must be a contiguous fp32 vector of head_dim values on %s" % (n, dev))
    w32 = _weights(d, dev, q_weight, k_weight)
    rope = _rope(freqs, interleaved, mscale, dev)
    _need(workspace is None or (workspace.is_contiguous() and workspace.device == dev), "workspace must be on %s" % dev)
    _launch(dev, "msa_qk_norm_rope_backward", _ref(rope), _at(dq_out), c_i64(strides[0]), _at(dk_out), c_i64(strides[2]), _at(q),
            c_i64(strides[1]), c_i32(dq_out.shape[1] if dq_out is not None else 0), _at(q_weight), _at(k), c_i64(strides[3]),
            c_i32(dk_out.shape[1] if dk_out is not None else 0), _at(k_weight), c_i32(d), c_i32(w32), ctypes.c_float(eps),
            _positions(positions, rows, dev), c_i64(rows), _at(dq), _at(dk), _at(dq_weight), _at(dk_weight), _at(workspace),
            c_sz(0 if workspace is None else workspace.numel() * workspace.element_size()), stream=stream)


def _paged(k_pool, v_pool, page_table, kv_lens, cu_q):
    """The cache structure of checked tensors."""
    _need(k_pool.is_cuda and k_pool.dim() == 4 and k_pool.is_contiguous() and
          k_pool.dtype in (torch.bfloat16, torch.float8_e4m3fn),
          "the key pool must be a contiguous [pages, page size, KV heads, head_dim] tensor of bf16 or float8_e4m3fn on a CUDA device")
    dev = k_pool.device
    _need(v_pool is None or (v_pool.shape == k_pool.shape and v_pool.dtype == k_pool.dtype and v_pool.is_contiguous() and
                             v_pool.device == dev), "the value pool must be like the key pool")
    _need(page_table.dim() == 2 and kv_lens.dim() == 1 and cu_q.dim() == 1 and kv_lens.shape[0] == page_table.shape[0] and
          cu_q.shape[0] == kv_lens.shape[0] + 1, "page_table [batch, pages], kv_lens [batch] and cu_q [batch + 1] must agree")
    for n, t in (("page_table", page_table), ("kv_lens", kv_lens), ("cu_q", cu_q)):
        _need(t.dtype == torch.int32 and t.is_contiguous() and t.device == dev, "%s must be contiguous int32 on %s" % (n, dev))
    pages, size, heads, d = k_pool.shape
    return MsaPagedCache(k_pool.data_ptr(), 0 if v_pool is None else v_pool.data_ptr(), page_table.data_ptr(),
                         kv_lens.data_ptr(), cu_q.data_ptr(), kv_lens.shape[0], page_table.shape[1], pages, size, heads, d,
                         1 if k_pool.dtype == torch.float8_e4m3fn else 0)


def msa_paged_append(k_pool, v_pool, page_table, kv_lens, cu_q, freqs, interleaved, mscale, q, q_weight, k, k_weight, v,
                     eps, q_out, stream=None):
    """k, v (and q): bf16 [rows, heads, d], rows may be strided; q None: no queries; v None: a cache without values."""
    cache = _paged(k_pool, v_pool, page_table, kv_lens, cu_q)
    dev, d, rows = k_pool.device, k_pool.shape[3], k.shape[0]
    ks = _heads(k, "k", d, rows, dev)
    _need(k.shape[1] == cache.n_kv_heads, "k must have the cache's heads")
    vs = qs = 0
    _need((v is None) == (v_pool is None), "values and a value pool come together")
    if v is not None:
        vs = _heads(v, "v", d, rows, dev)
        _need(v.shape[1] == cache.n_kv_heads, "v must have the cache's heads")
    if q is not None:
        qs = _heads(q, "q", d, rows, dev)
        _need(q_out.shape == q.shape, "q_out must have q's shape")
        _heads(q_out, "q_out", d, rows, dev, dense=True)
    w32 = _weights(d, dev, q_weight, k_weight)
    rope = _rope(freqs, interleaved, mscale, dev)
    _launch(dev, "msa_paged_append", ctypes.byref(cache), _ref(rope), _at(q), c_i64(qs), c_i32(q.shape[1] if q is not None else 0),
            _at(q_weight), _at(k), c_i64(ks), _at(k_weight), _at(v), c_i64(vs), c_i32(w32), ctypes.c_float(eps), c_i64(rows),
            _at(q_out), stream=stream)


# ------------------------------------------------------------------ allocation helpers
def score_ld(kv_len: int, block_size: int) -> int:
    """Row pitch (in floats) for a scores buffer: B rounded up to a multiple of 4."""
    return (-(-kv_len // block_size) + 3) // 4 * 4


def alloc_workspace(nbytes: int, device="cuda") -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
