"""Convenience layer over the binding: allocates outputs/workspaces with torch and calls the
C ABI.  No arithmetic happens here (but for the table of frequencies of rope_frequencies)."""

from __future__ import annotations

import math
from typing import Dict, NamedTuple, Optional

import torch

from . import binding as B
from .inputs import MSAConfig


def prefill_forward(cfg: MSAConfig, x: Dict[str, torch.Tensor], workspace: Optional[torch.Tensor] = None,
                    want_lse: bool = True, workspace_bytes: Optional[int] = None):
    """Algorithm 1 lines 3-5 on device tensors q,k,v,q_idx,k_idx -> (out, lse, block_idx)."""
    shape = B.shape_of(cfg)
    T = x["q"].shape[0]
    dev = x["q"].device
    out = torch.empty(x["q"].shape, dtype=torch.bfloat16, device=dev)  # (Q itself may be fp8)
    lse = torch.empty((T, cfg.n_q_heads), dtype=torch.float32, device=dev) if want_lse else None
    block_idx = torch.empty((T, cfg.n_kv_heads, cfg.top_k), dtype=torch.int32, device=dev)
    if workspace is None:
        mn, pf = B.msa_prefill_forward_workspace_bytes(shape, T)
        workspace = B.alloc_workspace(pf if workspace_bytes is None else max(mn, workspace_bytes), dev)
    B.msa_prefill_forward(shape, x["q"], x["k"], x["v"], x["q_idx"], x["k_idx"], T, out, lse,
                          block_idx, workspace)
    return out, lse, block_idx


def prefill_forward_varlen(cfg: MSAConfig, x: Dict[str, torch.Tensor], cu_seqlens,
                           workspace: Optional[torch.Tensor] = None, want_lse: bool = True):
    """The same for sequences packed token-major; cu_seqlens: n_seqs+1 row offsets (host ints).
    block_idx holds block numbers relative to each row's own sequence."""
    shape = B.shape_of(cfg)
    T = x["q"].shape[0]
    dev = x["q"].device
    out = torch.empty(x["q"].shape, dtype=torch.bfloat16, device=dev)
    lse = torch.empty((T, cfg.n_q_heads), dtype=torch.float32, device=dev) if want_lse else None
    block_idx = torch.empty((T, cfg.n_kv_heads, cfg.top_k), dtype=torch.int32, device=dev)
    if workspace is None:
        _, pf = B.msa_prefill_forward_varlen_workspace_bytes(shape, cu_seqlens)
        workspace = B.alloc_workspace(pf, dev)
    B.msa_prefill_forward_varlen(shape, x["q"], x["k"], x["v"], x["q_idx"], x["k_idx"], cu_seqlens, out, lse,
                                 block_idx, workspace)
    return out, lse, block_idx


def index_lse(cfg: MSAConfig, q_idx: torch.Tensor, k_idx: torch.Tensor, block_idx: torch.Tensor,
              q_begin: int = 0, q_count: Optional[int] = None, kv_len: Optional[int] = None,
              workspace_bytes: Optional[int] = None) -> torch.Tensor:
    """Section 4.3: log-sum-exp of the index scores over the selected blocks, rows
    [q_begin, q_begin+q_count); q_idx and block_idx hold the whole sequence's rows."""
    shape = B.shape_of(cfg)
    kv_len = k_idx.shape[0] if kv_len is None else kv_len
    q_count = q_idx.shape[0] - q_begin if q_count is None else q_count
    out = torch.empty((q_count, cfg.n_kv_heads), dtype=torch.float32, device=q_idx.device)
    mn, pf = B.msa_index_lse_prefill_workspace_bytes(shape, q_count, kv_len)
    ws = B.alloc_workspace(pf if workspace_bytes is None else max(mn, workspace_bytes), q_idx.device)
    B.msa_index_lse_prefill(shape, q_idx[q_begin:q_begin + q_count], k_idx, block_idx[q_begin:q_begin + q_count],
                            q_begin, q_count, kv_len, out, ws)
    return out


def index_scores(cfg: MSAConfig, q_idx: torch.Tensor, k_idx: torch.Tensor, q_begin: int, q_count: int,
                 kv_len: Optional[int] = None, score_runs: int = 0) -> torch.Tensor:
    """Eq. 6 for rows [q_begin, q_begin+q_count); q_idx holds the whole sequence's rows.
    score_runs = 1: the columns of a row come in run order (run_order_columns gives the map)."""
    shape = B.shape_of(cfg, score_runs=score_runs)
    kv_len = k_idx.shape[0] if kv_len is None else kv_len
    ld = B.score_ld(kv_len, cfg.block_size)
    if score_runs:
        ld = (ld + 7) // 8 * 8
    scores = torch.full((q_count, cfg.n_kv_heads, ld), float("nan"), dtype=torch.float32,
                        device=q_idx.device)
    B.msa_index_scores(shape, q_idx[q_begin:q_begin + q_count], k_idx, q_begin, q_count, kv_len,
                       scores, ld)
    return scores


def run_order_columns(n_blocks: int, block_size: int) -> torch.Tensor:
    """Column of block b in a score row in run order (msa_shape_t.score_runs = 1), for b < n_blocks."""
    n = 128 // block_size
    b = torch.arange(n_blocks, dtype=torch.int64)
    w = b % 8
    return (b - w) + 4 * ((w // n) % 2) + n * (w // (2 * n)) + (w % n)


def topk_select(cfg: MSAConfig, scores: torch.Tensor, q_begin: int, kv_len: int, score_runs: int = 0) -> torch.Tensor:
    shape = B.shape_of(cfg, score_runs=score_runs)
    q_count, _, ld = scores.shape
    block_idx = torch.empty((q_count, cfg.n_kv_heads, cfg.top_k), dtype=torch.int32,
                            device=scores.device)
    B.msa_topk_select(shape, scores, ld, q_begin, q_count, kv_len, block_idx)
    return block_idx


def sparse_attn_prefill(cfg: MSAConfig, q, k, v, block_idx, q_begin: int = 0,
                        workspace_bytes: Optional[int] = None):
    shape = B.shape_of(cfg)
    q_count, kv_len = q.shape[0], k.shape[0]
    out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
    lse = torch.empty((q_count, cfg.n_q_heads), dtype=torch.float32, device=q.device)
    mn, pf = B.msa_sparse_attn_prefill_workspace_bytes(shape, q_count, kv_len)
    ws = B.alloc_workspace(pf if workspace_bytes is None else max(mn, workspace_bytes), q.device)
    B.msa_sparse_attn_prefill(shape, q, k, v, block_idx, q_begin, q_count, kv_len, out, lse, ws)
    return out, lse


def decode_forward(cfg: MSAConfig, x: Dict[str, torch.Tensor]):
    """One decode step for a batch of cached sequences -> (out, lse, block_idx, scores)."""
    shape = B.shape_of(cfg)
    batch = x["q"].shape[0]
    dev = x["q"].device
    max_len = int(max(cfg.seq_lens))
    ld = B.score_ld(max_len, cfg.block_size)
    scores = torch.empty((batch, cfg.n_kv_heads, ld), dtype=torch.float32, device=dev)
    block_idx = torch.empty((batch, cfg.n_kv_heads, cfg.top_k), dtype=torch.int32, device=dev)
    out = torch.empty_like(x["q"])
    lse = torch.empty((batch, cfg.n_q_heads), dtype=torch.float32, device=dev)
    ws = B.alloc_workspace(B.msa_sparse_attn_decode_workspace_bytes(shape, batch), dev)
    B.msa_decode_forward(shape, x["q"], x["q_idx"], x["k_cache"], x["v_cache"], x["k_idx_cache"],
                         x["k_cache"].shape[0], x["seq_offsets"], x["seq_lens"], batch, max_len,
                         scores, ld, block_idx, out, lse, ws)
    return out, lse, block_idx, scores


# ------------------------------------------------------------------ around the path
class Rope(NamedTuple):
    """A position rotation: fp64 radians per position of each pair (on the device), the pairs' layout (elements i and
    i + n, or 2i and 2i+1), and a factor on the rotated elements."""
    freqs: torch.Tensor
    interleaved: bool = False
    mscale: float = 1.0


class PagedCache(NamedTuple):
    """Pools [pages, page size, KV heads, d] (bf16 or float8_e4m3fn; v may be None), the pages of each sequence int32
    [batch, pages], its length with the new tokens int32 [batch], and the first new row of each int32 [batch + 1]."""
    k: torch.Tensor
    v: Optional[torch.Tensor]
    page_table: torch.Tensor
    kv_lens: torch.Tensor
    cu_q: torch.Tensor


_NO_ROPE = Rope(None)


def _no_graph(call: str, instead: str, *tensors: Optional[torch.Tensor]) -> None:
    """Refuses tensors whose gradients a call would lose: it records nothing for automatic differentiation."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        raise ValueError("%s records no graph and gradients would be lost: %s" % (call, instead))



def _workspace(t: torch.Tensor, size, *args) -> torch.Tensor:
    """A workspace of size(*args) bytes on t's device (the size may depend on the device)."""
    if t.get_device() == torch.cuda.current_device():
        n = size(*args)
    else:
        with torch.cuda.device(t.device):
            n = size(*args)
    return t.new_empty(max(n, 256), dtype=torch.uint8)


def rope_frequencies(rot_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                     original_len: int = 4096, low: float = 1.0, high: float = 32.0, device="cuda") -> torch.Tensor:
    """fp64 frequencies base^(-2i/rot_dim) of a rotation of rot_dim elements, stretched for contexts `factor` times
    the original length: "linear" divides all by factor; "base" raises the base so that the slowest pair turns factor
    times slower and the fastest as before; "bands" keeps pairs that turn more than `high` times within original_len,
    divides those that turn fewer than `low` times, and blends linearly in the number of turns between."""
    i = torch.arange(rot_dim // 2, dtype=torch.float64)
    if scaling == "base":
        if rot_dim > 2:
            base = base * factor ** (rot_dim / (rot_dim - 2))
    elif scaling not in ("none", "linear", "bands"):
        raise ValueError("unknown scaling %r" % scaling)
    f = base ** (-2.0 * i / rot_dim)
    if scaling == "linear":
        f = f / factor
    elif scaling == "bands":
        keep = ((original_len * f / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        f = f * keep + f / factor * (1 - keep)
    return f.to(device)


def qk_norm_rope(q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: Optional[torch.Tensor],
                 rope: Optional[Rope] = None, q_weight: Optional[torch.Tensor] = None,
                 k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, q_out: Optional[torch.Tensor] = None,
                 k_out: Optional[torch.Tensor] = None):
    """Norm of each head (where there is a weight) and position rotation of q and k [rows, heads, d], which may be
    slices of one projection; either may be None -> (q_out, k_out), dense.  Records no graph: inputs that require
    gradients are refused outside torch.no_grad (qk_norm_rope_backward has the gradients)."""
    _no_graph("qk_norm_rope", "call it under torch.no_grad, and qk_norm_rope_backward in the backward pass", q, k, q_weight, k_weight)
    freqs, interleaved, mscale = rope or _NO_ROPE
    return B.msa_qk_norm_rope(freqs, interleaved, mscale, q, q_weight, k, k_weight, eps, positions, q_out, k_out)


def qk_norm_rope_backward(dq_out: Optional[torch.Tensor], dk_out: Optional[torch.Tensor], q: Optional[torch.Tensor],
                          k: Optional[torch.Tensor], positions: Optional[torch.Tensor], rope: Optional[Rope] = None,
                          q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
                          eps: float = 1e-6):
    """Gradients of qk_norm_rope's inputs for those of its outputs -> (dq, dk, dq_weight, dk_weight); the weights'
    are fp32, None without a weight."""
    dy = dq_out if dq_out is not None else dk_out
    d = dy.shape[-1]
    dwq = None if q_weight is None else dy.new_empty(d, dtype=torch.float32)
    dwk = None if k_weight is None else dy.new_empty(d, dtype=torch.float32)
    ws = None
    if dwq is not None or dwk is not None:
        ws = _workspace(dy, B.msa_qk_norm_rope_backward_workspace_bytes, d, dy.shape[0])
    freqs, interleaved, mscale = rope or _NO_ROPE
    dq, dk = B.msa_qk_norm_rope_backward(freqs, interleaved, mscale, dq_out, dk_out, q, q_weight, k, k_weight, eps, positions,
                                         None, None, dwq, dwk, ws)
    return dq, dk, dwq, dwk


def paged_append(cache: PagedCache, k: torch.Tensor, v: Optional[torch.Tensor], q: Optional[torch.Tensor] = None,
                 rope: Optional[Rope] = None, q_weight: Optional[torch.Tensor] = None,
                 k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, q_out: Optional[torch.Tensor] = None):
    """Writes the new tokens' keys (normed, turned) and values into the cache and returns their queries, treated like
    the keys (None without queries).  Rows behind the last sequence are left as they are (uninitialised in a q_out
    made here).  Inputs that require gradients are refused outside torch.no_grad."""
    _no_graph("paged_append", "a cache takes none; call it under torch.no_grad", q, k, v, q_weight, k_weight)
    freqs, interleaved, mscale = rope or _NO_ROPE
    return B.msa_paged_append(cache.k, cache.v, cache.page_table, cache.kv_lens, cache.cu_q, freqs, interleaved, mscale, q,
                              q_weight, k, k_weight, v, eps, q_out)


def paged_attn(cache: PagedCache, q: torch.Tensor, softmax_scale: float = 0.0, out: Optional[torch.Tensor] = None,
               want_lse: bool = True, workspace: Optional[torch.Tensor] = None, max_new: int = 0):
    """Dense causal attention of the new tokens q [rows, heads, d] over the cache, which already holds their keys and
    values -> (out, lse).  Rows behind the last sequence are left as they are (uninitialised in outputs made here).
    max_new: the most new tokens that a sequence has, if known (a hint, results do not depend on it; worth giving on fp8
    caches where sequences may have no new tokens beside one of many).  A q that requires gradients is refused outside
    torch.no_grad."""
    _no_graph("paged_attn", "it has no backward pass; call it under torch.no_grad", q)
    lse = q.new_empty(q.shape[:2], dtype=torch.float32) if want_lse else None
    if workspace is None:
        workspace = _workspace(q, B.msa_paged_attn_workspace_bytes, cache.k, q.shape[1])
    out = B.msa_paged_attn(cache.k, cache.v, cache.page_table, cache.kv_lens, cache.cu_q, q, softmax_scale, out, lse, workspace,
                           max_new=max_new)
    return out, lse
