"""Outputs that a call on a given stream makes: no work of the caller's current stream may still use their memory, and
none may get it while the call writes."""

import pytest
import torch

from paper_2606_13392_b200 import api
from paper_2606_13392_b200 import binding as B
from test_paged_append import batch, rows_of

DEV = "cuda"
BUSY = 40_000_000  # cycles, some 20 ms


def calls():
    """Name, call(outs..., stream) -> outputs, how many of them it makes; 600 rows, so that each output fills a block of its own."""
    n = 600
    q, k = rows_of(n, 8, 128, 1), rows_of(n, 8, 128, 2)
    w = torch.ones(128, device=DEV)
    positions, freqs = torch.arange(n, device=DEV), api.rope_frequencies(64)
    yield "rotation", lambda a, b, s: B.msa_qk_norm_rope(freqs, False, 1.0, q, w, k, w, 1e-6, positions, a, b, stream=s), 2
    sums = torch.zeros(2, 128, device=DEV)
    ws = B.alloc_workspace(B.msa_qk_norm_rope_backward_workspace_bytes(128, n), DEV)
    yield ("gradients", lambda a, b, s: B.msa_qk_norm_rope_backward(freqs, False, 1.0, q, k, q, w, k, w, 1e-6, positions, a, b, sums[0],
                                                                    sums[1], ws, stream=s), 2)
    cache = batch([(n, 300)], 16, 8, 128, False)
    yield ("append", lambda a, s: (B.msa_paged_append(*cache, freqs, False, 1.0, q, w, k, w, k, 1e-6, a, stream=s),), 1)
    qd = q.contiguous()
    work = B.alloc_workspace(B.msa_paged_attn_workspace_bytes(cache.k, 8), DEV)
    yield "attention", lambda a, s: (B.msa_paged_attn(*cache, qd, 0.0, a, None, work, stream=s),), 1


@pytest.mark.gpu
def test_outputs_made_while_the_current_stream_is_busy():
    side = torch.cuda.Stream()
    for name, call, n in calls():
        outs = [torch.empty(600, 8, 128, dtype=torch.bfloat16, device=DEV) for _ in range(n)]
        call(*outs, None)
        want = [o.clone() for o in outs]
        side.wait_stream(torch.cuda.current_stream())
        torch.cuda.synchronize()
        # blocks of the outputs' size that work still to come on the current stream writes
        torch.cuda._sleep(BUSY)
        for o in outs:
            o.fill_(7.0)
        del outs, o
        got = call(*[None] * n, side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name


@pytest.mark.gpu
def test_outputs_freed_while_the_given_stream_writes():
    side = torch.cuda.Stream()
    for name, call, n in calls():
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(BUSY)
        call(*[None] * n, side)  # (the outputs are dropped at once)
        mine = [torch.full((600, 8, 128), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(4)]
        torch.cuda.synchronize()
        assert all((m == 3).all() for m in mine), name


@pytest.mark.gpu
def test_outputs_read_by_the_current_stream_after_they_are_dropped():
    side = torch.cuda.Stream()
    for name, call, n in calls():
        want = [o.clone() for o in call(*[None] * n, None)]
        torch.cuda.synchronize()
        got = call(*[None] * n, side)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda._sleep(BUSY)
        seen = [o.clone() for o in got]
        del got
        with torch.cuda.stream(side):  # memory of the side stream, asked for again while the copies are still to come
            for _ in range(4):
                torch.full((600, 8, 128), 3.0, dtype=torch.bfloat16, device=DEV)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(seen, want)), name
