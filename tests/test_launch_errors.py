"""A launch that the host refuses is reported by its own call and by no other.

The refusal is made on the host: while a stream that synchronises with the legacy stream is being captured, the runtime
turns down launches on the legacy stream (it would be an implicit dependency on the capture).  Nothing runs."""

import contextlib
import ctypes

import pytest
import torch

from paper_2606_13392_b200 import api
from paper_2606_13392_b200 import binding as B
from paper_2606_13392_b200.inputs import MSAConfig, make_decode_inputs
from test_paged_append import batch, rows_of

DEV = "cuda"


@contextlib.contextmanager
def a_capture_elsewhere():
    torch.zeros(1, device=DEV)
    torch.cuda.synchronize()
    driver = ctypes.CDLL("libcuda.so.1")
    stream, graph = ctypes.c_void_p(), ctypes.c_void_p()
    assert driver.cuStreamCreate(ctypes.byref(stream), 0) == 0
    assert driver.cuStreamBeginCapture_v2(stream, 2) == 0
    try:
        yield
    finally:
        driver.cuStreamEndCapture(stream, ctypes.byref(graph))
        if graph.value:
            driver.cuGraphDestroy(graph)
        assert driver.cuStreamDestroy_v2(stream) == 0


def calls():
    """Name, call, outputs of each; every call has its buffers."""
    legacy = torch.cuda.default_stream()
    assert legacy.cuda_stream == 0
    q, k = rows_of(40, 8, 128, 1), rows_of(40, 2, 128, 2)
    w = torch.ones(128, device=DEV)
    positions, freqs = torch.arange(40, device=DEV), api.rope_frequencies(64)
    made = [torch.zeros_like(x, memory_format=torch.contiguous_format) for x in (q, k, q, k, q, q, q)]
    yield "rotation", lambda: B.msa_qk_norm_rope(freqs, False, 1.0, q, w, k, w, 1e-6, positions, made[0], made[1], stream=legacy), made[:2]
    sums = torch.zeros(2, 128, device=DEV)
    ws = B.alloc_workspace(B.msa_qk_norm_rope_backward_workspace_bytes(128, 40), DEV)
    yield "gradients", lambda: B.msa_qk_norm_rope_backward(freqs, False, 1.0, q, k, q, w, k, w, 1e-6, positions, made[2], made[3], sums[0],
                                                           sums[1], ws, stream=legacy), [made[2], made[3], sums]
    for i, (fp8, lens) in enumerate(((False, [(39, 700), (1, 300)]), (True, [(39, 700), (1, 300)]), (True, [(1, 90)] * 40))):
        cache = batch(lens, 16, 2, 128, fp8)
        out, lse, qd = torch.zeros_like(made[0]), torch.zeros(40, 8, device=DEV), q.contiguous()
        work = B.alloc_workspace(B.msa_paged_attn_workspace_bytes(cache.k, 8), DEV)
        turned = made[4 + i]
        yield ("append", lambda c=cache, t=turned: B.msa_paged_append(*c, freqs, False, 1.0, q, w, k, w, k, 1e-6, t, stream=legacy),
               [turned, cache.k, cache.v])
        yield ("attention", lambda c=cache, o=out, ls=lse, ws=work, x=qd: B.msa_paged_attn(*c, x, 0.0, o, ls, ws, stream=legacy), [out, lse])
    cfg = MSAConfig("small", "decode", 600, 16, 2, 128, 4, seq_lens=(600, 257))
    x = make_decode_inputs(cfg, device=DEV)
    res = api.decode_forward(cfg, x)
    shape, work = B.shape_of(cfg), B.alloc_workspace(B.msa_sparse_attn_decode_workspace_bytes(B.shape_of(cfg), 2), DEV)
    out, lse, idx, scores = [torch.zeros_like(t) for t in res]
    yield ("sparse decode", lambda: B.msa_decode_forward(shape, x["q"], x["q_idx"], x["k_cache"], x["v_cache"], x["k_idx_cache"],
                                                         x["k_cache"].shape[0], x["seq_offsets"], x["seq_lens"], 2, 600, scores,
                                                         scores.shape[-1], idx, out, lse, work, stream=legacy), [out, lse, idx])


@pytest.mark.gpu
def test_a_refused_launch_is_reported_once():
    bits = lambda t: t.clone().view(torch.uint8)  # noqa: E731
    seen = list(calls())
    wants = []
    for name, call, outs in seen:
        call()
        wants.append([bits(t) for t in outs])
    assert B.check_async_status() == (0, 0)
    for (name, call, outs), want in zip(seen, wants):
        with a_capture_elsewhere(), pytest.raises(B.MsaError) as e:
            call()
        assert e.value.code == 4, name
        for (other, again, outs2), want2 in zip(seen, wants):  # this call and every other one: as if nothing had been
            for t in outs2:
                if other != "append" or t.dim() == 3:
                    t.zero_()
            again()
            assert all(torch.equal(bits(t), w) for t, w in zip(outs2, want2)), (name, other)
        assert float(torch.ones(1000, device=DEV).sum()) == 1000
    assert B.check_async_status() == (0, 0)
