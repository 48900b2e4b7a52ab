"""The calls around the path record no graph for automatic differentiation: tensors whose gradients would be lost are
refused where a graph would be recorded, and taken where none is (no GPU needed: refusals come first)."""

import pytest
import torch

from paper_2606_13392_b200 import api


def cases():
    q, k, w = [torch.zeros(s, dtype=torch.bfloat16) for s in ((2, 3, 128), (2, 1, 128), (128,))]
    pool = torch.zeros(4, 16, 1, 128, dtype=torch.bfloat16)
    cache = api.PagedCache(pool, pool, *[torch.zeros(s, dtype=torch.int32) for s in ((1, 4), (1,), (2,))])
    rotation = lambda t: api.qk_norm_rope(t["q"], t["k"], None, None, t["wq"], t["wk"])  # noqa: E731
    append = lambda t: api.paged_append(cache, t["k"], t["v"], t["q"], None, t["wq"], t["wk"])  # noqa: E731
    attention = lambda t: api.paged_attn(cache, t["q"], workspace=torch.zeros(256, dtype=torch.uint8))  # noqa: E731
    tensors = dict(q=q, k=k, v=k, wq=w, wk=w)
    for call, names in ((rotation, "q k wq wk"), (append, "q k v wq wk"), (attention, "q")):
        for name in names.split():
            yield call, tensors | {name: tensors[name].clone().requires_grad_()}


@pytest.mark.parametrize("i", range(10))
def test_tensors_that_require_gradients(i):
    call, tensors = list(cases())[i]
    with pytest.raises(ValueError, match="gradients would be lost"):
        call(tensors)
    with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):  # taken, up to the check of the device
        call(tensors)
    with pytest.raises(ValueError, match="CUDA"):
        call({n: t.detach() for n, t in tensors.items()})


@pytest.mark.gpu
def test_parameters_without_a_graph():
    w = torch.nn.Parameter(torch.ones(128, device="cuda"))
    q = torch.randn(5, 2, 128, device="cuda").bfloat16()
    with torch.no_grad():
        out, _ = api.qk_norm_rope(q, None, None, None, w)
    assert torch.equal(out, api.qk_norm_rope(q, None, None, None, w.detach())[0])

    class Turned(torch.autograd.Function):  # as a training program wires the two calls up
        @staticmethod
        def forward(ctx, x, w):
            ctx.save_for_backward(x, w)
            return api.qk_norm_rope(x, None, None, None, w)[0]

        @staticmethod
        def backward(ctx, dy):
            x, w = ctx.saved_tensors
            dx, _, dw, _ = api.qk_norm_rope_backward(dy.contiguous(), None, x, None, None, None, w)
            return dx, dw

    x = q.clone().requires_grad_()
    dy = torch.randn(5, 2, 128, device="cuda").bfloat16()
    Turned.apply(x, w).backward(dy)
    want = api.qk_norm_rope_backward(dy, None, q, None, None, None, w.detach())
    assert torch.equal(x.grad, want[0]) and torch.equal(w.grad, want[2])
