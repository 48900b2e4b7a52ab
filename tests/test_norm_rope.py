"""Norms of queries and keys with the position rotation: forward and gradients against the definition in 64 bits
(a rotation as a complex product, gradients by automatic differentiation and by differences), and refusals.

Tolerances.  The one rounding is the store in bf16: at most half a step, 2^-8 of the value.  Before it everything is
fp32 (2^-24 a step): the mean of squares of d <= 256 values is off by at most d steps, the angle's remainder by 2^-25
turns, a rotated element is a sum of two products whose size its pair bounds; together below 2^-15 of the largest
element of the row.  A weight gradient is a sum over tokens and heads whose longest chain of additions is below 400 at
these sizes (a lane's items, then lanes, warps and rows), each term off by at most d + 20 steps."""

import math

import pytest
import torch

from paper_2606_13392_b200 import api
from paper_2606_13392_b200 import binding as B

DEV = "cuda"


def turn(x, w, positions, freqs, interleaved, mscale, eps):
    """The definition, in the type of x."""
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * w
    if freqs is None:
        return x
    n = freqs.shape[0]
    first = torch.arange(n, device=x.device) * (2 if interleaved else 1)
    second = first + (1 if interleaved else n)
    angle = (positions.double()[:, None] * freqs)[:, None]
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.full_like(angle, mscale), angle)
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def make(rows, hq, hk, d, rot, norm, w32, strided, seed=0, far=1 << 20):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    width = (hq + hk) * d
    if strided:  # slices of a wider projection, 16 bytes into a row
        x = (rand(rows, width + 24) * 3).bfloat16()[:, 8:]
        q, k = x[:, :hq * d].unflatten(1, (hq, d)) if hq else None, x[:, hq * d:width].unflatten(1, (hk, d)) if hk else None
    else:
        q = (rand(rows, hq, d) * 3).bfloat16() if hq else None
        k = (rand(rows, hk, d) * 3).bfloat16() if hk else None
    kind = torch.float32 if w32 else torch.bfloat16
    wq, wk = ((1 + rand(d) * 0.5).to(kind), (1 + rand(d) * 0.5).to(kind)) if norm else (None, None)
    positions = torch.randint(-far, far, (rows,), generator=g, device=DEV)
    freqs = api.rope_frequencies(rot, 5e6, "bands", 8.0, 32768) if rot else None
    return q, k, wq, wk, positions, freqs


CASES = [  # rows, q heads, k heads, d, rot, interleaved, norm, fp32 weights, strided, mscale
    (1, 64, 8, 128, 128, False, True, False, True, 1.0),
    (33, 64, 8, 128, 64, False, True, True, True, 1.3),
    (700, 64, 4, 128, 128, True, True, False, False, 0.7),
    (2999, 8, 1, 64, 32, True, False, False, True, 1.0),
    (257, 3, 5, 64, 64, False, True, False, True, 1.0),
    (130, 7, 1, 96, 48, False, True, False, False, 1.0),
    (65, 5, 3, 80, 24, True, True, True, True, 1.0),
    (40, 9, 2, 256, 256, False, True, False, False, 1.0),
    (19, 0, 3, 128, 16, False, True, False, False, 1.0),
    (19, 6, 0, 8, 8, True, True, False, False, 1.0),
    (50, 4, 2, 128, 0, False, True, False, True, 1.0),
    (5000, 2, 1, 32, 16, False, False, False, False, 1.0),
    (9501, 2, 1, 128, 128, False, True, False, True, 1.0),   # more rows than CTAs hold at a time
]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,hq,hk,d,rot,inter,norm,w32,strided,mscale", CASES)
def test_forward(rows, hq, hk, d, rot, inter, norm, w32, strided, mscale):
    q, k, wq, wk, positions, freqs = make(rows, hq, hk, d, rot, norm, w32, strided)
    rope = api.Rope(freqs, inter, mscale) if rot else None
    outs = api.qk_norm_rope(q, k, positions, rope, wq, wk, 1e-5)
    for x, w, y in ((q, wq, outs[0]), (k, wk, outs[1])):
        if x is None:
            assert y is None
            continue
        ref = turn(x.double(), None if w is None else w.double(), positions, freqs, inter, mscale, 1e-5)
        tol = 2.0 ** -8 * ref.abs() + 2.0 ** -15 * ref.abs().amax(-1, keepdim=True)
        assert y.is_contiguous() and (y.double() - ref).abs().le(tol).all()
        if not norm:  # what is not turned is copied
            assert torch.equal(y[..., rot:], x[..., rot:])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,hq,hk,d,rot,inter,norm,w32,strided,mscale", CASES)
def test_gradients(rows, hq, hk, d, rot, inter, norm, w32, strided, mscale):
    q, k, wq, wk, positions, freqs = make(rows, hq, hk, d, rot, norm, w32, strided)
    dys = make(rows, hq, hk, d, 0, False, False, strided, seed=1)[:2]
    rope = api.Rope(freqs, inter, mscale) if rot else None
    got = api.qk_norm_rope_backward(dys[0], dys[1], q, k, positions, rope, wq, wk, 1e-5)
    again = api.qk_norm_rope_backward(dys[0], dys[1], q, k, positions, rope, wq, wk, 1e-5)
    for x, w, dy, dx, dw in ((q, wq, dys[0], got[0], got[2]), (k, wk, dys[1], got[1], got[3])):
        if x is None:
            assert dx is None
            continue
        xd = x.double().requires_grad_()
        wd = None if w is None else w.double().requires_grad_()
        turn(xd, wd, positions, freqs, inter, mscale, 1e-5).backward(dy.double())
        # the terms whose difference dx is bound the fp32 error before the store
        g = torch.autograd.grad(turn(xd, None, positions, freqs, inter, mscale, 0.0), xd, dy.double())[0].detach()
        if w is None:
            size = g.abs().amax(-1, keepdim=True)
        else:
            r = torch.rsqrt(xd.detach().square().mean(-1, keepdim=True) + 1e-5)
            xh, gw = xd.detach() * r, g * wd.detach()
            size = r * (gw.abs() + xh.abs() * (gw * xh).abs().mean(-1, keepdim=True)).amax(-1, keepdim=True)
        assert (dx.double() - xd.grad).abs().le(2.0 ** -8 * xd.grad.abs() + 2.0 ** -15 * size).all()
        if w is None:
            assert dw is None
            continue
        terms = (g * xh).abs().sum((0, 1))
        assert dw.dtype == torch.float32 and (dw.double() - wd.grad).abs().le((400 + d + 20) * 2.0 ** -24 * terms).all()
        # differences of the definition along a direction
        u = torch.randn(x.shape, generator=torch.Generator(device=DEV).manual_seed(5), device=DEV).double()
        f = lambda t: (turn(t, wd.detach(), positions, freqs, inter, mscale, 1e-5) * dy.double()).sum()  # noqa: E731
        h = 1e-5
        slope = (f(x.double() + h * u) - f(x.double() - h * u)) / (2 * h)
        terms = (dx.double() * u).abs().sum() + (size * u.abs()).sum() * 2.0 ** -7
        assert abs(float((dx.double() * u).sum() - slope)) <= float(terms) * 2.0 ** -8 + 1e-4
    for a, b in zip(got, again):
        assert a is None or torch.equal(a, b)


@pytest.mark.gpu
def test_far_positions_and_in_place():
    # 2^53 positions behind the origin are still whole turns plus the exact remainder (a frequency that is a power
    # of two fraction of a turn), and an output may be its own input
    q = torch.randn(4, 2, 32, device=DEV).bfloat16()
    freqs = torch.full((16,), 2 * math.pi / 8, dtype=torch.float64, device=DEV)
    positions = torch.tensor([0, 1 << 20, (1 << 40) + 8, (1 << 20) + 2], device=DEV)
    ref = turn(q.double(), None, positions % 8, freqs, False, 1.0, 0.0)
    out, _ = api.qk_norm_rope(q, None, positions, api.Rope(freqs), q_out=q)
    assert out is q
    # four roundings of 2^-53 (the frequency, 1 / 2 pi, their product, the position's) of 2^37 turns: 2^-14 turns
    assert (q.double() - ref).abs().le(2.0 ** -8 * ref.abs() + 2 * math.pi * 2.0 ** -14 * 2 ** 0.5 * ref.abs().max()).all()


@pytest.mark.gpu
def test_gradients_in_place_and_on_a_given_stream():
    q, k, wq, wk, positions, freqs = make(777, 6, 2, 128, 64, True, True, True)
    rope = api.Rope(freqs, False, 1.1)
    dq, dk = torch.randn(777, 6, 128, device=DEV).bfloat16(), torch.randn(777, 2, 128, device=DEV).bfloat16()
    want = api.qk_norm_rope_backward(dq, dk, q, k, positions, rope, wq, wk)
    ws = B.alloc_workspace(B.msa_qk_norm_rope_backward_workspace_bytes(128, 777), DEV)
    sums = torch.empty(2, 128, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.msa_qk_norm_rope_backward(freqs, False, 1.1, dq, dk, q, wq, k, wk, 1e-6, positions, dq, dk, sums[0], sums[1], ws, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((dq, dk, sums[0], sums[1]), want))


@pytest.mark.gpu
def test_zeros_infinities_and_empty_calls():
    q = torch.zeros(3, 3, 128, device=DEV).bfloat16()
    q[1, 1, 5] = math.inf
    w = torch.ones(128, device=DEV)
    positions = torch.arange(3, device=DEV)
    rope = api.Rope(api.rope_frequencies(64))
    out, _ = api.qk_norm_rope(q, None, positions, rope, w)
    assert (out[0] == 0).all() and (out[2] == 0).all() and (out[1, 0] == 0).all() and out[1, 1, 5].isnan()
    # without a norm an infinity stays in its own pair
    out, _ = api.qk_norm_rope(q, None, positions, rope)
    rest = torch.ones(128, dtype=torch.bool, device=DEV)
    rest[[5, 37]] = False
    assert (out[1, 1][rest] == 0).all() and not out[1, 1, 5].isfinite()
    # eps = 0 with an odd number of heads: the lanes of the head that is not there add nothing
    q = torch.randn(3, 3, 128, device=DEV).bfloat16()
    assert api.qk_norm_rope_backward(q, None, q, None, positions, rope, w, eps=0.0)[2].isfinite().all()
    none = q[:0]
    out, _ = api.qk_norm_rope(none, None, positions[:0], rope, w)
    assert out.shape == (0, 3, 128)
    dq, _, dw, _ = api.qk_norm_rope_backward(none, None, none, None, positions[:0], rope, w)
    assert dq.shape == (0, 3, 128) and (dw == 0).all()


@pytest.mark.gpu
def test_streams_and_graphs():
    q, k, wq, wk, positions, freqs = make(300, 8, 2, 128, 64, True, False, True)
    rope = api.Rope(freqs, True)
    dq = torch.randn(300, 8, 128, device=DEV).bfloat16()
    dk = torch.randn(300, 2, 128, device=DEV).bfloat16()
    want = api.qk_norm_rope(q, k, positions, rope, wq, wk) + api.qk_norm_rope_backward(dq, dk, q, k, positions, rope, wq, wk)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = api.qk_norm_rope(q, k, positions, rope, wq, wk) + api.qk_norm_rope_backward(dq, dk, q, k, positions, rope, wq, wk)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = api.qk_norm_rope(q, k, positions, rope, wq, wk) + api.qk_norm_rope_backward(dq, dk, q, k, positions, rope, wq, wk)
    positions += 17  # a replay follows the values
    graph.replay()
    torch.cuda.synchronize()
    want = api.qk_norm_rope(q, k, positions, rope, wq, wk) + api.qk_norm_rope_backward(dq, dk, q, k, positions, rope, wq, wk)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals_of_the_abi():
    import ctypes
    lib = B.lib()
    one = ctypes.c_void_p(256)  # non-null and aligned, never followed on these paths
    f = ctypes.c_float

    def call(rope=B.MsaRope(256, 64, 0, 1.0), q=one, qs=512, hq=4, d=128, w32=0, eps=1e-6, pos=one, n=5, qo=one, k=one, ks=128, hk=1, ko=one):
        return lib.msa_qk_norm_rope(None if rope is None else ctypes.byref(rope), q, B.c_i64(qs), B.c_i32(hq), None, k, B.c_i64(ks),
                                    B.c_i32(hk), None, B.c_i32(d), B.c_i32(w32), f(eps), pos, B.c_i64(n), qo, ko, None)

    assert call(n=0) == 0 and call(hq=0, hk=0) == 0
    assert call(q=None) == 1 and call(qo=None) == 1 and call(ko=None) == 1 and call(pos=None) == 1
    assert call(q=ctypes.c_void_p(264)) == 1                     # not on 16 bytes
    assert call(qs=511) == 1 and call(qs=516) == 1 and call(ks=120) == 1
    assert call(n=-1) == 1 and call(hq=-1) == 1 and call(w32=2) == 1 and call(d=0) == 1
    assert call(eps=-1.0) == 1 and call(eps=math.nan) == 1 and call(eps=math.inf) == 1
    assert call(d=100) == 2 and call(d=264) == 2 and call(hq=2000, qs=1 << 20) == 2
    assert call(rope=B.MsaRope(256, 130, 0, 1.0)) == 1 and call(rope=B.MsaRope(256, -2, 0, 1.0)) == 1
    assert call(rope=B.MsaRope(None, 64, 0, 1.0)) == 1 and call(rope=B.MsaRope(256, 64, 2, 1.0)) == 1
    assert call(rope=B.MsaRope(256, 64, 0, math.nan)) == 1
    assert call(rope=B.MsaRope(256, 24, 0, 1.0)) == 2 and call(rope=B.MsaRope(256, 12, 1, 1.0)) == 2
    i64, i32, sz = B.c_i64, B.c_i32, B.c_sz
    back = lambda ws, nbytes, n=5, dq=one: lib.msa_qk_norm_rope_backward(  # noqa: E731
        None, one, i64(512), None, i64(0), one, i64(512), i32(4), one, None, i64(0), i32(0), None, i32(128), i32(0), f(1e-6),
        None, i64(n), dq, None, one, None, ws, sz(nbytes), None)
    assert back(one, 16) == 3 and back(None, 1 << 20) == 1 and back(one, 1 << 20, dq=None) == 1 and back(one, 1 << 20, n=-1) == 1


def test_refusals_of_the_binding():
    q = torch.zeros(2, 3, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        api.qk_norm_rope(q, None, None)
    with pytest.raises(ValueError, match="scaling"):
        api.rope_frequencies(64, scaling="other", device="cpu")


@pytest.mark.gpu
def test_refusals_of_tensors():
    q = torch.zeros(2, 3, 128, dtype=torch.bfloat16, device=DEV)
    rope, pos = api.Rope(api.rope_frequencies(64)), torch.zeros(2, dtype=torch.int64, device=DEV)
    bad = [dict(q=q.float()), dict(q=q.transpose(0, 1)), dict(k=q[:1]), dict(k=q[..., :64]), dict(positions=pos.int()),
           dict(positions=pos[:1]), dict(rope=api.Rope(rope.freqs.float())), dict(rope=api.Rope(rope.freqs.cpu())),
           dict(q_weight=torch.ones(64, device=DEV)), dict(q_weight=torch.ones(128, device=DEV).half()),
           dict(q_weight=torch.ones(128, device=DEV), k_weight=torch.ones(128, device=DEV).bfloat16()),
           dict(q_out=torch.empty(2, 4, 128, dtype=torch.bfloat16, device=DEV)),
           dict(q_out=torch.empty(2, 3, 256, dtype=torch.bfloat16, device=DEV)[..., ::2])]
    for change in bad:
        args = dict(q=q, k=q, positions=pos, rope=rope) | change
        with pytest.raises(ValueError):
            api.qk_norm_rope(**args)
    with pytest.raises(B.MsaError):  # rows that do not start on 16 bytes
        api.qk_norm_rope(torch.zeros(2, 3 * 128 + 4, dtype=torch.bfloat16, device=DEV)[:, 4:].unflatten(1, (3, 128)), None, pos, rope)
    with pytest.raises(B.MsaError):
        api.qk_norm_rope(q, None, None, rope)


def test_frequencies():
    f = api.rope_frequencies(8, 10000.0, device="cpu")
    assert torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-14)
    assert torch.allclose(api.rope_frequencies(8, scaling="linear", factor=4.0, device="cpu"), f / 4, rtol=1e-14)
    g = api.rope_frequencies(8, scaling="base", factor=4.0, device="cpu")
    assert math.isclose(g[0], 1.0) and math.isclose(g[-1], f[-1] / 4, rel_tol=1e-12)
    g = api.rope_frequencies(64, 1e4, "bands", 8.0, 4096, 1.0, 32.0, device="cpu")
    f = api.rope_frequencies(64, 1e4, device="cpu")
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(g[turns >= 32], f[turns >= 32]) and torch.equal(g[turns <= 1], f[turns <= 1] / 8)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and (g[mid] < f[mid]).all() and (g[mid] > f[mid] / 8).all()
