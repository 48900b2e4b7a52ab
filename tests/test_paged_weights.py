"""The attention weight that cached tokens receive: against the definition in 64 bits.

Tolerance.  A term is exp(x), x = scale <q, k> - lse.  In fp32 x is off by at most 128 * 2^-24 * scale * sum |q_c k_c| (a sum of
d products, any order; d <= 256 taken as twice that), by 2^-23 (|scale <q, k>| + |lse|) for the factors, the difference and the change to
base two, and the exponential by 2^-21 of itself; fp8 caches take powers of two out of the queries, which is exact down to 2^-24 of
what is left, below the sum's bound.  Terms are positive, so a sum of n of them is off by n 2^-24 of itself at most, whatever
its order, and the faded old weight by two roundings."""

import ctypes
import math

import pytest
import torch

from paper_2606_13392_b200 import api
from paper_2606_13392_b200 import binding as B
from test_paged_append import batch

DEV = "cuda"


def filled(cache, seed=0):
    """The cache with its new tokens' keys as well (paged_append's work), in place."""
    g = torch.Generator(device=DEV).manual_seed(seed + 1)
    cu, table = cache.cu_q.tolist(), cache.page_table.cpu()
    page = cache.k.shape[1]
    for s, n in enumerate(cache.kv_lens.tolist()):
        for p in range(max(0, n - (cu[s + 1] - cu[s])), n):
            row = torch.randn(cache.k.shape[2:], generator=g, device=DEV).to(cache.k.dtype)
            cache.k.view(torch.uint8)[int(table[s, p // page]), p % page] = row.view(torch.uint8)
    return cache


def queries(cache, hq, extra=0, seed=3, scale=1.5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = int(cache.cu_q[-1])
    q = (scale * torch.randn(n + extra, hq, cache.k.shape[3], generator=g, device=DEV)).bfloat16()
    q[n:] = math.nan
    return q


def reference(cache, q, lse, weights, decay, scale=None):
    """(weights, tolerance) in 64 bits; lse None: computed here, and returned."""
    cu, kv, table = cache.cu_q.tolist(), cache.kv_lens.tolist(), cache.page_table.long()
    page, heads, d = cache.k.shape[1:]
    g = q.shape[1] // heads
    scale = d ** -0.5 if scale is None else scale
    out, tol = weights.double(), torch.zeros_like(weights, dtype=torch.float64)
    made = torch.full(q.shape[:2], math.nan, device=DEV) if lse is None else lse
    for s, n in enumerate(kv):
        new = cu[s + 1] - cu[s]
        if new == 0 or n == 0:
            if lse is None:
                made[cu[s]:cu[s + 1]] = -math.inf
            continue
        place = torch.arange(n, device=DEV)
        at = (table[s][place // page], place % page)
        k = cache.k.view(torch.uint8)[at].view(cache.k.dtype).double()
        seen = place <= torch.arange(n - new, n, device=DEV)[:, None]
        for h in range(heads):
            rows = q[cu[s]:cu[s + 1], h * g:(h + 1) * g].double().transpose(0, 1)
            x = scale * rows @ k[:, h].T
            size = scale * rows.abs() @ k[:, h].abs().T
            if lse is None:
                made[cu[s]:cu[s + 1], h * g:(h + 1) * g] = x.masked_fill(~seen, -math.inf).logsumexp(-1).T.float()
            ls = made[cu[s]:cu[s + 1], h * g:(h + 1) * g].T.double()[..., None]
            term = torch.where(seen & (ls != -math.inf), (x - ls).exp(), 0.0)
            off = size * max(128, d) * 2.0 ** -24 + 2.0 ** -23 * (x.abs() + ls.abs()) + 2.0 ** -21
            off = torch.where(term > 0, off, 0.0)
            got = term.sum((0, 1))
            old = out[at[0], h, at[1]]
            old = torch.where((place < n - new) & (decay != 0), decay * old, 0.0)
            out[at[0], h, at[1]] = old + got
            tol[at[0], h, at[1]] = (term * off).sum((0, 1)) * 1.01 + got * (new * g) * 2.0 ** -24 + (old + got).abs() * 2.0 ** -22 + 2.0 ** -100
    return out, tol, made


CASES = [  # lens (new, old), page, q heads, kv heads, d, fp8, decay
    ([(1, 0)], 1, 4, 1, 128, False, 1.0),
    ([(1, 77), (1, 0), (1, 4095), (0, 64), (1, 64)], 64, 64, 8, 128, False, 0.5),
    ([(1, 77), (1, 0), (1, 2095), (0, 64), (1, 64)], 64, 64, 4, 128, True, 0.5),
    ([(0, 9), (5, 0), (0, 0), (130, 31), (1, 15)], 16, 16, 4, 128, True, 0.0),
    ([(333, 5), (64, 64), (3, 700)], 7, 6, 2, 128, False, 1.0),
    ([(20, 500), (900, 0)], 128, 8, 8, 128, True, 1.0),
    ([(257, 515), (1, 1000)], 16, 16, 2, 128, False, 0.25),
    ([(2, 1), (0, 3)] * 600, 4, 1, 1, 128, False, 1.0),          # more sequences than threads
    ([(2, 130), (5, 30)], 24, 128, 1, 128, False, 1.0),
    ([(3, 50), (1, 40)], 8, 300, 1, 128, True, 1.0),              # a group beyond a tile of rows
    ([(33, 100)], 32, 6, 2, 64, False, 0.9),
    ([(70, 1), (0, 4), (2, 150)], 48, 3, 1, 96, True, 0.9),
    ([(9, 9)], 5, 2, 2, 256, False, 0.0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("lens,page,hq,hkv,d,fp8,decay", CASES)
def test_weights(lens, page, hq, hkv, d, fp8, decay):
    cache = filled(batch(lens, page, hkv, d, fp8, values=False))
    q = queries(cache, hq, extra=5)
    g = torch.Generator(device=DEV).manual_seed(9)
    pages = cache.k.shape[0]
    weights = torch.rand(pages, hkv, page, generator=g, device=DEV)
    if decay == 0:
        weights.fill_(math.nan)  # not read
    want, tol, lse = reference(cache, q, None, weights, decay)
    before = weights.clone()
    assert api.paged_weights(cache, q, lse, weights, decay) is weights
    assert B.check_async_status() == (0, 0)
    table, cu = cache.page_table.cpu(), cache.cu_q.tolist()
    touched = torch.zeros_like(weights, dtype=torch.bool)
    for s, n in enumerate(cache.kv_lens.tolist()):
        for p in range(n if cu[s + 1] > cu[s] else 0):
            touched[int(table[s, p // page]), :, p % page] = True
    assert torch.equal(weights.view(torch.int32)[~touched], before.view(torch.int32)[~touched])
    assert (weights.double() - want)[touched].abs().le(tol[touched]).all()
    assert touched.any()


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens", [[(1, 700), (1, 33)], [(40, 300), (7, 1000), (1, 5)]])
def test_equal_calls_give_equal_bits_and_a_hint_changes_little(lens, fp8):
    cache = filled(batch(lens, 16, 2, 128, fp8, values=False))
    q = queries(cache, 16)
    start = torch.rand(cache.k.shape[0], 2, 16, device=DEV)
    _, _, lse = reference(cache, q, None, start, 1.0)
    outs = [api.paged_weights(cache, q, lse, start.clone(), 0.7, max_new=m) for m in (0, 0, 40, 1000)]
    assert torch.equal(outs[0], outs[1])
    want, tol, _ = reference(cache, q, lse, start, 0.7)
    for o in outs:
        assert (o.double() - want).abs().le(tol + 1e-9).all()


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[(1, 300)], [(200, 100)]])
@pytest.mark.parametrize("d", [64, 128])
def test_what_is_masked_or_not_finite_stays_where_it_is(lens, d):
    cache = filled(batch(lens, 16, 1, d, False, values=False))
    q = queries(cache, 8)
    start = torch.rand(cache.k.shape[0], 1, 16, device=DEV)
    want, tol, lse = reference(cache, q, None, start, 1.0)
    table, n = cache.page_table.cpu(), lens[0][0] + lens[0][1]
    # a query that saw nothing
    lse2 = lse.clone()
    lse2[0, 3] = -math.inf
    want2, tol2, _ = reference(cache, q, lse2, start, 1.0)
    got = api.paged_weights(cache, q, lse2, start.clone())
    assert (got.double() - want2).abs().le(tol2 + 1e-9).all()
    # a key that is not a number: its own place only
    for value in (math.nan, math.inf):
        last = (int(table[0, (n - 1) // 16]), (n - 1) % 16)
        cache.k[last] = value
        got = api.paged_weights(cache, q, lse, start.clone())
        other = torch.ones_like(got, dtype=torch.bool)
        other[last[0], 0, last[1]] = False
        assert (got.double() - want)[other].abs().le((tol + 1e-9)[other]).all()
    # more new tokens than the length says: the first ones see nothing
    cache = filled(batch(lens, 16, 1, d, False, values=False))
    short = cache._replace(kv_lens=torch.tensor([max(1, lens[0][0] - 7)], dtype=torch.int32, device=DEV))
    want, tol, lse = reference(short, q, None, start, 1.0)
    got = api.paged_weights(short, q, lse, start.clone())
    assert B.check_async_status() == (0, 0)
    assert (got.double() - want).abs().le(tol + 1e-9).all()


@pytest.mark.gpu
@pytest.mark.parametrize("hq,new", [(8, 1), (64, 200)])
def test_scale_and_large_scores(hq, new):
    cache = filled(batch([(new, 400)], 64, 1, 128, True, values=False))
    q = queries(cache, hq, scale=40.0)  # the largest score takes it all
    start = torch.zeros(cache.k.shape[0], 1, 64, device=DEV)
    want, tol, lse = reference(cache, q, None, start, 1.0, scale=0.3)
    got = api.paged_weights(cache, q, lse, start.clone(), softmax_scale=0.3)
    assert (got.double() - want).abs().le(tol + 1e-9).all()


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
def test_against_the_attention_call(fp8):
    """The weights of each query sum up to one: of all of them, to their number."""
    cache = filled(batch([(1, 2000), (60, 900), (3, 0)], 16, 2, 128, fp8, values=True))
    cache.v.view(torch.uint8).zero_()
    q = queries(cache, 16)
    _, lse = api.paged_attn(cache, q)
    got = api.paged_weights(cache, q, lse, torch.zeros(cache.k.shape[0], 2, 16, device=DEV))
    # an lse is off by what the scores are (2^-16 of their size, some ten) and by its rounding
    assert abs(float(got.double().sum()) / (64 * 16) - 1) < 1e-3


@pytest.mark.gpu
def test_bad_pages_and_lengths_are_reported_and_left_out():
    cache = filled(batch([(1, 100), (1, 50), (40, 60)], 16, 2, 128, False, values=False))
    q = queries(cache, 16)
    start = torch.rand(cache.k.shape[0], 2, 16, device=DEV)
    want, tol, lse = reference(cache, q, None, start, 1.0)
    for bad in (-1, 10 ** 6):
        table = cache.page_table.clone()
        lost = int(table[0, 2])
        table[0, 2] = bad
        got = api.paged_weights(cache._replace(page_table=table), q, lse, start.clone())
        torch.cuda.synchronize()
        assert B.check_async_status()[0] != 0
        assert torch.equal(got[lost], start[lost])
        rest = torch.arange(got.shape[0], device=DEV) != lost
        assert (got.double() - want)[rest].abs().le((tol + 1e-9)[rest]).all()
    lens = cache.kv_lens.clone()
    lens[1] = 10 ** 6
    api.paged_weights(cache._replace(kv_lens=lens), q, lse, start.clone())
    torch.cuda.synchronize()
    assert B.check_async_status()[0] != 0
    assert B.check_async_status() == (0, 0)


def cache_struct(**other):
    at = ctypes.c_void_p(4096)
    fields = dict(k=at, v=at, page_table=at, kv_lens=at, cu_q=at, batch=2, max_pages=3, n_pages=9, page_size=16, n_kv_heads=2,
                  head_dim=128, fp8=0, max_new=0)
    fields.update(other)
    return B.MsaPagedCache(**fields)


def test_refusals_without_a_launch():
    B.lib()
    call = B._fn("msa_paged_weights")
    c = cache_struct()

    def go(cache=c, q=4096, hq=8, lse=4096, n=2, scale=0.0, decay=1.0, w=4096):
        return call(ctypes.byref(cache) if cache is not None else None, q, hq, lse, n, scale, decay, w, None, 0, None)

    assert go(cache=None) == 1
    assert go(hq=7) == 1 and go(hq=0) == 1 and go(n=-1) == 1
    assert go(decay=-0.1) == 1 and go(decay=math.nan) == 1 and go(decay=math.inf) == 1 and go(scale=-1.0) == 1
    assert go(q=None) == 1 and go(q=4100) == 1 and go(lse=None) == 1 and go(lse=4097) == 1 and go(w=None) == 1 and go(w=4098) == 1
    assert go(hq=2048) == 2
    assert go(cache=cache_struct(head_dim=100)) == 2 and go(cache=cache_struct(fp8=2)) == 1 and go(cache=cache_struct(cu_q=None)) == 1
    assert go(n=0) == 0 and go(cache=cache_struct(batch=0)) == 0
    size = ctypes.c_size_t(0)
    assert B._fn("msa_paged_weights_workspace_bytes")(ctypes.byref(c), 8, ctypes.byref(size)) == 0
    assert B._fn("msa_paged_weights_workspace_bytes")(ctypes.byref(c), 7, ctypes.byref(size)) == 1


@pytest.mark.gpu
def test_refusals_of_tensors():
    cache = filled(batch([(1, 20), (2, 3)], 16, 2, 128, False, values=False))
    q = queries(cache, 4)
    lse, w = torch.zeros(3, 4, device=DEV), torch.zeros(cache.k.shape[0], 2, 16, device=DEV)
    for bad in (w.double(), w[:, :1], w.transpose(1, 2), w.cpu(), w[1:]):
        with pytest.raises(ValueError):
            api.paged_weights(cache, q, lse, bad)
    for bad in (lse.half(), lse[:2], lse.t(), lse.cpu()):
        with pytest.raises(ValueError):
            api.paged_weights(cache, q, bad, w)
    for bad in (q.float(), q[:, :, :64], q.cpu()):
        with pytest.raises(ValueError):
            api.paged_weights(cache, bad, lse, w)
    with pytest.raises(B.MsaError):
        api.paged_weights(cache, q, lse, w, decay=-1.0)
    with pytest.raises(ValueError):
        api.paged_weights(cache, q.clone().requires_grad_(), lse, w)
    assert (w == 0).all()
