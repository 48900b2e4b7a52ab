"""The calls of a bounded cache at their edges: what is not a number, waits that run out, bad lengths and pages, settings out of
the ordinary.  References and tolerances are those of test_paged_weights.py."""

import math

import pytest
import torch

from paper_2606_13392_b200 import api
from paper_2606_13392_b200 import binding as B
from test_paged_append import batch
from test_paged_weights import filled, queries, reference

DEV = "cuda"
KERNELS = [  # new tokens, head size, fp8: single tokens, a few, many (tensor memory), head sizes without tensor cores
    (1, 128, False), (1, 128, True), (3, 128, False), (3, 128, True), (200, 128, False), (200, 128, True), (20, 64, False)]


@pytest.mark.gpu
@pytest.mark.parametrize("new,d,fp8", KERNELS)
@pytest.mark.parametrize("what", ["lse", "q"])
def test_a_row_that_is_not_a_number_shows_wherever_it_stands(new, d, fp8, what):
    """Token and head of every column that a product of rows has: the places that the token sees get no number, the rest stay right."""
    cache = filled(batch([(new, 300)], 16, 1, d, fp8, values=False))
    q = queries(cache, 8)
    start = torch.rand(cache.k.shape[0], 1, 16, device=DEV)
    want, tol, lse = reference(cache, q, None, start, 0.5)
    place = torch.arange(new + 300, device=DEV)
    at = (cache.page_table[0].long()[place // 16], 0, place % 16)
    for tok in sorted({0, 1, 2, 15, 16, 31, 100, new - 1} & set(range(new))):
        for head in range(8):
            q2, lse2 = q.clone(), lse.clone()
            if what == "q":
                q2[tok, head, 5] = math.nan
            else:
                lse2[tok, head] = math.nan
            got = api.paged_weights(cache, q2, lse2, start.clone(), 0.5)[at].double()
            sees = place <= 300 + tok
            assert got[sees].isnan().all(), (tok, head, int((~got[sees].isnan()).sum()))
            assert (got - want[at])[~sees].abs().le(tol[at][~sees]).all()
    assert B.check_async_status() == (0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("new", [1, 200])
def test_scores_far_above_the_lse_overflow(new):
    """2^x of any size, by whatever way: finite as long as it is, infinite beyond, nothing at minus infinity."""
    cache = filled(batch([(new, 40)], 16, 1, 128, False, values=False))
    q = queries(cache, 8)
    q.zero_()
    for x in (126.5, 127.25, 127.75, 200.0, math.inf, -126.0, -130.0, -200.0, -math.inf):
        lse = torch.full((new, 8), -x * math.log(2.0), device=DEV)
        if x == -math.inf:
            lse.fill_(math.inf)
        if x == math.inf:
            lse.fill_(-1e30)  # (minus infinity itself gives nothing)
        for head in range(8):
            one = torch.full_like(lse, math.inf)
            one[0, head] = lse[0, head]
            got = api.paged_weights(cache, q, one, torch.zeros(cache.k.shape[0], 1, 16, device=DEV), 1.0)
            value = got[int(cache.page_table[0, 0]), 0, 0].double().item()
            # x is made of two products in 32 bits: off by 2^-22 of itself, its power by as much again; below 2^-126 anything down to 0
            size = 2.0 ** x if abs(x) < 1000 else (math.inf if x > 0 else 0.0)
            if x >= 200:
                assert value == math.inf
            elif x <= -126:
                assert 0 <= value <= 2.0 ** -125
            else:
                assert abs(value / size - 1) < 1e-4, (x, head, value)


@pytest.mark.gpu
@pytest.mark.parametrize("new,d,fp8", KERNELS)
def test_a_row_whose_lse_is_minus_infinity_gives_nothing_whatever_it_holds(new, d, fp8):
    """Rows that are to be left out: their queries need not be numbers."""
    cache = filled(batch([(new, 300), (1, 40)], 16, 2, d, fp8, values=False))
    q = queries(cache, 16)
    start = torch.rand(cache.k.shape[0], 2, 16, device=DEV)
    _, _, lse = reference(cache, q, None, start, 0.5)
    g = torch.Generator(device=DEV).manual_seed(3)
    out = torch.rand(lse.shape, generator=g, device=DEV) < 0.3
    out[0, 3] = out[new - 1, :9] = True
    lse[out] = -math.inf
    want, tol, _ = reference(cache, q, lse, start, 0.5)
    for value in (math.nan, math.inf, -math.inf, 3e38):
        bad = q.clone()
        bad[out] = value
        got = api.paged_weights(cache, bad, lse, start.clone(), 0.5)
        assert (got.double() - want).abs().le(tol + 1e-9).all(), value
    assert B.check_async_status() == (0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens", [[(70, 700), (100, 90)], [(300, 5000), (1, 40), (64, 3000)]])
def test_a_wait_that_runs_out_leaves_weights_old_or_new(lens, fp8):
    """The pool holds sums of many steps: nothing half added is written to it."""
    cache = filled(batch(lens, 16, 2, 128, fp8, values=False))
    q = queries(cache, 16)
    start = torch.rand(cache.k.shape[0], 2, 16, device=DEV)
    _, _, lse = reference(cache, q, None, start, 1.0)
    want = api.paged_weights(cache, q, lse, start.clone(), 0.9)
    assert B.check_async_status() == (0, 0)
    try:
        B.msa_debug_set_wait(20000, 2000000)  # 10 us against a copy role that is 1 ms late
        got = api.paged_weights(cache, q, lse, start.clone(), 0.9)
        assert B.check_async_status()[0] == 5
    finally:
        B.msa_debug_set_wait(0, 0)
    assert ((got == start) | (got == want)).all()
    assert torch.equal(api.paged_weights(cache, q, lse, start.clone(), 0.9), want)
    assert B.check_async_status() == (0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [1, 5])
@pytest.mark.parametrize("length", [-4, 97, 10 ** 8])
def test_compact_reports_bad_lengths(heads, length):
    """Pages hold 96 places: a length beyond is cut down to them, one below zero to nothing."""
    cache = batch([(0, 96), (0, 70)], 16, heads, 128, False)
    lens = cache.kv_lens.clone()
    lens[0] = length
    keep = torch.full((2, heads, 4), -1, dtype=torch.int32, device=DEV)
    before = cache.k.view(torch.int16).clone()
    for places in ([], [2, 50, 95]):  # nothing to move, something
        for i, p in enumerate(places):
            keep[0, :, i] = p
        cache.k.view(torch.int16).copy_(before)
        api.paged_compact(cache._replace(kv_lens=lens), keep)
        torch.cuda.synchronize()
        assert B.check_async_status()[0] != 0, places
        want, table = before.clone(), cache.page_table[0].long()
        for i, p in enumerate(places if length > 0 else []):
            want[table[0], i] = before[table[p // 16], p % 16]
        assert torch.equal(cache.k.view(torch.int16), want)
    lens[0] = 96
    api.paged_compact(cache._replace(kv_lens=lens), keep)
    assert B.check_async_status() == (0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("entry", [-1, -2, -3, -2147483648, 2147483647])
@pytest.mark.parametrize("which", [0, 3])
def test_compact_reports_every_bad_page(entry, which):
    """The page that a token comes from, or goes to, whatever number stands there."""
    cache = batch([(0, 100)], 16, 2, 128, False)
    before = [p.view(torch.int16).clone() for p in (cache.k, cache.v)]
    bad = cache.page_table.clone()
    bad[0, which] = entry
    keep = torch.tensor([[[7, 50]] * 2], dtype=torch.int32, device=DEV)
    api.paged_compact(cache._replace(page_table=bad), keep)
    torch.cuda.synchronize()
    assert B.check_async_status()[0] != 0
    table = cache.page_table[0].long()
    for p, b in zip((cache.k, cache.v), before):
        want = b.clone()
        if which == 3:
            want[table[0], 0] = b[table[0], 7]
        assert torch.equal(p.view(torch.int16), want)


@pytest.mark.gpu
def test_whole_numbers_beyond_32_bits_mean_what_they_say():
    cache = batch([(0, 100), (0, 30)], 16, 2, 128, False, values=False)
    w = torch.rand(cache.k.shape[0], 2, 16, device=DEV)
    for many in (1 << 31, (1 << 32) + 3, 1 << 62):
        for sinks, recent in ((many, 4), (0, many), (many, many)):
            got, want = api.paged_keep(cache, w, 40, sinks, recent), api.paged_keep(cache, w, 40, min(sinks, 1000), min(recent, 1000))
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        for bad in (dict(sinks=-many), dict(recent=-many), dict(budget=-many)):
            with pytest.raises(B.MsaError):
                api.paged_keep(cache, w, **(dict(budget=40) | bad))


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hint", [1, 2, 5])
def test_a_hint_below_the_longest_changes_little(hint, fp8):
    cache = filled(batch([(1, 300), (45, 200), (6, 20), (0, 50)], 16, 2, 128, fp8, values=False))
    q = queries(cache, 16)
    start = torch.rand(cache.k.shape[0], 2, 16, device=DEV)
    want, tol, lse = reference(cache, q, None, start, 0.7)
    got = api.paged_weights(cache, q, lse, start.clone(), 0.7, max_new=hint)
    assert (got.double() - want).abs().le(tol + 1e-9).all() and B.check_async_status() == (0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[(1, 900), (1, 3000)], [(70, 700), (100, 90)]])
def test_weights_and_moves_on_a_given_stream(lens):
    """Their results, and that they run there: work that is queued on that stream comes first."""
    cache = filled(batch(lens, 16, 2, 128, False), 1)
    q = queries(cache, 16)
    start = torch.rand(cache.k.shape[0], 2, 16, device=DEV)
    _, _, lse = reference(cache, q, None, start, 0.7)
    places = (cache.page_table, cache.kv_lens, cache.cu_q)
    ws = B.alloc_workspace(B.msa_paged_weights_workspace_bytes(cache.k, 16), DEV)
    weights = api.paged_weights(cache, q, lse, start.clone(), 0.7)
    keep, _ = api.paged_keep(cache, weights, 64, 4, 8)
    k, v, w = cache.k.clone(), cache.v.clone(), weights.clone()
    api.paged_compact(cache._replace(k=k, v=v), keep, w)
    side = torch.cuda.Stream()
    late = [torch.zeros_like(t) for t in (start, cache.k, cache.v)]  # filled on the side stream, behind a long wait
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(40_000_000)
        for t, source in zip(late, (start, cache.k, cache.v)):
            t.view(torch.uint8).copy_(source.view(torch.uint8))
    B.msa_paged_weights(late[1], *places, q, lse, 0.0, 0.7, late[0], ws, stream=side)
    with torch.cuda.stream(side):
        seen = late[0].clone()
    B.msa_paged_compact(late[1], late[2], *places, keep, late[0], stream=side)
    torch.cuda.synchronize()
    assert torch.equal(seen, weights)
    for a, b in zip(late, (w, k, v)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert B.check_async_status() == (0, 0)
