"""Keeping a paged cache within a budget: the choice of the tokens that stay and their move, exactly."""

import ctypes
import math

import pytest
import torch

from paper_2606_13392_b200 import api
from paper_2606_13392_b200 import binding as B
from test_paged_append import batch
from test_paged_weights import cache_struct

DEV = "cuda"


def chosen(w, n, budget, sinks, recent):
    """Places that stay of weights w [n] (a list of floats), as a sorted list."""
    stay = min(n, budget)
    r = min(recent, stay)
    s = min(sinks, stay - r)
    middle = sorted(range(s, n - r), key=lambda p: (-(w[p] if w[p] == w[p] else -math.inf), w[p] != w[p], p))
    return sorted(list(range(s)) + middle[:stay - r - s] + list(range(n - r, n)))


def weights_of(cache, kind, seed=5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    pages, page, heads, _ = cache.k.shape
    w = torch.rand(pages, heads, page, generator=g, device=DEV)
    if kind == "ties":
        w = (w * 4).floor()
    elif kind == "equal":
        w.fill_(0.25)
    elif kind == "odd":  # negative ones, both zeros, infinities, not numbers
        r = torch.rand(w.shape, generator=g, device=DEV)
        w = torch.where(r < 0.3, -w, w)
        for i, v in enumerate((0.0, -0.0, math.inf, -math.inf, math.nan)):
            w = torch.where((r > 0.5 + 0.08 * i) & (r < 0.58 + 0.08 * i), torch.full_like(w, v), w)
    elif kind == "close":  # differ in the last bits only
        w = (1 + (w * 40).floor() * 2.0 ** -23).float()
    return w


def flat(cache, w, s, h):
    n = int(cache.kv_lens[s])
    return w[cache.page_table[s].long().clamp(min=0), h].flatten()[:n].tolist()


KEEP = [  # lengths, page, heads, budget, sinks, recent, kind
    ([0, 1, 2, 64, 65, 200], 16, 3, 64, 4, 8, "random"),
    ([300, 33, 97], 7, 2, 32, 0, 0, "random"),
    ([300, 33, 97, 31], 48, 2, 32, 1, 31, "ties"),
    ([300, 20], 4, 1, 16, 20, 0, "random"),     # sinks alone
    ([300, 20], 4, 1, 16, 3, 20, "random"),     # the last alone
    ([300, 20], 4, 1, 16, 10, 10, "random"),    # some of the first
    ([500, 129, 4096], 64, 2, 128, 4, 16, "equal"),
    ([500, 129, 3000], 64, 2, 128, 4, 16, "odd"),
    ([5000], 128, 1, 1111, 0, 100, "close"),
    ([700], 12, 2, 1, 0, 0, "random"),
    ([5000, 30000], 32, 2, 4095, 4, 255, "random"),
    ([20000], 1, 1, 19999, 0, 1, "ties"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("lens,page,heads,budget,sinks,recent,kind", KEEP)
def test_keep(lens, page, heads, budget, sinks, recent, kind):
    cache = batch([(0, 0)] * len(lens), page, heads, 128, False, values=False)
    used = [-(-n // page) for n in lens]
    order = torch.randperm(sum(used) + 2, generator=torch.Generator().manual_seed(1)).int()
    table = torch.full((len(lens), max(used + [1])), -5, dtype=torch.int32)
    at = 0
    for i, u in enumerate(used):
        table[i, :u] = order[at:at + u]
        at += u
    cache = cache._replace(k=torch.zeros(sum(used) + 2, page, heads, 128, dtype=torch.bfloat16, device=DEV), page_table=table.to(DEV),
                           kv_lens=torch.tensor(lens, dtype=torch.int32, device=DEV))
    w = weights_of(cache, kind)
    results = [api.paged_keep(cache, w, budget, sinks, recent)]
    if page % 4 == 0:  # the same values where no 16 bytes can be read at once
        shifted = torch.zeros(w.numel() + 1, device=DEV)[1:].view(w.shape)
        results.append(api.paged_keep(cache, shifted.copy_(w), budget, sinks, recent))
    assert B.check_async_status() == (0, 0)
    for keep, new in results:
        assert new.tolist() == [min(n, budget) for n in lens]
        got = keep.cpu()
        for s, n in enumerate(lens):
            for h in range(heads):
                want = chosen(flat(cache, w, s, h), n, budget, sinks, recent)
                assert got[s, h].tolist() == want + [-1] * (budget - len(want)), (s, h)


@pytest.mark.gpu
@pytest.mark.parametrize("length,budget", [(300007, 2048), (1000000, 16384), (140000, 139000)])
def test_keep_of_long_sequences(length, budget):
    page, heads = 64, 2
    used = -(-length // page)
    table = torch.randperm(used, device=DEV).int()[None]
    cache = api.PagedCache(torch.zeros(used, page, heads, 8, dtype=torch.bfloat16, device=DEV), None, table,
                           torch.tensor([length], dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV))
    w = (torch.rand(used, heads, page, device=DEV) * 5000).floor()  # ties by the dozen
    keep, new = api.paged_keep(cache, w, budget, 4, 100)
    assert new.tolist() == [budget]
    for h in range(heads):
        x = w[table[0].long(), h].flatten()[4:length - 100].double()
        best = torch.argsort(x, descending=True, stable=True)[:budget - 104] + 4
        want = torch.cat([torch.arange(4, device=DEV), best, torch.arange(length - 100, length, device=DEV)]).sort().values
        assert torch.equal(keep[0, h].long(), want)


MOVE = [  # lengths, page, heads, d, fp8, budget, sinks, recent, values
    ([0, 1, 64, 65, 200], 16, 3, 128, False, 64, 4, 8, True),
    ([300, 33, 97], 7, 2, 96, True, 32, 0, 0, True),
    ([1300, 20], 48, 1, 8, True, 500, 1, 31, False),
    ([700], 1, 2, 256, False, 650, 3, 20, True),
    ([5000, 4100], 64, 8, 128, False, 4096, 4, 64, True),
    ([5000, 300], 128, 2, 64, True, 4096, 4, 64, True),
    ([2600] * 40, 32, 8, 128, True, 2048, 0, 0, True),
    ([900], 24, 5, 40, False, 800, 0, 1, False),
]


@pytest.mark.gpu
@pytest.mark.parametrize("lens,page,heads,d,fp8,budget,sinks,recent,values", MOVE)
def test_compact(lens, page, heads, d, fp8, budget, sinks, recent, values):
    used = [-(-n // page) for n in lens]
    g = torch.Generator(device=DEV).manual_seed(2)
    pages = sum(used) + 2
    order = torch.randperm(pages, generator=g, device=DEV).int()
    table = torch.full((len(lens), max(used)), -5, dtype=torch.int32, device=DEV)
    at = 0
    for i, u in enumerate(used):
        table[i, :u] = order[at:at + u]
        at += u
    kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
    pools = [torch.randint(0, 256, (pages, page, heads, d * (1 if fp8 else 2)), generator=g, device=DEV, dtype=torch.uint8).view(kind)
             for _ in range(2)]
    cache = api.PagedCache(pools[0], pools[1] if values else None, table, torch.tensor(lens, dtype=torch.int32, device=DEV),
                           torch.zeros(len(lens) + 1, dtype=torch.int32, device=DEV))
    w = torch.rand(pages, heads, page, generator=g, device=DEV)
    keep, new = api.paged_keep(cache, w, budget, sinks, recent)
    want = [p.view(torch.uint8).clone() for p in pools]
    want_w = w.clone()
    for s in range(len(lens)):
        for h in range(heads):
            src = keep[s, h][keep[s, h] >= 0].long()
            dst = torch.arange(len(src), device=DEV)
            t = table[s].long()
            for p in want[:2 if values else 1]:
                p[t[dst // page], dst % page, h] = p[t[src // page], src % page, h].clone()
            want_w[t[dst // page], h, dst % page] = want_w[t[src // page], h, src % page].clone()
    with_weights = values
    api.paged_compact(cache, keep, w if with_weights else None)
    assert B.check_async_status() == (0, 0)
    assert torch.equal(pools[0].view(torch.uint8), want[0]) and torch.equal(pools[1].view(torch.uint8), want[1])
    if with_weights:
        assert torch.equal(w, want_w)


@pytest.mark.gpu
def test_compact_reports_bad_lists_and_moves_the_rest():
    cache = batch([(0, 100), (0, 70)], 16, 1, 128, False)
    before = [p.view(torch.int16).clone() for p in (cache.k, cache.v)]
    table = cache.page_table.long()
    for entry in (100, 10 ** 9, 0):  # behind the end, far behind it, in front of its own place
        keep = torch.full((2, 1, 4), -1, dtype=torch.int32, device=DEV)
        keep[0, 0, :4] = torch.tensor([0, 50, entry, 60])
        for p, b in zip((cache.k, cache.v), before):
            p.view(torch.int16).copy_(b)
        api.paged_compact(cache, keep)
        torch.cuda.synchronize()
        assert B.check_async_status()[0] != 0
        for p, b in zip((cache.k, cache.v), before):
            want = b.clone()
            for to, place in ((1, 50), (3, 60)):
                want[table[0, 0], to, 0] = b[table[0, place // 16], place % 16, 0]
            assert torch.equal(p.view(torch.int16), want)
    # a bad page holds nothing and takes nothing
    bad = cache.page_table.clone()
    bad[0, 3] = 77777
    keep = torch.full((2, 1, 2), -1, dtype=torch.int32, device=DEV)
    keep[0, 0, 1] = 50
    for p, b in zip((cache.k, cache.v), before):
        p.view(torch.int16).copy_(b)
    api.paged_compact(cache._replace(page_table=bad), keep)
    torch.cuda.synchronize()
    assert B.check_async_status()[0] != 0
    assert all(torch.equal(p.view(torch.int16), b) for p, b in zip((cache.k, cache.v), before))


@pytest.mark.gpu
def test_keep_reports_bad_pages_and_lengths():
    cache = batch([(0, 100), (0, 70)], 16, 1, 128, False, values=False)
    w = torch.rand(cache.k.shape[0], 1, 16, device=DEV)
    bad = cache.page_table.clone()
    bad[0, 3] = 77777
    keep, new = api.paged_keep(cache._replace(page_table=bad), w, 20)
    torch.cuda.synchronize()
    assert B.check_async_status()[0] != 0
    x = flat(cache, w, 0, 0)
    x[48:64] = [math.nan] * 16
    assert keep[0, 0].tolist() == chosen(x, 100, 20, 0, 0) and keep[1, 0].tolist() == chosen(flat(cache, w, 1, 0), 70, 20, 0, 0)
    lens = cache.kv_lens.clone()
    lens[0], lens[1] = -4, 10 ** 8
    keep, new = api.paged_keep(cache._replace(kv_lens=lens), w, 500)
    torch.cuda.synchronize()
    assert B.check_async_status()[0] != 0
    assert new.tolist() == [0, cache.page_table.shape[1] * 16]
    assert B.check_async_status() == (0, 0)


def test_refusals_without_a_launch():
    B.lib()
    c = cache_struct()
    keep, compact = B._fn("msa_paged_keep"), B._fn("msa_paged_compact")

    def k(cache=c, w=4096, budget=4, sinks=0, recent=0, to=4096, lens=8192):
        return keep(ctypes.byref(cache) if cache is not None else None, w, budget, sinks, recent, to, lens, None)

    assert k(cache=None) == 1 and k(w=None) == 1 and k(w=4097) == 1 and k(to=None) == 1 and k(to=4098) == 1 and k(lens=4097) == 1
    assert k(budget=0) == 1 and k(sinks=-1) == 1 and k(recent=-1) == 1 and k(budget=(1 << 30) + 1) == 2
    assert k(lens=4096) == 1  # (the old lengths are still read)
    assert k(cache=cache_struct(kv_lens=None)) == 1 and k(cache=cache_struct(page_table=None)) == 1
    assert k(cache=cache_struct(n_kv_heads=5000)) == 2 and k(cache=cache_struct(page_size=0)) == 1
    assert k(cache=cache_struct(batch=0)) == 0

    def m(cache=c, at=4096, width=4, w=4096):
        return compact(ctypes.byref(cache) if cache is not None else None, at, width, w, None)

    assert m(cache=None) == 1 and m(at=None) == 1 and m(at=4097) == 1 and m(w=4098) == 1 and m(width=-1) == 1
    assert m(cache=cache_struct(k=None)) == 1 and m(cache=cache_struct(k=4100)) == 1 and m(cache=cache_struct(v=4100)) == 1
    assert m(width=(1 << 30) + 1) == 2
    assert m(width=0) == 0 and m(cache=cache_struct(batch=0)) == 0


@pytest.mark.gpu
def test_refusals_of_tensors():
    cache = batch([(0, 100), (0, 70)], 16, 2, 128, False)
    w = torch.rand(cache.k.shape[0], 2, 16, device=DEV)
    for bad in (w.half(), w[:, :1], w.cpu(), w.transpose(0, 1)):
        with pytest.raises(ValueError):
            api.paged_keep(cache, bad, 10)
        with pytest.raises(ValueError):
            api.paged_compact(cache, torch.zeros(2, 2, 3, dtype=torch.int32, device=DEV), bad)
    for budget, sinks, recent in ((0, 0, 0), (-3, 0, 0), (4, -1, 0), (4, 0, -1)):
        with pytest.raises(B.MsaError):
            api.paged_keep(cache, w, budget, sinks, recent)
    keep = torch.zeros(2, 2, 3, dtype=torch.int32, device=DEV)
    for bad in (keep.long(), keep[:1], keep[:, :1], keep.cpu(), keep.transpose(1, 2), keep[:, :, 0]):
        with pytest.raises(ValueError):
            api.paged_compact(cache, bad)
