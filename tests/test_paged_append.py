"""Appending to a paged cache: against a token-by-token restatement in 64 bits, and refusals.

Tolerances as for the rotation itself (test_norm_rope.py); an E4M3 store is off by at most half a step, 2^-4 of the
value, or half of the smallest subnormal, 2^-10.  Values that are not turned or normed are rounded directly."""

import ctypes
import math
import random

import pytest
import torch

from paper_2606_13392_b200 import api
from paper_2606_13392_b200 import binding as B
from test_norm_rope import turn

DEV = "cuda"


def batch(lens, page, heads, d, fp8, spare=2, seed=0, table_cols=None, values=True):
    """A cache of randomly placed pages for sequences of (new, old) tokens; old rows are random, the rest NaN."""
    r = random.Random(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    used = [-(-(n + c) // page) for n, c in lens]
    cols = max(used + [1]) if table_cols is None else table_cols
    order = list(range(sum(used) + spare))
    r.shuffle(order)
    table = torch.full((len(lens), cols), -7, dtype=torch.int32)
    at = 0
    for i, u in enumerate(used):
        table[i, :u] = torch.tensor(order[at:at + u], dtype=torch.int32)
        at += u
    shape = (len(order), page, heads, d)
    pools = []
    for _ in range(2 if values else 1):
        pool = torch.full(shape, math.nan, device=DEV)
        for i, (n, c) in enumerate(lens):
            for p in range(c):
                pool[int(table[i, p // page]), p % page] = torch.randn(heads, d, generator=g, device=DEV)
        pools.append(pool.to(torch.float8_e4m3fn if fp8 else torch.bfloat16))
    cu = torch.tensor([sum(n for n, _ in lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=DEV)
    kv = torch.tensor([n + c for n, c in lens], dtype=torch.int32, device=DEV)
    return api.PagedCache(pools[0], pools[1] if values else None, table.to(DEV), kv, cu)


def rows_of(n, heads, d, seed, scale=1.0, strided=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = (torch.randn(n, heads * d + 16, generator=g, device=DEV) * scale).bfloat16()
    return x[:, 8:8 + heads * d].unflatten(1, (heads, d)) if strided else x[:, :heads * d].unflatten(1, (heads, d)).contiguous()


CASES = [  # lens (new, old), page, q heads, kv heads, d, fp8, rot, interleaved, norm
    ([(1, 0)], 1, 4, 1, 128, False, 128, False, True),
    ([(1, 77), (1, 0), (1, 4095), (1, 64)], 64, 64, 8, 128, False, 64, False, True),
    ([(0, 9), (5, 0), (0, 0), (130, 31), (1, 15)], 16, 16, 4, 128, True, 128, True, True),
    ([(333, 5), (64, 64)], 7, 6, 3, 64, False, 32, False, False),
    ([(70, 1)], 48, 3, 1, 96, True, 96, True, True),
    ([(20, 500), (900, 0)], 128, 8, 8, 128, True, 16, False, True),
    ([(3, 2)] * 70, 4, 2, 1, 128, False, 0, False, True),
    ([(2, 1), (0, 3)] * 600, 4, 1, 1, 64, False, 64, True, False),   # more sequences than a search takes in one step
]


@pytest.mark.gpu
@pytest.mark.parametrize("lens,page,hq,hkv,d,fp8,rot,inter,norm", CASES)
def test_append(lens, page, hq, hkv, d, fp8, rot, inter, norm):
    cache = batch(lens, page, hkv, d, fp8)
    n = sum(x for x, _ in lens)
    extra = 5  # rows of a padded batch
    q, k, v = [rows_of(n + extra, h, d, s, 1.5) for s, h in ((1, hq), (2, hkv), (3, hkv))]
    wq, wk = [(1 + 0.3 * torch.randn(d, device=DEV)).bfloat16() if norm else None for _ in range(2)]
    freqs = api.rope_frequencies(rot, 1e6) if rot else None
    before = [p.clone() for p in (cache.k, cache.v)]
    q_out = torch.full((n + extra, hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
    api.paged_append(cache, k, v, q, api.Rope(freqs, inter, 1.25) if rot else None, wq, wk, 1e-5, q_out)
    assert B.check_async_status() == (0, 0)
    assert (q_out[n:] == 7).all()
    positions = torch.cat([torch.arange(c, c + x) for x, c in lens]).to(DEV)
    refs = [turn(x[:n].double(), None if w is None else w.double(), positions, freqs, inter, 1.25, 1e-5) for x, w in ((q, wq), (k, wk))]
    bound = lambda ref, eps, least: eps * ref.abs() + 2.0 ** -15 * ref.abs().amax(-1, keepdim=True) + least  # noqa: E731
    assert (q_out[:n].double() - refs[0]).abs().le(bound(refs[0], 2.0 ** -8, 0)).all()
    # the places of the new tokens, one by one
    places, i = [], 0
    table = cache.page_table.cpu()
    for s, (x, c) in enumerate(lens):
        places += [(int(table[s, p // page]), p % page) for p in range(c, c + x)]
    where = torch.tensor(places, device=DEV).reshape(-1, 2)
    for pool, old, ref in ((cache.k, before[0], refs[1]), (cache.v, before[1], v[:n].double())):
        got = pool.float()[where[:, 0], where[:, 1]].double()
        assert (got - ref).abs().le(bound(ref, 2.0 ** -4 if fp8 else 2.0 ** -8, 2.0 ** -10 if fp8 else 0)).all()
        untouched = torch.ones(pool.shape[:2], dtype=torch.bool, device=DEV)
        untouched[where[:, 0], where[:, 1]] = False
        assert torch.equal(pool.view(torch.uint8)[untouched], old.view(torch.uint8)[untouched])
    # values are stored as they are, rounded once
    assert torch.equal(cache.v.view(torch.uint8).reshape(cache.v.shape[:3] + (-1,))[where[:, 0], where[:, 1]],
                       v[:n].to(cache.v.dtype).view(torch.uint8).reshape(n, hkv, -1))


@pytest.mark.gpu
def test_the_largest_e4m3_value_and_keys_without_values_or_queries():
    cache = batch([(2, 0)], 16, 1, 64, True, values=False)
    k = torch.full((2, 1, 64), 1000.0, dtype=torch.bfloat16, device=DEV)
    k[1] = -math.inf
    assert api.paged_append(cache, k, None) is None
    rows = cache.k[int(cache.page_table[0, 0])].float()
    assert (rows[0] == 448).all() and (rows[1] == -448).all() and rows[2:].isnan().all()


@pytest.mark.gpu
def test_places_that_are_not_there_are_reported_and_left():
    # a page outside the pool, a length beyond the table, more new tokens than the length: nothing is written for them
    # (the kernel looks a place up, checks it against the pool and skips the store), the query still is
    for change in ("page", "negative page", "length", "front"):
        cache = batch([(3, 5), (2, 0)], 4, 2, 64, False)
        if change == "page":
            cache.page_table[0, 1] = cache.k.shape[0]
        elif change == "negative page":
            cache.page_table[0, 1] = -1
        elif change == "length":
            cache.kv_lens[0] = 4 * cache.page_table.shape[1] + 3
        else:
            cache.kv_lens[0] = 0
        old = cache.k.clone(), cache.v.clone()
        k, q = rows_of(5, 2, 64, 1), rows_of(5, 4, 64, 2)
        out = api.paged_append(cache, k, k, q)
        assert B.check_async_status()[0] == 6
        assert torch.equal(out, q)
        # the second sequence has its page, nothing else changed
        page = int(cache.page_table[1, 0])
        assert torch.equal(cache.k[page, :2], k[3:]) and torch.equal(cache.v[page, :2], k[3:])
        keep = torch.ones(cache.k.shape[:2], dtype=torch.bool, device=DEV)
        keep[page, :2] = False
        for new, was in zip((cache.k, cache.v), old):
            assert torch.equal(new.view(torch.int16)[keep], was.view(torch.int16)[keep])
    assert B.check_async_status() == (0, 0)


@pytest.mark.gpu
def test_graph_replay_follows_the_lengths():
    cache = batch([(1, 10), (1, 30)], 16, 2, 128, False)
    cache = cache._replace(page_table=torch.tensor([[0, 1, 2], [3, 4, 5]], dtype=torch.int32, device=DEV) % cache.k.shape[0])
    k, q = rows_of(2, 2, 128, 1), rows_of(2, 8, 128, 2)
    rope = api.Rope(api.rope_frequencies(128))
    api.paged_append(cache, k, k, q, rope)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = api.paged_append(cache, k, k, q, rope)
    cache.kv_lens.add_(1)
    graph.replay()
    torch.cuda.synchronize()
    positions = cache.kv_lens.long() - 1
    want, _ = api.qk_norm_rope(q, None, positions, rope)
    assert torch.equal(out, want)
    want, _ = api.qk_norm_rope(k, None, positions, rope)
    for s in range(2):
        p = int(positions[s])
        assert torch.equal(cache.k[int(cache.page_table[s, p // 16]), p % 16], want[s])


def test_refusals_of_the_abi():
    lib = B.lib()
    one = ctypes.c_void_p(256)  # non-null and aligned, never followed on these paths

    def call(n=5, x=one, ks=256, y=one, vs=256, q=None, hq=0, qo=None, rope=None, eps=1e-6, **c):
        c = dict(k=256, v=256, page_table=256, kv_lens=256, cu_q=256, batch=2, max_pages=3, n_pages=9, page_size=16, n_kv_heads=2,
                 head_dim=128, fp8=0) | c
        cache = B.MsaPagedCache(**c)
        return lib.msa_paged_append(ctypes.byref(cache), rope, q, B.c_i64(1024), B.c_i32(hq), None, x, B.c_i64(ks), None, y, B.c_i64(vs),
                                    B.c_i32(0), ctypes.c_float(eps), B.c_i64(n), qo, None)

    assert call(n=0) == 0 and call(batch=0) == 0
    for bad in (dict(n=-1), dict(n=1 << 31), dict(batch=-1), dict(page_size=0), dict(n_pages=-1), dict(max_pages=-1), dict(n_kv_heads=0),
                dict(fp8=2), dict(cu_q=None), dict(kv_lens=None), dict(page_table=None), dict(k=None), dict(k=264), dict(x=None), dict(y=None), dict(ks=255), dict(ks=128),
                dict(v=None), dict(vs=8), dict(hq=4), dict(hq=4, q=one), dict(eps=-1.0), dict(page_table=258), dict(hq=-1)):
        assert call(**bad) == 1, bad
    assert lib.msa_paged_append(None, None, None, B.c_i64(0), B.c_i32(0), None, one, B.c_i64(256), None, one, B.c_i64(256), B.c_i32(0),
                                ctypes.c_float(0), B.c_i64(1), None, None) == 1
    assert call(head_dim=100) == 2 and call(head_dim=264) == 2 and call(n_kv_heads=5000) == 2


@pytest.mark.gpu
def test_refusals_of_tensors():
    cache = batch([(2, 1)], 4, 2, 64, False)
    k = rows_of(2, 2, 64, 1)
    bad = [cache._replace(k=cache.k.float()), cache._replace(v=cache.v[:, :2]), cache._replace(v=None),
           cache._replace(kv_lens=cache.kv_lens.long()), cache._replace(cu_q=cache.cu_q[:1]), cache._replace(page_table=cache.page_table[0]),
           cache._replace(page_table=cache.page_table.cpu()), cache._replace(k=cache.k[:, ::2], v=cache.v[:, ::2])]
    for c in bad:
        with pytest.raises(ValueError):
            api.paged_append(c, k, k)
    for args in ((k[:, :1], k), (k, k[:1]), (k, None), (k.float(), k)):
        with pytest.raises(ValueError):
            api.paged_append(cache, *args)
