"""Attention of new tokens over a paged cache against the definition in 64 bits, sequence by sequence.

Tolerances (per row; A = sum_j p_j |v_j|, the largest the sum's terms can be).  Scores are fp32 sums of d exact
products: off by at most d steps of 2^-24 of sum |q_i k_i|, and the scaled maximum that is subtracted by 2^-23 of
itself; a probability is off by that factor, delta.  The tensor-core kernel rounds P to bf16 (half a step, 2^-8 of the
value) before P V, sums in fp32 (2^-14 of A is over 500 steps), and the result is rounded to bf16 once:
    |out - ref| <= 2^-8 |ref| + (2^-8 + 2 delta + 2^-14) A
On fp8 caches P is rounded to fp16 instead, held 2^10 up: half a step is 2^-11 of the value or, among its subnormal
numbers, 2^-25, that is 2^-35 of the row's largest probability (which is at least that of its reference maximum, so the
sum it is divided by is no smaller): where the large probabilities meet values that are exactly zero, A does not cover
that, and 2^-35 sum_j |v_j| is added.
    |lse - ref| <= delta + 2^-15 + 2^-21 |ref|        (the sum of p: at most 500 additions; its logarithm)"""

import ctypes
import math
import random

import pytest
import torch

from paper_2606_13392_b200 import api
from paper_2606_13392_b200 import binding as B

DEV = "cuda"


def make(lens, page, heads, d, fp8, seed=0, spare=2, extra_cols=1):
    """Sequences of (new, old) tokens on randomly placed pages; what lies behind a sequence's end, in pages no sequence
    has and in unused columns of the table is NaN or not a page."""
    r = random.Random(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    used = [-(-(n + c) // page) for n, c in lens]
    order = list(range(sum(used) + spare))
    r.shuffle(order)
    table = torch.full((len(lens), max(used + [0]) + extra_cols), -7, dtype=torch.int32)
    pools = [torch.full((len(order), page, heads, d), math.nan, device=DEV, dtype=torch.bfloat16) for _ in range(2)]
    at = 0
    for i, u in enumerate(used):
        mine = order[at:at + u]
        table[i, :u] = torch.tensor(mine, dtype=torch.int32)
        at += u
        n = sum(lens[i])
        where = torch.tensor([p * page + t for p in mine for t in range(page)][:n], dtype=torch.int64, device=DEV)
        for pool in pools:
            pool.view(-1, heads, d)[where] = torch.randn(n, heads, d, generator=g, device=DEV).bfloat16()
    kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
    cu = torch.tensor([sum(n for n, _ in lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=DEV)
    kv = torch.tensor([n + c for n, c in lens], dtype=torch.int32, device=DEV)
    return api.PagedCache(pools[0].to(kind), pools[1].to(kind), table.to(DEV), kv, cu)


def gathered(pool, table_row, n):
    page = pool.shape[1]
    t = torch.arange(n, device=DEV)
    raw = pool.view(torch.uint8)[table_row.long()[t // page], t % page]  # (as bytes: pools may be large)
    return raw.view(pool.dtype).double()


def check(cache, q, out, lse, scale=None):
    """Every row against the definition."""
    cu, kv = cache.cu_q.tolist(), cache.kv_lens.tolist()
    hkv, d = cache.k.shape[2:]
    group = q.shape[1] // hkv
    scale = d ** -0.5 if scale is None else scale
    for s in range(len(kv)):
        rows = slice(cu[s], cu[s + 1])
        n = cu[s + 1] - cu[s]
        if n == 0:
            continue
        k, v = gathered(cache.k, cache.page_table[s], kv[s]), gathered(cache.v, cache.page_table[s], kv[s])
        hidden = torch.arange(kv[s], device=DEV) > torch.arange(kv[s] - n, kv[s], device=DEV)[:, None]
        for h in range(hkv):
            heads = slice(h * group, (h + 1) * group)
            x = q[rows, heads].double()                                   # [n, G, d]
            logit = (x @ k[:, h].T * scale).masked_fill(hidden[:, None], -math.inf)
            p = torch.softmax(logit, -1).nan_to_num(0.0)                  # rows that see nothing: zeros
            ref, size = p @ v[:, h], p @ v[:, h].abs()
            ref_lse = torch.logsumexp(logit, -1)
            most = (x.abs() @ k[:, h].abs().T * scale).masked_fill(hidden[:, None], 0.0).amax(-1) if kv[s] else torch.zeros_like(ref_lse)
            delta = d * 2.0 ** -24 * most + 2.0 ** -23 * most
            tol = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2 * delta[..., None] + 2.0 ** -14) * size
            if cache.k.dtype == torch.float8_e4m3fn:
                tol = tol + 2.0 ** -35 * v[:, h].abs().sum(0)
            err = (out[rows, heads].double() - ref).abs()
            assert err.le(tol).all(), (s, h, float((err - tol).max()))
            if lse is not None:
                empty = hidden.all(-1)[:, None].expand_as(ref_lse)
                assert (lse[rows, heads][empty] == -math.inf).all()
                off = (lse[rows, heads].double() - ref_lse).abs()[~empty]
                assert off.le((delta + 2.0 ** -15 + 2.0 ** -21 * ref_lse.abs())[~empty]).all(), (s, h, float(off.max()))


def queries(n, heads, d, seed=1, scale=2.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (scale * torch.randn(n, heads, d, generator=g, device=DEV)).bfloat16()


CASES = [  # lens (new, old), page, query heads per KV head, KV heads, d, fp8
    ([(1, 0)], 64, 8, 1, 128, False),                                  # one token that sees itself
    ([(1, 126)], 64, 8, 2, 128, False),                                # one short of a tile
    ([(1, 127)], 16, 16, 1, 128, False),
    ([(1, 128)], 128, 8, 1, 128, True),
    ([(1, 2046)], 64, 8, 8, 128, False),                               # one sequence cut over many CTAs
    ([(1, 5000), (1, 3), (1, 0), (1, 777), (1, 12345)], 64, 8, 4, 128, False),
    ([(1, 5000), (1, 3), (1, 0), (1, 777), (1, 12345)], 128, 16, 4, 128, True),
    ([(1, 300 + 7 * i) for i in range(70)], 32, 16, 2, 128, False),
    ([(1, 300 + 7 * i) for i in range(70)], 32, 16, 2, 128, True),
    ([(1, 2046)], 64, 8, 8, 128, True),
    ([(1, 9000), (1, 0), (0, 70), (1, 127)], 16, 1, 2, 128, True),
    ([(1, 500), (1, 129), (1, 128)], 48, 5, 3, 128, True),
    ([(1, 500), (1, 129), (1, 4000)], 256, 12, 2, 128, True),
    ([(3, 40), (0, 9), (2, 700), (0, 0), (0, 3)], 24, 4, 2, 128, True),   # no more tokens than sequences, not one each
    ([(5, 300)] + [(0, 4)] * 4, 64, 16, 1, 128, True),
    ([(3, 40), (0, 9), (7, 1000), (16, 0), (1, 64), (0, 0), (17, 512)], 16, 8, 2, 128, False),
    ([(3, 40), (0, 9), (7, 1000), (16, 0), (1, 64), (0, 0), (17, 512)], 48, 8, 2, 128, True),
    ([(1 + i % 3 // 2, i % 150) for i in range(700)], 16, 8, 1, 128, False),   # more sequences than threads
    ([(1, i % 150) for i in range(700)], 16, 8, 1, 128, True),
    ([(32, 0)], 64, 8, 1, 128, False),                                 # both contexts full
    ([(33, 0)], 64, 8, 1, 128, False),                                 # and one token more
    ([(1000, 0)], 64, 8, 2, 128, False),
    ([(513, 2000)], 256, 16, 1, 128, False),
    ([(200, 3000), (1, 9000), (90, 90), (31, 4)], 64, 4, 2, 128, True),
    ([(129, 1), (5, 130)], 8, 1, 3, 128, False),
    ([(40, 400), (2, 70)], 24, 5, 2, 128, False),                      # groups that do not divide a tile
    ([(9, 400), (3, 70)], 64, 100, 1, 128, False),
    ([(80, 90000)], 64, 8, 1, 128, False),                             # several tiles on keys beyond a third of L2
    ([(80, 170000)], 128, 8, 1, 128, True),
    ([(2, 3000), (1, 300), (3, 70), (2, 5)], 16, 8, 2, 128, True),     # two tokens of eight heads on average
    ([(9, 3000), (1, 300), (0, 70), (1, 5)], 32, 4, 2, 128, True),
    ([(9, 400), (130, 70)], 64, 128, 1, 128, True),
    ([(300, 7)], 64, 3, 2, 128, True),
    ([(4, 60), (1, 0), (0, 3)], 7, 4, 2, 128, False),                  # other shapes: odd pages,
    ([(4, 60), (20, 0)], 16, 2, 2, 64, True),                          # other head sizes,
    ([(3, 50)], 1, 3, 1, 256, False),
    ([(3, 50), (1, 1)], 16, 7, 2, 40, False),
    ([(2, 33)], 16, 160, 1, 128, False),                               # other groups
]


@pytest.mark.gpu
@pytest.mark.parametrize("lens,page,group,hkv,d,fp8", CASES)
def test_attention(lens, page, group, hkv, d, fp8):
    cache = make(lens, page, hkv, d, fp8)
    n, extra = sum(x for x, _ in lens), 3
    q = queries(n + extra, group * hkv, d)
    out = torch.full_like(q, 5.0)
    got, lse = api.paged_attn(cache, q, out=out)
    assert got is out and B.check_async_status() == (0, 0)
    assert (out[n:] == 5).all()  # rows of a padded batch
    check(cache, q, out, lse)
    again, lse2 = api.paged_attn(cache, q)
    assert torch.equal(again[:n], out[:n]) and torch.equal(lse[:n], lse2[:n])
    no_lse, none = api.paged_attn(cache, q, want_lse=False)
    assert none is None and torch.equal(no_lse[:n], out[:n])
    assert B.check_async_status() == (0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("seed", range(6))
def test_random_batches(seed, fp8):
    r = random.Random(seed)
    top = r.choice([200, 2000, 12000])
    lens = [(r.choice([0, 1, 1, 2, 5, 16, 17, 60, 300]), r.randint(0, top)) for _ in range(r.randint(1, 12))]
    if not any(n for n, _ in lens):
        lens.append((1, 5))
    page, group, hkv = r.choice([8, 16, 40, 64, 128, 192]), r.choice([1, 2, 4, 8, 16, 6]), r.choice([1, 2, 4])
    cache = make(lens, page, hkv, 128, fp8, seed)
    q = queries(sum(n for n, _ in lens), group * hkv, 128, seed)
    out, lse = api.paged_attn(cache, q, 0.11)
    assert B.check_async_status() == (0, 0)
    check(cache, q, out, lse, 0.11)


@pytest.mark.gpu
@pytest.mark.parametrize("d,page", [(128, 16), (64, 16)])
def test_rows_that_see_nothing(d, page):
    # more new tokens than the sequence has: the first ones stand in front of position 0
    cache = make([(6, 0), (1, 4), (40, 0)], page, 2, d, False)
    cache.kv_lens.copy_(torch.tensor([2, 0, 7], dtype=torch.int32))
    q = queries(47, 16, d)
    out, lse = api.paged_attn(cache, q)
    assert (out[:4] == 0).all() and (lse[:4] == -math.inf).all()
    assert (out[6] == 0).all() and (lse[6] == -math.inf).all()
    assert (out[7:40] == 0).all() and (lse[7:40] == -math.inf).all()
    assert lse[4:6].isfinite().all() and lse[40:].isfinite().all()
    check(cache, q, out, lse)
    assert B.check_async_status() == (0, 0)


@pytest.mark.gpu
def test_growing_maxima_and_large_scores():
    # scores that grow along the keys make the running maximum move in every tile; scores far beyond the range of fp16 exponents stay exact
    cache = make([(1, 2000), (50, 1500)], 64, 2, 128, False)
    ramp = torch.linspace(0.01, 6.0, 3000, device=DEV)
    for s, n in ((0, 2001), (1, 1550)):
        t = torch.arange(n, device=DEV)
        where = cache.page_table[s].long()[t // 64], t % 64
        cache.k[where] = (ramp[:n, None, None] * (1 + 0.1 * torch.randn(n, 2, 128, device=DEV))).bfloat16()
    q = queries(51, 16, 128).abs()
    out, lse = api.paged_attn(cache, q)
    assert lse.max() > 80
    check(cache, q, out, lse)
    falling = cache._replace(k=cache.k.neg())
    out, lse = api.paged_attn(falling, q)
    check(falling, q, out, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
def test_queries_of_any_size(fp8):
    # rows of one tile that are powers of two apart, beyond what fp16 holds (fp8 caches multiply in fp16)
    for lens in ([(3, 900), (60, 300)], [(1, 900), (1, 300)]):
        cache = make(lens, 16, 2, 128, fp8)
        n = sum(x for x, _ in lens)
        q = queries(n, 16, 128)
        size = torch.tensor([2.0 ** e for e in (-140, -100, -40, -17, 0, 12, 17, 30)], device=DEV).repeat(n * 2).view(n, 16, 1)
        q = (q.float() * size).bfloat16()
        for scale in (2.0 ** -21, 2.0 ** -34):
            out, lse = api.paged_attn(cache, q, scale)
            check(cache, q, out, lse, scale)


@pytest.mark.gpu
@pytest.mark.parametrize("lens,fp8", [([(1, 700), (1, 90)], False), ([(70, 700), (1, 3000)], False), ([(1, 700), (1, 90)], True)])
def test_graphs_and_streams(lens, fp8):
    cache = make(lens, 16, 2, 128, fp8)
    n = sum(x for x, _ in lens)
    q = queries(n, 16, 128)
    want = api.paged_attn(cache, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = api.paged_attn(cache, q)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = api.paged_attn(cache, q)
    # a replay follows lengths, tables, queries
    cache.kv_lens.sub_(5)
    q.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    check(cache, q, out, lse)
    want = api.paged_attn(cache, q)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    # two calls in flight on two streams have a workspace each
    other = make(lens, 16, 2, 128, fp8, seed=9)
    with torch.cuda.stream(side):
        a = [api.paged_attn(other, q) for _ in range(5)]
    b = [api.paged_attn(cache, q) for _ in range(5)]
    torch.cuda.synchronize()
    check(other, q, *a[-1])
    assert all(torch.equal(x[0], want[0]) for x in b) and all(torch.equal(x[0], a[0][0]) for x in a)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [128, 64])
def test_bad_pages_and_lengths_are_reported(d):
    # the kernels check a page against the pool before they form an address, and a length against the table; the other
    # sequences' results stay right
    for change, fp8 in [(c, f) for c in ("page", "negative page", "length", "negative length") for f in (False, True)]:
        cache = make([(2, 500), (1, 300)] + [(0, 1)] * fp8, 16, 1, d, fp8)
        if change == "page":
            cache.page_table[0, 3] = cache.k.shape[0]
        elif change == "negative page":
            cache.page_table[0, 0] = -(1 << 31)
        elif change == "length":
            cache.kv_lens[0] = (1 << 31) - 1
        else:
            cache.kv_lens[0] = -4
        q = queries(3, 8, d)
        out, lse = api.paged_attn(cache, q)
        assert B.check_async_status()[0] == 6, change
        rest = api.PagedCache(cache.k, cache.v, cache.page_table[1:2].contiguous(), cache.kv_lens[1:2].clone(),
                              torch.tensor([0, 1], dtype=torch.int32, device=DEV))
        check(rest, q[2:], out[2:], lse[2:])
    assert B.check_async_status() == (0, 0)


@pytest.mark.gpu
def test_guard_bands():
    lens = [(70, 700), (1, 3000), (3, 4)]
    cache = make(lens, 16, 2, 128, False)
    q = queries(74, 16, 128)
    need = B.msa_paged_attn_workspace_bytes(cache.k, 16)
    raw = torch.full((need + 8192,), 0xCD, dtype=torch.uint8, device=DEV)
    outs = torch.full((74 + 2, 16, 128), 3.0, dtype=torch.bfloat16, device=DEV)
    out, lse = api.paged_attn(cache, q, out=outs[1:75], workspace=raw[4096:4096 + need])
    check(cache, q, out, lse)
    assert (raw[:4096] == 0xCD).all() and (raw[4096 + need:] == 0xCD).all() and (outs[0] == 3).all() and (outs[75] == 3).all()


@pytest.mark.gpu
@pytest.mark.parametrize("lens,fp8", [([(70, 200), (1, 400)], False), ([(70, 200), (1, 400)], True), ([(1, 200), (1, 400)], True)])
def test_operands_on_16_byte_boundaries(lens, fp8):
    cache = make(lens, 16, 2, 128, fp8)
    n = sum(x for x, _ in lens)
    q = queries(n, 16, 128)
    want, lse = api.paged_attn(cache, q)
    buffers = [torch.zeros(n * 16 * 128 + 8, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    moved, out = [b[8:].view(n, 16, 128) for b in buffers]
    moved.copy_(q)
    assert moved.data_ptr() % 32 == 16 and out.data_ptr() % 32 == 16
    got, lse2 = api.paged_attn(cache, moved, out=out)
    assert torch.equal(got, want) and torch.equal(lse, lse2)
    check(cache, q, got, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("lens,fp8", [([(40, 3000), (1, 900)], False), ([(40, 3000), (1, 900)], True), ([(1, 3000), (1, 900)], True)])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right(lens, fp8):
    cache = make(lens, 16, 2, 128, fp8)
    q = queries(sum(n for n, _ in lens), 16, 128)
    try:
        B.msa_debug_set_wait(20000, 2000000)  # 10 us against a copy role that is 1 ms late
        api.paged_attn(cache, q)
        assert B.check_async_status()[0] == 5
    finally:
        B.msa_debug_set_wait(0, 0)
    out, lse = api.paged_attn(cache, q)
    assert B.check_async_status() == (0, 0)
    check(cache, q, out, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
def test_a_layer_step_by_step(fp8):
    """Norm and rotation, append, attention as a serving loop runs them: a prompt in chunks, then single tokens, against
    one dense pass in 64 bits over all tokens' rotated keys as the cache holds them."""
    hq, hkv, d, page, total = 16, 2, 128, 16, 300
    g = torch.Generator(device=DEV).manual_seed(3)
    qkv = torch.randn(2, total, (hq + 2 * hkv) * d, generator=g, device=DEV).bfloat16()
    wq, wk = [(1 + 0.2 * torch.randn(d, generator=g, device=DEV)).bfloat16() for _ in range(2)]
    rope = api.Rope(api.rope_frequencies(64, 1e5))
    kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
    pools = [torch.full((44, page, hkv, d), math.nan, device=DEV).to(kind) for _ in range(2)]
    table = torch.randperm(44, generator=g, device=DEV)[:42].to(torch.int32).view(2, 21)
    done = [0, 0]
    outs = [[], []]
    turned = [[], []]
    for step in [(130, 40), (0, 200), (100, 59)] + [(1, 1)] * 1 + [(69, 0)]:
        rows = torch.cat([qkv[s, done[s]:done[s] + step[s]] for s in range(2)])
        q, k, v = [x.unflatten(1, (-1, d)) for x in rows.split([hq * d, hkv * d, hkv * d], 1)]
        done = [done[s] + step[s] for s in range(2)]
        cache = api.PagedCache(pools[0], pools[1], table, torch.tensor(done, dtype=torch.int32, device=DEV),
                               torch.tensor([0, step[0], step[0] + step[1]], dtype=torch.int32, device=DEV))
        q = api.paged_append(cache, k, v, q, rope, wq, wk)
        out, lse = api.paged_attn(cache, q)
        check(cache, q, out, lse)
        for s in range(2):
            at = slice(0, step[0]) if s == 0 else slice(step[0], None)
            outs[s].append(out[at])
            turned[s].append(q[at])
    assert done == [total, total] and B.check_async_status() == (0, 0)
    for s in range(2):  # all at once
        one = cache._replace(page_table=table[s:s + 1], kv_lens=cache.kv_lens[s:s + 1],
                             cu_q=torch.tensor([0, total], dtype=torch.int32, device=DEV))
        check(one, torch.cat(turned[s]), torch.cat(outs[s]), None)
        rows = qkv[s].split([hq * d, hkv * d, hkv * d], 1)
        q, k = api.qk_norm_rope(rows[0].unflatten(1, (-1, d)), rows[1].unflatten(1, (-1, d)), torch.arange(total, device=DEV), rope, wq, wk)
        assert torch.equal(q, torch.cat(turned[s]))
        if not fp8:
            assert torch.equal(gathered(cache.k, table[s], total), k.double())


@pytest.mark.gpu
@pytest.mark.parametrize("fp8,lens", [(False, [(70, 900), (1, 400)]), (True, [(70, 900), (1, 400)]), (True, [(1, 900), (1, 400)])])
def test_places_beyond_32_bits(fp8, lens):
    # the last pages of a pool of over 2^31 elements, written by the append and read back
    page, heads, d = 64, 8, 128
    pages = (1 << 31) // (page * heads * d) + 40
    kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
    pools = [torch.empty(pages, page, heads, d, dtype=kind, device=DEV) for _ in range(2)]
    table = torch.arange(pages - 40, pages, dtype=torch.int32, device=DEV).flip(0).view(2, 20)  # 1280 tokens each
    g = torch.Generator(device=DEV).manual_seed(1)
    for n in ([c for _, c in lens], [x for x, _ in lens]):  # what was there, then the new tokens
        done = [c for _, c in lens] if n[0] == lens[0][1] else [x + c for x, c in lens]
        cache = api.PagedCache(pools[0], pools[1], table, torch.tensor(done, dtype=torch.int32, device=DEV),
                               torch.tensor([0, n[0], sum(n)], dtype=torch.int32, device=DEV))
        k, v = [torch.randn(sum(n), heads, d, generator=g, device=DEV).bfloat16() for _ in range(2)]
        api.paged_append(cache, k, v)
        for s in range(2):
            rows = slice(0, n[0]) if s == 0 else slice(n[0], None)
            assert torch.equal(gathered(cache.k, table[s], done[s])[done[s] - n[s]:], k[rows].to(kind).double())
            assert torch.equal(gathered(cache.v, table[s], done[s])[done[s] - n[s]:], v[rows].to(kind).double())
    q = queries(sum(n), 16, d)
    out, lse = api.paged_attn(cache, q)
    assert B.check_async_status() == (0, 0)
    check(cache, q, out, lse)


@pytest.mark.gpu
def test_the_sparse_path_reads_the_same_pool_and_agrees_where_every_block_fits():
    """Pages in order are the packed cache of msa_sparse_attn_decode, and with k * B_k >= context its result is the dense
    one: the same call on the same pool."""
    from paper_2606_13392_b200.inputs import MSAConfig
    lens = [1000, 2048]
    cfg = MSAConfig("paged", "decode", max(lens), 16, 2, 128, 16, seq_lens=tuple(lens))
    page, hkv, d = 64, 2, 128
    g = torch.Generator(device=DEV).manual_seed(0)
    pools = [torch.randn(16 + 32, page, hkv, d, generator=g, device=DEV).bfloat16() for _ in range(2)]
    table = torch.zeros(2, 32, dtype=torch.int32, device=DEV)
    table[0, :16], table[1] = torch.arange(16), torch.arange(16, 48)
    kv = torch.tensor(lens, dtype=torch.int32, device=DEV)
    cache = api.PagedCache(pools[0], pools[1], table, kv, torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV))
    q = queries(2, 16, d)
    out, lse = api.paged_attn(cache, q)
    shape = B.shape_of(cfg)
    blocks = torch.full((2, hkv, 16), -1, dtype=torch.int32, device=DEV)
    for s, n in enumerate(lens):
        blocks[s, :, :-(-n // 128)] = torch.arange(-(-n // 128), dtype=torch.int32, device=DEV)
    flat = [p.view(-1, hkv, d) for p in pools]
    sparse, sparse_lse = torch.empty_like(q), torch.empty(2, 16, device=DEV)
    B.msa_sparse_attn_decode(shape, q, flat[0], flat[1], flat[0].shape[0], torch.tensor([0, 16 * page], device=DEV), kv, 2, blocks, sparse,
                             sparse_lse, B.alloc_workspace(B.msa_sparse_attn_decode_workspace_bytes(shape, 2), DEV))
    check(cache, q, out, lse)
    check(cache, q, sparse, sparse_lse)


def test_refusals_of_the_abi():
    lib = B.lib()
    one = ctypes.c_void_p(256)  # non-null and aligned, never followed on these paths

    def call(n=5, q=one, hq=8, out=one, lse=None, scale=0.0, ws=one, nbytes=16, **c):
        c = dict(k=256, v=256, page_table=256, kv_lens=256, cu_q=256, batch=2, max_pages=3, n_pages=9, page_size=16, n_kv_heads=2,
                 head_dim=128, fp8=0) | c
        return lib.msa_paged_attn(ctypes.byref(B.MsaPagedCache(**c)), q, B.c_i32(hq), B.c_i64(n), ctypes.c_float(scale), out, lse, ws,
                                  B.c_sz(nbytes), None)

    assert call() == 3                                    # the workspace is too small
    assert call(n=0) == 0 and call(batch=0) == 0
    for bad in (dict(n=-1), dict(n=1 << 31), dict(q=None), dict(out=None), dict(q=ctypes.c_void_p(264)), dict(hq=0), dict(hq=7), dict(v=None),
                dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(ws=None), dict(ws=ctypes.c_void_p(264)),
                dict(lse=ctypes.c_void_p(258)), dict(page_size=0), dict(n_kv_heads=0), dict(fp8=3), dict(kv_lens=None)):
        assert call(**bad) == 1, bad
    assert call(head_dim=100) == 2 and call(head_dim=512) == 2 and call(hq=2048) == 2
    size = ctypes.c_size_t(0)
    cache = B.MsaPagedCache(page_size=16, n_kv_heads=2, head_dim=128, n_pages=4)
    assert lib.msa_paged_attn_workspace_bytes(ctypes.byref(cache), B.c_i32(16), ctypes.byref(size)) == 0 and size.value > 0
    assert lib.msa_paged_attn_workspace_bytes(ctypes.byref(cache), B.c_i32(15), ctypes.byref(size)) == 1
    assert lib.msa_paged_attn_workspace_bytes(ctypes.byref(cache), B.c_i32(16), None) == 1


@pytest.mark.gpu
def test_refusals_of_tensors():
    cache = make([(2, 1)], 16, 2, 128, False)
    q = queries(2, 8, 128)
    for c, x in ((cache._replace(v=None), q), (cache, q.float()), (cache, q[:, ::2]), (cache, q[..., :64]), (cache, q.cpu()),
                 (cache._replace(cu_q=cache.cu_q.long()), q)):
        with pytest.raises(ValueError):
            api.paged_attn(c, x)
    with pytest.raises(ValueError):
        api.paged_attn(cache, q, out=torch.empty(2, 4, 128, dtype=torch.bfloat16, device=DEV))
    with pytest.raises(B.MsaError):  # heads that are no multiple of the cache's
        api.paged_attn(cache, q[:, :7].contiguous())
    with pytest.raises(B.MsaError):
        api.paged_attn(cache, q, workspace=B.alloc_workspace(1024))
