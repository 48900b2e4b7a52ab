"""Batches on fp8 caches whose sequences go to two kernels: those of few new tokens, whose rows one small tile holds, and
the others.  Against the definition in 64 bits; tolerances as in test_paged_attn.py."""

import random

import pytest
import torch

from paper_2606_13392_b200 import api
from paper_2606_13392_b200 import binding as B
from test_paged_attn import check, make, queries

DEV = "cuda"

CASES = [  # lens (new, old), page, query heads per KV head, KV heads
    ([(1, 40 + 9 * i) for i in range(63)] + [(65, 5000)], 64, 8, 2),       # one chunk beside single tokens
    ([(70, 5000)] + [(1, 40 + 9 * i) for i in range(63)], 64, 8, 2),
    ([(1, 700)] * 5 + [(33, 900), (0, 7), (2, 300), (3, 300), (0, 0), (130, 1), (1, 0)], 16, 8, 2),
    ([(1, 700), (2, 65), (1, 0), (2, 3000)], 48, 16, 1),                    # one token fits, two do not
    ([(1, 700), (2, 65), (3, 1000), (4, 127), (0, 3)] * 3, 16, 5, 2),       # tiles of 5 rows, or 15
    ([(16, 700), (17, 65), (1, 1000), (8, 127), (9, 3)], 16, 1, 3),
    ([(5, 700), (6, 65), (2, 1000), (3, 127), (1, 3)], 8, 3, 2),
    ([(1, 700), (2, 65), (5, 1000), (0, 3)], 64, 12, 2),
    ([(40, 700), (50, 20), (0, 9)], 128, 4, 2),                             # none for the small kernel
    ([(2, 70), (2, 2000), (1, 20), (0, 9)], 128, 4, 2),                     # none for the other
    ([(0, 5), (2, 3000), (0, 0)], 64, 8, 1),
    ([(0, 5), (3, 3000), (0, 0)], 64, 8, 1),
    ([(0, 40 + i) for i in range(62)] + [(63, 900), (1, 50)], 64, 8, 2),     # empty ones leave room for a long one
    ([(0, 9)] * 20 + [(19, 400)] + [(1, 70)] * 20, 16, 16, 1),
    ([(1 + 29 * (i % 50 == 7), i % 150) for i in range(700)], 16, 8, 1),    # more sequences than threads
]


@pytest.mark.gpu
@pytest.mark.parametrize("lens,page,group,hkv", CASES)
@pytest.mark.parametrize("extra", [0, 37])
def test_mixed_batches(lens, page, group, hkv, extra):
    cache = make(lens, page, hkv, 128, True)
    n = sum(x for x, _ in lens)
    q = queries(n + extra, group * hkv, 128)
    out = torch.full_like(q, 5.0)
    got, lse = api.paged_attn(cache, q, out=out)
    assert B.check_async_status() == (0, 0)
    assert (out[n:] == 5).all()  # rows of a padded batch
    check(cache, q, out, lse)
    again, lse2 = api.paged_attn(cache, q)
    assert torch.equal(again[:n], out[:n]) and torch.equal(lse[:n], lse2[:n])
    for said in (1, max(x for x, _ in lens), 5000, (1 << 31) - 1):  # a hint, which may be wrong
        out.fill_(5.0)
        _, lse = api.paged_attn(cache, q, out=out, max_new=said)
        assert B.check_async_status() == (0, 0) and (out[n:] == 5).all()
        check(cache, q, out, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(8))
def test_random_mixed_batches(seed):
    r = random.Random(100 + seed)
    top = r.choice([100, 2000, 20000])
    lens = [(r.choice([1, 1, 1, 1, 2, 3, 0, 9, 70]), r.randint(0, top)) for _ in range(r.randint(2, 60))] + [(r.choice([40, 300]), r.randint(0, top))]
    r.shuffle(lens)
    page, group, hkv = r.choice([8, 16, 40, 64, 128]), r.choice([1, 2, 4, 7, 8, 16]), r.choice([1, 2, 4])
    cache = make(lens, page, hkv, 128, True, seed)
    q = queries(sum(n for n, _ in lens), group * hkv, 128, seed)
    out, lse = api.paged_attn(cache, q, 0.11)
    assert B.check_async_status() == (0, 0)
    check(cache, q, out, lse, 0.11)


@pytest.mark.gpu
def test_which_kernels_a_call_launches():
    def launches(lens, group, fp8=True, said=0):
        cache = make(lens, 16, 2, 128, fp8)
        q = queries(sum(n for n, _ in lens), 2 * group, 128)
        before = B.lib().msa_launch_count()
        api.paged_attn(cache, q, max_new=said)
        return B.lib().msa_launch_count() - before

    chunk = [(1, 50)] * 63 + [(65, 500)]
    assert launches(chunk, 8) == 3               # a chunk does not go to the small tiles, however many single tokens there are
    assert launches(chunk, 8, False) == 2
    assert launches([(1, 90)], 8) == 2 and launches([(1, 90)] * 2, 8) == 2   # no room for a longer one
    assert launches([(1, 90)] * 40, 8) == 2 and launches([(1, 90)] * 40, 16) == 2   # nor here
    assert launches([(2, 90)] * 40, 8) == 3 and launches([(5, 90)] * 40, 8) == 2     # some may be longer; all are
    idle = [(0, 90)] * 63 + [(64, 500)]              # sequences without new tokens leave room that the sum does not show
    assert launches(idle, 8) == 2 and launches(idle, 8, said=64) == 3
    assert launches([(2, 90)] * 40, 8, said=2) == 2 and launches([(3, 90), (1, 5)] * 20, 8, said=3) == 3
    assert launches([(65, 90)], 32) == 2         # groups beyond the small tiles


@pytest.mark.gpu
def test_a_replay_follows_lengths_across_the_kernels():
    batch, rows, hkv = 12, 24, 2
    cache = make([(2, 400 + 50 * i) for i in range(batch)], 16, hkv, 128, True)
    q = queries(rows, 8 * hkv, 128)
    api.paged_attn(cache, q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = api.paged_attn(cache, q)
    for news in ([2] * 12, [1] * 11 + [13], [24] + [0] * 11, [0, 3, 3, 3, 3, 3, 3, 3, 3, 0, 0, 0], [1] * 12):
        cache.cu_q.copy_(torch.tensor([sum(news[:i]) for i in range(batch + 1)], dtype=torch.int32))
        n = sum(news)
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        check(cache, q, out, lse)
        assert (out[n:] == 5).all()
        want, want_lse = api.paged_attn(cache, q)
        assert torch.equal(out[:n], want[:n]) and torch.equal(lse[:n], want_lse[:n])
    assert B.check_async_status() == (0, 0)


@pytest.mark.gpu
def test_guard_bands_and_two_streams():
    lens = [(1, 40 + 90 * i) for i in range(30)] + [(70, 5000), (3, 4)]
    n = sum(x for x, _ in lens)
    cache, other = make(lens, 16, 2, 128, True), make(lens, 16, 2, 128, True, seed=9)
    q = queries(n, 16, 128)
    need = B.msa_paged_attn_workspace_bytes(cache.k, 16)
    raw = torch.full((need + 8192,), 0xCD, dtype=torch.uint8, device=DEV)
    outs = torch.full((n + 2, 16, 128), 3.0, dtype=torch.bfloat16, device=DEV)
    out, lse = api.paged_attn(cache, q, out=outs[1:n + 1], workspace=raw[4096:4096 + need])
    check(cache, q, out, lse)
    assert (raw[:4096] == 0xCD).all() and (raw[4096 + need:] == 0xCD).all() and (outs[0] == 3).all() and (outs[n + 1] == 3).all()
    with pytest.raises(B.MsaError):
        api.paged_attn(cache, q, workspace=raw[4096:4096 + need - 256])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = [api.paged_attn(other, q) for _ in range(5)]
    b = [api.paged_attn(cache, q) for _ in range(5)]
    torch.cuda.synchronize()
    check(other, q, *a[-1])
    assert all(torch.equal(x[0], out) and torch.equal(x[1], lse) for x in b) and all(torch.equal(x[0], a[0][0]) for x in a)


@pytest.mark.gpu
def test_a_wait_that_runs_out_in_both_kernels():
    lens = [(1, 900 + 10 * i) for i in range(20)] + [(40, 3000)]
    cache = make(lens, 16, 2, 128, True)
    q = queries(sum(n for n, _ in lens), 16, 128)
    try:
        B.msa_debug_set_wait(20000, 2000000)  # 10 us against copy roles that are 1 ms late
        api.paged_attn(cache, q)
        assert B.check_async_status()[0] == 5
    finally:
        B.msa_debug_set_wait(0, 0)
    out, lse = api.paged_attn(cache, q)
    assert B.check_async_status() == (0, 0)
    check(cache, q, out, lse)


def test_a_hint_below_zero_is_refused():
    import ctypes
    one = ctypes.c_void_p(256)  # non-null and aligned, never followed on this path
    cache = B.MsaPagedCache(k=256, v=256, page_table=256, kv_lens=256, cu_q=256, batch=2, max_pages=3, n_pages=9, page_size=16, n_kv_heads=2,
                            head_dim=128, fp8=1, max_new=-1)
    assert B.lib().msa_paged_attn(ctypes.byref(cache), one, B.c_i32(8), B.c_i64(5), ctypes.c_float(0), one, None, one, B.c_sz(16), None) == 1
    cache.max_new = 3
    assert B.lib().msa_paged_attn(ctypes.byref(cache), one, B.c_i32(8), B.c_i64(5), ctypes.c_float(0), one, None, one, B.c_sz(16), None) == 3
