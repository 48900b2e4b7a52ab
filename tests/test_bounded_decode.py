"""A decode loop on a cache with a budget - append, attention, weights, choice, move, next token - against lists of tokens in
64 bits; the same calls captured, on several streams and threads, refused, and with waits that run out."""

import math
import os
import subprocess
import sys
import threading

import pytest
import torch

from paper_2606_13392_b200 import api
from paper_2606_13392_b200 import binding as B
from test_launch_errors import a_capture_elsewhere
from test_paged_append import batch
from test_paged_evict import chosen
from test_paged_weights import filled, queries, reference

DEV = "cuda"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
def test_a_bounded_cache_step_by_step(fp8):
    hq, hkv, d, page, budget, limit = 16, 2, 128, 16, 80, 112
    g = torch.Generator(device=DEV).manual_seed(11)
    kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
    pools = [torch.zeros(20, page, hkv, d, device=DEV).to(kind) for _ in range(2)]
    weights = torch.full((20, hkv, page), math.nan, device=DEV)  # (nothing is read that was not written)
    table = torch.randperm(20, generator=g, device=DEV)[:16].int().view(2, 8)
    rope = api.Rope(api.rope_frequencies(64, 1e5))
    wq, wk = [(1 + 0.2 * torch.randn(d, generator=g, device=DEV)).bfloat16() for _ in range(2)]
    lens, seen = torch.zeros(2, dtype=torch.int32, device=DEV), [0, 0]
    held = [[] for _ in range(2)]  # of each sequence: per head a list of (key bytes, value bytes)
    evictions = 0
    for step in [(70, 33), (20, 1)] + [(1, 1)] * 30 + [(3, 40), (1, 0), (1, 1)]:
        n = sum(step)
        qkv = torch.randn(n, (hq + 2 * hkv) * d, generator=g, device=DEV).bfloat16()
        q, k, v = [x.unflatten(1, (-1, d)) for x in qkv.split([hq * d, hkv * d, hkv * d], 1)]
        positions = torch.cat([torch.arange(seen[s], seen[s] + step[s]) for s in range(2)]).to(DEV)
        seen = [seen[s] + step[s] for s in range(2)]
        cu = torch.tensor([0, step[0], n], dtype=torch.int32, device=DEV)
        lens = lens + torch.tensor(step, dtype=torch.int32, device=DEV)
        cache = api.PagedCache(pools[0], pools[1], table, lens, cu)
        q, k = api.qk_norm_rope(q, k, positions, rope, wq, wk)
        api.paged_append(cache, k, v)
        out, lse = api.paged_attn(cache, q)
        old = weights.clone()
        api.paged_weights(cache, q, lse, weights, 0.9)
        want, tol, _ = reference(cache, q, lse, old, 0.9)
        # the cache holds the tokens that it should, and attention sees them
        kv = lens.tolist()
        for s in range(2):
            for i in range(step[s]):
                row = int(cu[s]) + i
                if not held[s]:
                    held[s] = [[] for _ in range(hkv)]
                for h in range(hkv):
                    held[s][h].append((k[row, h].to(kind).view(torch.uint8), v[row, h].to(kind).view(torch.uint8)))
            place = torch.arange(kv[s], device=DEV)
            at = (table[s].long()[place // page], place % page)
            for h in range(hkv):
                assert len(held[s][h]) == kv[s]
                for which in range(2):
                    assert torch.equal(pools[which].view(torch.uint8)[at[0], at[1], h], torch.stack([t[which] for t in held[s][h]]))
                a = weights[at[0], h, at[1]].double()
                # (no term came in that the definition lacks: the attention's lse is off by 2^-10 at most on these scores)
                assert (a - want[at[0], h, at[1]]).abs().le(tol[at[0], h, at[1]] + 1e-9).all()
                kd, vd = [torch.stack([t[w] for t in held[s][h]]).view(kind).double() for w in range(2)]
                rows = q[int(cu[s]):int(cu[s + 1]), h * 8:(h + 1) * 8].double().transpose(0, 1)
                x = rows @ kd.T / math.sqrt(d)
                x = x.masked_fill(place > torch.arange(kv[s] - step[s], kv[s], device=DEV)[:, None], -math.inf)
                ref = (x.softmax(-1) @ vd).transpose(0, 1)
                got = out[int(cu[s]):int(cu[s + 1]), h * 8:(h + 1) * 8].double()
                assert (got - ref).abs().le(2.0 ** -8 * ref.abs() + 2.0 ** -7 * vd.abs().amax()).all()
        if max(kv) > limit:
            evictions += 1
            keep, new = api.paged_keep(cache, weights, budget, 4, 16)
            before = weights.clone()
            api.paged_compact(cache, keep, weights)
            for s in range(2):
                for h in range(hkv):
                    w = before[table[s].long(), h].flatten()[:kv[s]].tolist()
                    stay = chosen(w, kv[s], budget, 4, 16)
                    assert keep[s, h].tolist() == stay + [-1] * (budget - len(stay))
                    held[s][h] = [held[s][h][p] for p in stay]
                    now = weights[table[s].long(), h].flatten()[:len(stay)].tolist()
                    assert now == [w[p] for p in stay]
            lens = new
        logits = torch.randn(n, 1000, generator=g, device=DEV)
        token, _ = api.sample(logits, torch.rand(n, generator=g, device=DEV), 0.8, 40, 0.95)
        assert ((token >= 0) & (token < 1000)).all()
    assert evictions >= 1 and B.check_async_status() == (0, 0)


def step_of(cache, q, weights, logits, u, budget):
    """Everything behind an append, as a serving step runs it."""
    out, lse = api.paged_attn(cache, q)
    api.paged_weights(cache, q, lse, weights, 0.9)
    keep, lens = api.paged_keep(cache, weights, budget, 2, 8)
    api.paged_compact(cache, keep, weights)
    return [out, lse, weights, keep, lens, cache.k.view(torch.uint8), cache.v.view(torch.uint8), *api.sample(logits, u, 0.9, 30, 0.9)]


def state_of(lens, fp8, seed, heads=2, hq=16):
    cache = filled(batch(lens, 16, heads, 128, fp8, seed=seed), seed)
    cache.v.view(torch.uint8).copy_(cache.k.view(torch.uint8).flip(0))
    cache.v.copy_(torch.where(cache.v.float().isnan(), torch.zeros_like(cache.v, dtype=torch.float32), cache.v.float()).to(cache.v.dtype))
    cache.k.copy_(torch.where(cache.k.float().isnan(), torch.zeros_like(cache.k, dtype=torch.float32), cache.k.float()).to(cache.k.dtype))
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [cache, queries(cache, hq, seed=seed), torch.rand(cache.k.shape[0], heads, 16, generator=g, device=DEV),
            torch.randn(40, 5000, generator=g, device=DEV), torch.rand(40, generator=g, device=DEV), 64]


def copy_of(state):
    cache = state[0]._replace(k=state[0].k.clone(), v=state[0].v.clone(), kv_lens=state[0].kv_lens.clone(), cu_q=state[0].cu_q.clone())
    return [cache] + [x.clone() if torch.is_tensor(x) else x for x in state[1:]]


LENS = [[(1, 90), (1, 300), (1, 20)], [(40, 200), (1, 100), (90, 30)]]


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens", LENS)
def test_a_captured_step_follows_its_inputs(lens, fp8):
    state = state_of(lens, fp8, 3)
    step_of(*copy_of(state))
    static = copy_of(state)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step_of(*static)
    for seed in (4, 5):
        other = state_of(lens, fp8, seed)
        if seed == 5:  # shorter sequences, fewer new tokens, on the same pages
            other[0].kv_lens.sub_(torch.tensor([7, 0, 3], dtype=torch.int32, device=DEV))
            new = [max(1, n - 5) for n, _ in lens]
            other[0].cu_q.copy_(torch.tensor([sum(new[:i]) for i in range(4)], dtype=torch.int32))
        for a, b in zip(static, other):
            if torch.is_tensor(a):
                a.copy_(b)
        for a, b in zip(static[0], other[0]):
            (a.view(torch.uint8) if a.element_size() == 1 else a).copy_(b.view(torch.uint8) if b.element_size() == 1 else b)
        rows = int(other[0].cu_q[-1])
        want = step_of(*copy_of(other))
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            if i < 2:
                a, b = a[:rows], b[:rows]
            assert torch.equal(a, b), i
    assert B.check_async_status() == (0, 0)


@pytest.mark.gpu
def test_two_captured_steps_and_calls_of_several_threads_at_once():
    states = [state_of(lens, fp8, i) for i, (lens, fp8) in enumerate((x, f) for x in LENS for f in (False, True))]
    wants = [[t.clone() for t in step_of(*copy_of(s))] for s in states]
    torch.cuda.synchronize()
    graphs = []
    for s in states[:2]:
        static = copy_of(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step_of(*static)
        graphs.append((graph, static, got))
    for _ in range(5):
        for (_, static, _), s in zip(graphs, states):
            for a, b in zip([static[0].k.view(torch.uint8), static[0].v.view(torch.uint8), static[2]],
                            [s[0].k.view(torch.uint8), s[0].v.view(torch.uint8), s[2]]):
                a.copy_(b)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in graphs]
        for (graph, _, _), stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for (_, _, got), want in zip(graphs, wants):
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    faults = []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(15):
                    got = step_of(*copy_of(states[i]))
                    torch.cuda.current_stream().synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, wants[i])):
                        faults.append((i, "differs"))
        except Exception as e:  # (a thread's exception would be lost)
            faults.append((i, repr(e)))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(states))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not faults and B.check_async_status() == (0, 0)


@pytest.mark.gpu
def test_outputs_made_while_the_current_stream_is_busy():
    cache, _, weights, _, _, _ = state_of([(0, 3000)] * 8, False, 1)
    logits, u = torch.randn(3000, 600, device=DEV), torch.rand(3000, device=DEV)
    args = (cache.k, cache.page_table, cache.kv_lens, cache.cu_q, weights, 2000, 4, 9)
    side = torch.cuda.Stream()
    for name, call in (("keep", lambda s: B.msa_paged_keep(*args, stream=s)), ("sample", lambda s: B.msa_sample(logits, u, 0.8, 40, 0.9, 0.0, stream=s))):
        outs = call(None)
        want = [o.clone() for o in outs]
        side.wait_stream(torch.cuda.current_stream())
        torch.cuda.synchronize()
        torch.cuda._sleep(40_000_000)
        for o in outs:
            o.fill_(7)
        del outs, o
        got = call(side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), name


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
def test_a_wait_that_runs_out_is_reported(fp8):
    cache, q, weights, *_ = state_of([(70, 700), (100, 90)], fp8, 2)
    _, lse = api.paged_attn(cache, q)
    want = api.paged_weights(cache, q, lse, weights.clone(), 0.9)
    try:
        B.msa_debug_set_wait(20000, 2000000)  # 10 us against a copy role that is 1 ms late
        api.paged_weights(cache, q, lse, weights.clone(), 0.9)
        assert B.check_async_status()[0] == 5
    finally:
        B.msa_debug_set_wait(0, 0)
    got = api.paged_weights(cache, q, lse, weights.clone(), 0.9)
    assert B.check_async_status() == (0, 0) and torch.equal(got, want)


@pytest.mark.gpu
def test_a_refused_launch_is_reported_by_its_own_call():
    cache, q, weights, logits, u, _ = state_of([(70, 700), (1, 90)], True, 2)
    legacy = torch.cuda.default_stream()
    _, lse = api.paged_attn(cache, q)
    ws = B.alloc_workspace(B.msa_paged_weights_workspace_bytes(cache.k, 16), DEV)
    keep, lens = api.paged_keep(cache, weights, 50)
    token, logprob = api.sample(logits, u)
    places = (cache.k, cache.page_table, cache.kv_lens, cache.cu_q)
    calls = [lambda: B.msa_paged_weights(*places, q, lse, 0.0, 0.5, weights.clone(), ws, stream=legacy),
             lambda: B.msa_paged_keep(*places, weights, 50, 0, 0, keep, lens, stream=legacy),
             lambda: B.msa_paged_compact(cache.k, cache.v, *places[1:], keep, None, stream=legacy),
             lambda: B.msa_sample(logits, u, 1.0, 0, 1.0, 0.0, token, logprob, stream=legacy)]
    kept = [x.clone() for x in (keep, lens, token, logprob)]
    weights_now = weights.clone()
    calls[0] = lambda w=weights_now: B.msa_paged_weights(*places, q, lse, 0.0, 0.5, w, ws, stream=legacy)
    for call in calls:
        with a_capture_elsewhere(), pytest.raises(B.MsaError) as e:
            call()
        assert e.value.code == 4
        calls[1]()
        calls[3]()
        assert all(torch.equal(a, b) for a, b in zip((keep, lens, token, logprob), kept))
    assert B.check_async_status() == (0, 0)


FIRST = """
import sys
sys.path.insert(0, %r)
sys.path.insert(0, %r)
import torch
from test_bounded_decode import B, copy_of, state_of, step_of
states = [state_of(lens, fp8, 1) for lens, fp8 in (([(1, 90), (1, 300)], False), ([(40, 200), (1, 100)], True), ([(90, 10)], False))]
static = [copy_of(s) for s in states]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = [step_of(*s) for s in static]
graph.replay()
torch.cuda.synchronize()
assert B.check_async_status() == (0, 0)
assert all(torch.equal(a, b) for s, g in zip(states, got) for a, b in zip(g, step_of(*copy_of(s))))
print("ok")
"""


@pytest.mark.gpu
def test_the_first_call_of_a_process_is_captured():
    run = subprocess.run([sys.executable, "-c", FIRST % (ROOT, os.path.join(ROOT, "tests"))], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip().endswith("ok"), run.stderr[-3000:]
