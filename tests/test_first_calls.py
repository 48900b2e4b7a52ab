"""The first call of a process inside a capture, and calls of several host threads at once."""

import os
import subprocess
import sys
import threading

import pytest
import torch

from paper_2606_13392_b200 import api
from paper_2606_13392_b200 import binding as B
from test_norm_rope import make as make_rows
from test_paged_attn import check, make, queries

DEV = "cuda"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

FIRST = """
import sys
sys.path.insert(0, %r)
sys.path.insert(0, %r)
import torch
from paper_2606_13392_b200 import api, binding as B
from test_norm_rope import make as make_rows
from test_paged_attn import check, make, queries
q, k, wq, wk, pos, freqs = make_rows(50, 8, 2, 128, 64, True, False, False)
rope = api.Rope(freqs)
caches = [make(lens, 16, 2, 128, fp8) for lens, fp8 in (([(40, 300), (10, 5)], False), ([(40, 300), (1, 5)] + [(1, 9)] * 30, True), ([(1, 300)] * 9, True))]
qs = [queries(int(c.cu_q[-1]), 16, 128) for c in caches]
torch.cuda.synchronize()
def calls():
    got = list(api.qk_norm_rope(q, k, pos, rope, wq, wk)) + list(api.qk_norm_rope_backward(q, k, q, k, pos, rope, wq, wk))
    got.append(api.paged_append(caches[0], k, k, q, rope, wq, wk))
    for c, x in zip(caches, qs):
        got += api.paged_attn(c, x)
    return got
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = calls()
graph.replay()
torch.cuda.synchronize()
assert B.check_async_status() == (0, 0)
assert all(torch.equal(a, b) for a, b in zip(got, calls()))
for (c, x), i in zip(zip(caches, qs), range(3)):
    check(c, x, *got[7 + 2 * i:9 + 2 * i])
print("ok")
"""


@pytest.mark.gpu
def test_the_first_call_of_a_process_is_captured():
    run = subprocess.run([sys.executable, "-c", FIRST % (ROOT, os.path.join(ROOT, "tests"))], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip().endswith("ok"), run.stderr[-3000:]


@pytest.mark.gpu
def test_calls_of_several_threads():
    jobs = []
    for i, (lens, fp8) in enumerate((([(40, 900), (1, 500)], False), ([(33, 700)] + [(1, 40 * i) for i in range(20)], True), ([(1, 900)] * 8, True))):
        cache = make(lens, 16, 2, 128, fp8, seed=i)
        x = queries(sum(n for n, _ in lens), 16, 128, seed=i)
        jobs.append((cache, x, api.paged_attn(cache, x)))
    q, k, wq, wk, pos, freqs = make_rows(300, 8, 2, 128, 64, True, False, False)
    want = api.qk_norm_rope(q, k, pos, api.Rope(freqs), wq, wk)
    torch.cuda.synchronize()
    faults = []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(50):
                    if i < len(jobs):
                        cache, x, ref = jobs[i]
                        got = api.paged_attn(cache, x)
                    else:
                        ref, got = want, api.qk_norm_rope(q, k, pos, api.Rope(freqs), wq, wk)
                    torch.cuda.current_stream().synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, ref)):
                        faults.append((i, "differs"))
        except Exception as e:  # (a thread's exception would be lost)
            faults.append((i, repr(e)))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs) + 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not faults and B.check_async_status() == (0, 0)
    for cache, x, ref in jobs:
        check(cache, x, *ref)
