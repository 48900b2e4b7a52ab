"""The next token from its logits: against the definition, row by row in 64 bits.

A choice is a whole number and has to be equal.  Where the random number falls within 1e-9 of a border between two
tokens (or a nucleus's end within that of its target) the reference says so and the row is not compared; for the inputs here that is
none or next to none, which is asserted.  A log-probability is a difference of two 64-bit numbers of at most some hundred,
rounded once: 2^-24 of itself, plus 1e-9."""

import ctypes
import math

import pytest
import torch

from paper_2606_13392_b200 import api
from paper_2606_13392_b200 import binding as B

DEV = "cuda"
NEAR = 1e-9


def pick(x, u, t, k, p, m):
    """(token, log-probability, clear) of one row of logits, a CPU tensor; settings as numbers."""
    f = lambda v: float(torch.tensor(v, dtype=torch.float32))  # noqa: E731
    x, t, p, m, u = x.double(), f(t), f(p), f(m), f(u)
    if bool(x.isnan().any()) or x.max() == -math.inf or t != t or u != u:
        return -1, math.nan, True
    if t <= 0:
        return int(x.argmax()), 0.0, True  # (argmax of equal ones: the first, checked below)
    z = torch.where(x == x.max(), torch.zeros_like(x), (x - x.max()) / t)
    w = z.exp()
    order = torch.argsort(x, descending=True, stable=True)
    clear = True
    if 0 < k < len(x):
        order = order[:k]
    if p < 1:
        mass = w[order].cumsum(0)
        goal = max(p, 0.0) * mass[-1]
        n = int((mass < goal).sum()) + 1
        # (the border matters where another token could be kept)
        if p > 0 and ((mass - goal).abs() < NEAR * mass[-1]).any() and not bool((mass == goal).any()):
            clear = False
        order = order[:max(1, n)]
    if m > 0:
        least = math.log(m)
        clear = clear and not bool(((z[order] - least).abs() < NEAR).any())
        order = torch.tensor([i for i in order.tolist() if z[i] == 0 or z[i] >= least])
    live = order.sort().values
    live = live[w[live] > 0]
    mass = w[live].cumsum(0)
    j = min(int((mass <= u * mass[-1]).sum()), len(live) - 1)
    if u > 0 and ((mass - u * mass[-1]).abs() < NEAR * mass[-1]).any() and not bool((mass == u * mass[-1]).any()):
        clear = False
    return int(live[j]), float(z[live[j]] - mass[-1].log()), clear


def check(logits, u, t=1.0, k=0, p=1.0, m=0.0, unclear=0):
    token, logprob = api.sample(logits, u, t, k, p, m)
    at = lambda v, r: v[r].item() if torch.is_tensor(v) else v  # noqa: E731
    x, skipped = logits.cpu(), 0
    for r in range(len(x)):
        want, lp, clear = pick(x[r], at(u, r), at(t, r), at(k, r), at(p, r), at(m, r))
        if not clear:
            skipped += 1
            continue
        assert int(token[r]) == want, (r, int(token[r]), want)
        got = float(logprob[r])
        assert (got != got and lp != lp) or abs(got - lp) <= 2.0 ** -24 * abs(lp) + 1e-9, (r, got, lp)
    assert skipped <= unclear
    return token


def made(rows, vocab, kind, spread, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (spread * torch.randn(rows, vocab, generator=g, device=DEV)).to(kind), torch.rand(rows, generator=g, device=DEV)


SETTINGS = [(1.0, 0, 1.0, 0.0), (0.7, 50, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (0.8, 40, 0.95, 0.0), (1.3, 0, 1.0, 0.05), (0.9, 100, 0.8, 0.02),
            (1.0, 1, 1.0, 0.0), (1.0, 0, 0.0, 0.0), (0.0, 5, 0.5, 0.1), (2.0, 900, 0.99, 0.0), (0.05, 0, 0.999, 0.0), (1.5, 0, 0.5, 0.3)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("vocab", [1, 2, 31, 32, 33, 257, 1000, 4097, 32000])
def test_settings(kind, vocab):
    for i, s in enumerate(SETTINGS):
        logits, u = made(5, vocab, kind, 3.0, 100 * i + vocab)
        check(logits, u, *s)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,rows,vocab,spread", [(torch.bfloat16, 3, 128000, 3.0), (torch.float32, 2, 100003, 0.01), (torch.float16, 70, 5000, 1.0),
                                                    (torch.float32, 160, 2000, 8.0), (torch.bfloat16, 1, 300001, 2.0), (torch.float32, 1, 1 << 21, 1.0)])
def test_large(kind, rows, vocab, spread):
    logits, u = made(rows, vocab, kind, spread, vocab)
    for s in ((1.0, 0, 1.0, 0.0), (0.8, 50, 0.9, 0.0), (1.0, 0, 0.95, 0.0), (1.1, 20000, 0.97, 0.001), (1.0, 0, 0.9999, 0.0)):
        check(logits, u, *s, unclear=1)


@pytest.mark.gpu
def test_every_row_has_its_settings():
    logits, u = made(64, 3001, torch.bfloat16, 2.5, 8)
    g = torch.Generator(device=DEV).manual_seed(4)
    r = lambda: torch.rand(64, generator=g, device=DEV)  # noqa: E731
    t = torch.where(r() < 0.2, torch.zeros(64, device=DEV), 0.3 + r())
    k = (r() * 4000 - 500).int()
    p, m = r() * 1.3, (r() - 0.5).clamp(min=0) * 0.2
    check(logits, u, t, k, p, m)
    check(logits, u, t, 30, p, 0.0)
    check(logits, u, 0.9, k, 1.0, m)


@pytest.mark.gpu
def test_every_border_of_a_small_row():
    """All random numbers of a fine grid, equal logits in the row."""
    x = torch.tensor([0.5, 1.0, -math.inf, 1.0, -2.0, 0.5, 3.0, -7.0, 1.0], device=DEV)
    n = 4001
    u = torch.linspace(0, 1 - 2.0 ** -24, n, device=DEV)
    for s in ((1.0, 0, 1.0, 0.0), (0.5, 4, 1.0, 0.0), (1.0, 3, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (2.0, 0, 0.7, 0.0), (1.0, 0, 1.0, 0.1), (1.0, 5, 0.95, 0.05)):
        token = check(x.expand(n, -1).contiguous(), u, *s, unclear=2)
        assert (token[1:] >= token[:-1]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [7, 1000, 40000])
def test_equal_logits_go_by_index(kind, vocab):
    u = torch.tensor([0.0, 0.3, 0.6, 1 - 2.0 ** -24], device=DEV)
    flat = torch.full((4, vocab), 2.5, dtype=kind, device=DEV)
    assert check(flat, u).tolist() == [min(vocab - 1, int(float(v) * vocab)) for v in u]
    assert max(check(flat, u, 1.0, 3).tolist()) == 2
    assert max(check(flat, u, 1.0, 0, 0.5).tolist()) == (vocab + 1) // 2 - 1   # sums of ones are exact
    assert check(flat, u, 0.0).tolist() == [0] * 4
    few = (torch.arange(vocab, device=DEV) % 3).to(kind).expand(4, -1).contiguous()
    check(few, u, 1.0, vocab // 2)
    check(few, u, 1.0, 0, 0.8, 0.0)
    check(few, u, 0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16, torch.float32])
def test_rows_with_little_to_choose_from(kind):
    vocab = 2500
    x, u = made(9, vocab, kind, 2.0, 1)
    x[0] = -math.inf
    x[1, 77] = math.nan
    x[2], x[2, 1234] = -math.inf, -3.0
    x[3, 5] = x[3, 2000] = math.inf
    x[4] = torch.finfo(kind).min
    x[5] = torch.finfo(kind).min
    x[5, 9] = 1.0
    x[6, :2000] = -math.inf
    u[7] = math.nan
    x[8] = -math.inf
    x[8, [3, 4]] = torch.finfo(kind).max
    for s in SETTINGS:
        token = check(x, u, *s)
        assert token[0] == -1 and token[1] == -1 and token[2] == 1234 and int(token[3]) in (5, 2000) and token[7] == -1
    t = torch.full((9,), math.nan, device=DEV)
    assert (api.sample(x, u, t)[0] == -1).all()
    hot = torch.full((9,), math.inf, device=DEV)
    check(x, u, hot, 100)
    cold = torch.full((9,), 1e-45, device=DEV)
    assert check(x, u, cold)[5] == 9


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
def test_rows_anywhere_in_memory(kind):
    wide, u = made(6, 5013, kind, 3.0, 3)
    for lo, hi in ((0, 5000), (1, 5001), (3, 4999), (5, 6), (7, 40), (0, 4096)):
        part = wide[:, lo:hi]
        want = [t.clone() for t in api.sample(part.contiguous(), u, 0.9, 30, 0.9)]
        got = api.sample(part, u, 0.9, 30, 0.9)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        check(part, u, 1.0, 0, 0.95)
    # every other row; one row that is no matrix of its own
    check(wide[::2], u[::2].contiguous(), 1.0, 20)
    check(wide[3:4], u[3:4])
    # what surrounds the rows is not read into them: not numbers there
    framed = torch.full((4, 1030), math.nan, dtype=kind, device=DEV)
    framed[:, 9:1020] = wide[:4, :1011]
    check(framed[:, 9:1020], u[:4].contiguous(), 1.0, 0, 0.9)


@pytest.mark.gpu
def test_given_outputs_streams_and_graphs():
    logits, u = made(20, 9000, torch.bfloat16, 3.0, 6)
    want = api.sample(logits, u, 0.8, 50, 0.9)
    token, logprob = torch.full((20,), -9, device=DEV), torch.zeros(20, device=DEV)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    B.msa_sample(logits, u, 0.8, 50, 0.9, 0.0, token, logprob, stream=stream)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(token, want[0]) and torch.equal(logprob, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = api.sample(logits, u, 0.8, 50, 0.9)
    for seed in (7, 8):
        x, v = made(20, 9000, torch.bfloat16, 3.0, seed)
        logits.copy_(x)
        u.copy_(v)
        graph.replay()
        again = api.sample(logits, u, 0.8, 50, 0.9)
        assert torch.equal(out[0], again[0]) and torch.equal(out[1], again[1])
    assert api.sample(logits[:0], u[:0])[0].shape == (0,)


def test_refusals_without_a_launch():
    B.lib()
    call = B._fn("msa_sample")

    def go(s=B.MsaSampling(1.0, 0, 1.0, 0.0, None, None, None, None), x=4096, kind=0, stride=100, rows=2, vocab=100, u=4096, token=4096, lp=4096):
        return call(ctypes.byref(s) if s is not None else None, x, kind, stride, rows, vocab, u, token, lp, None)

    assert go(s=None) == 1 and go(x=None) == 1 and go(x=4097) == 1 and go(kind=2, x=4098) == 1 and go(kind=3) == 1 and go(kind=-1) == 1
    assert go(stride=99) == 1 and go(rows=-1) == 1 and go(vocab=0) == 1 and go(vocab=(1 << 21) + 1, stride=1 << 22) == 2
    assert go(u=None) == 1 and go(u=4097) == 1 and go(token=None) == 1 and go(token=4100) == 1 and go(lp=4097) == 1
    for bad in ((math.nan, 0, 1.0, 0.0), (1.0, 0, math.nan, 0.0), (1.0, 0, 1.0, math.nan)):
        assert go(s=B.MsaSampling(*bad, None, None, None, None)) == 1
    assert go(s=B.MsaSampling(1.0, 0, 1.0, 0.0, 4097, None, None, None)) == 1
    assert go(rows=0) == 0


def test_tensors_of_the_host_are_refused():
    with pytest.raises(ValueError):
        api.sample(torch.zeros(2, 5), torch.zeros(2))


@pytest.mark.gpu
def test_refusals_of_tensors():
    x, u = made(4, 50, torch.float32, 1.0, 1)
    for bad in (x.double(), x.t(), x[0], x[:, ::2], x.int(), x[:1].expand(4, -1)):
        with pytest.raises(ValueError):
            api.sample(bad, torch.rand(len(bad), device=DEV))
    for bad in (u.double(), u[:3], u.cpu(), u[:, None]):
        with pytest.raises(ValueError):
            api.sample(x, bad)
    for name, bad in (("temperature", u.half()), ("top_k", u), ("top_k", torch.ones(4, dtype=torch.int64, device=DEV)), ("top_p", u[:2]),
                      ("min_p", u.cpu())):
        with pytest.raises(ValueError):
            api.sample(x, u, **{name: bad})
    for name in ("temperature", "top_p", "min_p"):
        with pytest.raises(B.MsaError):
            api.sample(x, u, **{name: math.nan})
    with pytest.raises(ValueError):
        api.sample(x.requires_grad_(), u)


def pick_all(x, u, t, k, p, m):
    """pick() of many rows at once on the device -> (tokens, rows that are clear)."""
    x, u = x.double(), u.double()[:, None]
    t, p, m = [float(torch.tensor(v, dtype=torch.float32)) for v in (t, p, m)]
    z, index = x.sort(dim=-1, descending=True, stable=True)
    z = (z - z[:, :1]) / t
    w = z.exp()
    if 0 < k < x.shape[1]:
        w[:, k:] = 0
    clear = torch.ones(len(x), dtype=torch.bool, device=x.device)
    if p < 1:
        mass = w.cumsum(-1)
        goal = p * mass[:, -1:]
        clear &= ((mass - goal).abs() > NEAR * mass[:, -1:]).all(-1)
        w = torch.where(mass - w >= goal, 0.0, w)
    if m > 0:
        clear &= ((z - math.log(m)).abs() > NEAR).all(-1)
        w = torch.where(z < math.log(m), 0.0, w)
    w = torch.zeros_like(w).scatter_(1, index, w)
    upto = w.cumsum(-1)
    total = upto[:, -1:]
    clear &= ((upto - u * total).abs() > NEAR * total).all(-1)
    return (upto <= u * total).sum(-1), clear


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("vocab,spread,t,k,p,m", [(1159, 3.0, 1.5, 0, 0.99, 0.0), (4120, 2.0, 0.9, 0, 0.9, 0.0), (1500, 1.0, 1.0, 0, 0.5, 0.0),
                                                  (2001, 2.0, 1.0, 300, 0.9, 0.0), (1000, 2.0, 0.7, 20, 1.0, 0.05), (900, 2.5, 1.0, 0, 1.0, 0.0)])
def test_many_rows(kind, vocab, spread, t, k, p, m):
    """Enough rows that a token lost at the edge of a bin shows."""
    for seed in range(4):
        logits, u = made(8000, vocab, kind, spread, 50 + seed)
        token, _ = api.sample(logits, u, t, k, p, m)
        want, clear = pick_all(logits, u, t, k, p, m)
        assert clear.float().mean() > 0.99
        assert torch.equal(token[clear], want[clear]), (seed, (token != want)[clear].sum())
