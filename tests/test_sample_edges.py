"""Choices of the next token at the edges: few tokens allowed, settings out of the ordinary, rows anywhere.  The reference, its
tolerances and when a row is not compared are those of test_sample.py."""

import math

import pytest
import torch

from paper_2606_13392_b200 import api
from paper_2606_13392_b200 import binding as B
from test_sample import made, pick

DEV = "cuda"


def check_written(x, u, t, k, p, m=0.0, unclear=0):
    """As check() there, into given outputs that hold something else before."""
    token = torch.full((len(x),), -9, device=DEV)
    logprob = torch.full((len(x),), 99.0, device=DEV)
    B.msa_sample(x, u, t, k, p, m, token, logprob)
    skipped, rows, us = 0, x.cpu(), u.tolist()
    for r in range(len(x)):
        want, lp, clear = pick(rows[r], us[r], t, k, p, m)
        if not clear:
            skipped += 1
            continue
        assert int(token[r]) == want, (r, int(token[r]), want)
        got = float(logprob[r])
        assert (got != got and lp != lp) or abs(got - lp) <= 2.0 ** -24 * abs(lp) + 1e-9, (r, got, lp)
    assert skipped <= unclear


def leave_traces(kind):
    """Calls that leave counts, digits and sums of their own in the SMs' shared memory."""
    x, u = made(300, 3000, kind, 3.0, 5)
    api.sample(x, u)
    api.sample(x, u, 1.0, 0, 0.9)
    api.sample(x * 1e4, u, 1e-5, 100, 0.9)
    api.sample(-x.abs() * 1e4 - 1e4, u, 1e-5, 2900)


@pytest.mark.gpu
@pytest.mark.parametrize("k", [50, 1000])
@pytest.mark.parametrize("p", [1.0, 0.9])
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16, torch.float32])
def test_fewer_tokens_allowed_than_top_k_asks_for_at_low_temperatures(kind, k, p):
    vocab, allowed = 6000, [1, 2, 3, 10, 49, 50, 51, 200, 600, 999]
    x, u = made(len(allowed), vocab, kind, 3.0, k)
    g = torch.Generator().manual_seed(7)
    y = torch.full_like(x, -math.inf)
    for r, n in enumerate(allowed):
        places = torch.randperm(vocab, generator=g)[:n].to(DEV)
        y[r, places] = x[r, places]
        y[r, places[:2]] = -30.0 if r % 2 else 30.0  # (the largest is far from zero, or near it, of either sign)
        if r % 3 == 0:
            y[r, places] = -y[r, places].abs() - 9
    for t in (1e-6, 1e-5):
        for z in (y, -40 + y):
            leave_traces(kind)
            check_written(z, u, t, k, p)


@pytest.mark.gpu
@pytest.mark.parametrize("at", [1e6, -2e6])
@pytest.mark.parametrize("k,p,m", [(50, 1.0, 0.0), (1000, 1.0, 0.0), (1000, 0.9, 0.0), (700, 0.5, 0.01)])
def test_fewer_tokens_allowed_than_top_k_asks_for_far_from_zero(at, k, p, m):
    """Logits so far from zero that 32-bit steps between them are counted one by one; several of them weigh something."""
    vocab = 5000
    x, u = made(24, vocab, torch.float32, 3.0, 3)
    g = torch.Generator().manual_seed(8)
    y = torch.full_like(x, -math.inf)
    for r in range(24):
        places = torch.randperm(vocab, generator=g)[:3 + 25 * r].to(DEV)
        y[r, places] = at + x[r, places]
    leave_traces(torch.float32)
    check_written(y, u, 1.0, k, p, m, unclear=1)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16, torch.float32])
def test_one_infinite_logit_and_nothing_else(kind):
    x, u = made(4, 3000, kind, 1.0, 1)
    x.fill_(-math.inf)
    x[:, 1717] = math.inf
    for t, k, p, m in ((1.0, 50, 1.0, 0.0), (0.7, 2, 0.9, 0.0), (1.0, 2999, 0.5, 0.1), (1.0, 0, 0.9, 0.0), (0.0, 50, 0.9, 0.0)):
        leave_traces(kind)
        check_written(x, u, t, k, p, m)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [2, 400])
def test_more_equal_logits_than_a_list_holds_and_fewer_than_top_k(kind, rows):
    vocab = 20000
    x = torch.full((rows, vocab), -math.inf, dtype=kind, device=DEV)
    x[:, 100:19000:6] = -1.5  # 3150 of them
    u = made(rows, 1, kind, 1.0, rows)[1]
    for k, p in ((5000, 0.9), (3151, 0.5), (3150, 0.9), (3149, 0.9), (5000, 1.0)):
        leave_traces(kind)
        check_written(x, u, 0.8, k, p, unclear=2)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16, torch.float32])
def test_rows_that_begin_and_end_anywhere(kind):
    """Every place of the first and the last value in 16 bytes, rows of a piece or less among them."""
    for vocab in (1, 3, 5, 7, 8, 9, 15, 17, 23, 1001):
        wide, u = made(4, vocab + 16, kind, 3.0, vocab)
        for lo in range(9):
            for s in ((1.0, 0, 1.0, 0.0), (0.9, 4, 0.9, 0.0), (1.0, 0, 0.8, 0.0), (0.0, 0, 1.0, 0.0)):
                check_written(wide[:, lo:lo + vocab], u, *s, unclear=1)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["temperature", "top_p", "min_p"])
def test_a_setting_that_is_not_a_number_takes_its_row(name):
    """In a vector as in a number, which is refused: no filter is silently left out."""
    rows = 12
    x, u = made(rows, 4000, torch.bfloat16, 3.0, 2)
    settings = dict(temperature=torch.full((rows,), 0.8, device=DEV), top_k=torch.full((rows,), 30, dtype=torch.int32, device=DEV),
                    top_p=torch.full((rows,), 0.9, device=DEV), min_p=torch.full((rows,), 0.02, device=DEV))
    settings["top_k"][::2] = 0
    settings["min_p"][::3] = 0
    want = [t.clone() for t in api.sample(x, u, **settings)]
    assert (want[0] >= 0).all()
    settings[name] = settings[name].clone()
    settings[name][[1, 4, 6]] = math.nan
    token, logprob = api.sample(x, u, **settings)
    for r in range(rows):
        if r in (1, 4, 6):
            assert token[r] == -1 and logprob[r].isnan()
        else:
            assert token[r] == want[0][r] and logprob[r] == want[1][r]
    if name != "temperature":  # the largest logit, whatever the rest says
        settings["temperature"][:] = 0
        token, logprob = api.sample(x, u, **settings)
        assert torch.equal(token, x.float().argmax(1)) and (logprob == 0).all()
    with pytest.raises(B.MsaError):
        api.sample(x, u, **{name: math.nan})


@pytest.mark.gpu
def test_whole_numbers_beyond_32_bits_mean_what_they_say():
    x, u = made(40, 3000, torch.float32, 3.0, 9)
    want = [t.clone() for t in api.sample(x, u)]
    for k in (1 << 31, (1 << 32) + 5, (1 << 40) + 1, -(1 << 32) + 5, -(1 << 31) - 1):  # more than there are, or no limit
        assert all(torch.equal(a, b) for a, b in zip(api.sample(x, u, top_k=k), want)), k


@pytest.mark.gpu
def test_the_largest_logit_is_at_no_distance_of_itself():
    """Logits and temperatures whose product, rounded once more than it has to be, falls on the other side of a half: the largest
    logit's place would come out in front of the first, where nothing weighs anything."""
    pairs = [(352947.40625, 0.8524332046508789), (694587.375, 1.1001274585723877), (386510.59375, 0.8756565451622009),
             (613832.8125, 0.9162696003913879), (497531.15625, 0.7205303907394409), (645018.25, 0.9723894000053406)]
    for top, t in pairs:
        x = torch.full((3, 2000), top - 80.0, device=DEV)
        x[0, 1234] = x[1, 0] = x[2, [3, 1999]] = top
        for k, p in ((0, 1.0), (50, 1.0), (0, 0.9), (20, 0.9)):
            check_written(x, torch.full((3,), 0.6, device=DEV), t, k, p)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [400, 3000, 60000])
def test_min_p_of_a_flat_distribution(kind, vocab):
    """At an infinite temperature every logit is as likely as the largest, and at least once as likely."""
    x, _ = made(5, vocab, kind, 3.0, 4)
    u = torch.tensor([0.0, 0.2, 0.4, 0.7, 0.96], device=DEV)
    for m in (1.0, 0.5, 0.0):
        token, logprob = api.sample(x, u, math.inf, 0, 1.0, m)
        assert token.tolist() == [int(float(v) * vocab) for v in u], m  # (sums of ones are exact)
        assert torch.equal(logprob, torch.full((5,), -math.log(vocab), device=DEV))
        order = x.float().argsort(dim=1, descending=True, stable=True)[:, :64].sort(dim=1).values
        token, _ = api.sample(x, u, math.inf, 64, 1.0, m)
        assert token.tolist() == [int(order[r, int(float(u[r]) * 64)]) for r in range(5)], m
