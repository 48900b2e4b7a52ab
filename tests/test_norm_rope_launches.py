"""Launch shapes of the norm and rotation kernel: every documented size launches and agrees with the definition in 64
bits (tolerances as in test_norm_rope.py), and the rule asks for no more shared memory than a launch gets.

A token's coefficients take 2 * lanes * 64 bytes of a CTA's shared memory, so few heads - which make a CTA prepare many
tokens at a time - are the sizes where the request is largest."""

import pytest
import torch

from paper_2606_13392_b200 import api
from paper_2606_13392_b200 import binding as B
from test_norm_rope import make, turn
from test_paged_append import rows_of

DEV = "cuda"
SHARED = 48 * 1024  # what a launch gets without asking for more
STATIC = 32 * 16    # positions and places of a CTA's tokens


def close(y, ref, eps=2.0 ** -8, least=0.0):
    tol = eps * ref.abs() + 2.0 ** -15 * ref.abs().amax(-1, keepdim=True) + least
    assert (y.double() - ref).abs().le(tol).all()


def test_the_rule_stays_within_a_launch():
    seen = set()
    for d in (8, 40, 64, 72, 96, 128, 136, 192, 256):
        for heads in ((1, 0, 0), (0, 1, 0), (0, 1, 1), (4, 1, 0), (8, 1, 0), (16, 0, 0), (8, 4, 0), (0, 8, 8), (16, 2, 2), (64, 8, 0), (64, 8, 8),
                      (1024, 1024, 1024)):
            for n in (1, 2, 31, 600, 4736, 7089, 9473, 14177, 16384, 32768, 100000, 1 << 22, (1 << 31) - 1):
                tile, grid, parts, shared = B.msa_norm_rope_plan(d, *heads, n)
                assert 1 <= tile <= 32 and shared + STATIC <= SHARED, (d, heads, n, tile, shared)
                assert 1 <= grid < 1 << 31 and 1 <= parts < 1 << 16
                assert (grid - 1) * tile < n  # no CTA without tokens
                seen.add(tile)
    assert len(seen) > 3
    with pytest.raises(B.MsaError):
        B.msa_norm_rope_plan(100, 1, 1, 0, 5)
    with pytest.raises(B.MsaError):
        B.msa_norm_rope_plan(128, -1, 1, 0, 5)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,hq,hk,d,rot,inter,norm", [
    (16384, 8, 1, 128, 128, False, True), (32768, 8, 1, 128, 64, True, True), (16411, 4, 1, 128, 64, False, False),
    (14177, 16, 0, 128, 128, False, True), (8192, 8, 1, 256, 256, False, True), (7089, 8, 4, 256, 64, True, True),
    (40001, 8, 1, 64, 32, True, False), (20000, 1, 1, 96, 96, False, True), (20000, 3, 1, 192, 64, False, True)])
def test_few_heads_many_tokens(rows, hq, hk, d, rot, inter, norm):
    q, k, wq, wk, positions, freqs = make(rows, hq, hk, d, rot, norm, False, True)
    outs = api.qk_norm_rope(q, k, positions, api.Rope(freqs, inter, 1.2), wq, wk, 1e-5)
    for x, w, y in ((q, wq, outs[0]), (k, wk, outs[1])):
        if x is not None:
            close(y, turn(x.double(), None if w is None else w.double(), positions, freqs, inter, 1.2, 1e-5))


@pytest.mark.gpu
@pytest.mark.parametrize("heads,d,values,fp8", [(8, 128, True, False), (16, 128, False, True), (4, 256, True, True), (1, 128, False, False)])
def test_append_without_queries(heads, d, values, fp8):
    lens, page = [(9000, 0), (0, 50), (7384, 1000)], 64
    n, kind = sum(x for x, _ in lens), torch.float8_e4m3fn if fp8 else torch.bfloat16
    pages = 290
    pools = [torch.zeros(pages, page, heads, d, dtype=kind, device=DEV) for _ in range(1 + values)]
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(3)).to(torch.int32)
    table = torch.full((3, 142), -7, dtype=torch.int32)
    table[0, :141], table[1, :1], table[2, :132] = order[:141], order[141:142], order[142:274]
    cache = api.PagedCache(pools[0], pools[1] if values else None, table.to(DEV),
                           torch.tensor([x + c for x, c in lens], dtype=torch.int32, device=DEV),
                           torch.tensor([0, 9000, 9000, n], dtype=torch.int32, device=DEV))
    k, v = rows_of(n, heads, d, 1), rows_of(n, heads, d, 2) if values else None
    w = (1 + 0.3 * torch.randn(d, device=DEV)).bfloat16()
    freqs = api.rope_frequencies(d // 2, 1e6)
    assert api.paged_append(cache, k, v, None, api.Rope(freqs, False, 1.1), None, w, 1e-5) is None
    assert B.check_async_status() == (0, 0)
    positions = torch.cat([torch.arange(c, c + x) for x, c in lens])
    seq = torch.repeat_interleave(torch.arange(3), torch.tensor([x for x, _ in lens]))
    at = (table[seq, positions // page].long() * page + positions % page).to(DEV)
    ref = turn(k.double(), w.double(), positions.to(DEV), freqs, False, 1.1, 1e-5)
    close(pools[0].view(torch.uint8).flatten(0, 1)[at].view(kind), ref, *((2.0 ** -4, 2.0 ** -10) if fp8 else ()))
    if values:
        assert torch.equal(pools[1].view(torch.uint8).flatten(0, 1)[at], v.to(kind).contiguous().view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hk,d,rot,inter,norm,tokens", [(64, 8, 128, 64, False, True, 9600), (8, 1, 128, 128, True, True, 19200),
                                                           (2, 1, 64, 64, False, False, 38400)])
def test_more_tokens_than_ctas_hold_at_a_time(hq, hk, d, rot, inter, norm, tokens):
    # a CTA's second round: the coefficients and positions of the first are overwritten behind the barrier that ends it
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    rows = tokens * sms // 148 + 3
    tile, ctas, parts, _ = B.msa_norm_rope_plan(d, hq, hk, 0, rows)
    assert tile > 1 and parts == 1 and ctas * tile < rows and rows % tile != 0
    q, k, wq, wk, positions, freqs = make(rows, hq, hk, d, rot, norm, False, True)
    outs = api.qk_norm_rope(q, k, positions, api.Rope(freqs, inter, 1.2), wq, wk, 1e-5)
    for x, w, y in ((q, wq, outs[0]), (k, wk, outs[1])):
        for lo in range(0, rows, 4096):  # (the definition's intermediates are large)
            part = slice(lo, lo + 4096)
            close(y[part], turn(x[part].double(), None if w is None else w.double(), positions[part], freqs, inter, 1.2, 1e-5))


@pytest.mark.gpu
@pytest.mark.parametrize("fp8", [False, True])
def test_an_append_of_more_tokens_than_ctas_hold_at_a_time(fp8):
    hq, heads, d, page = 64, 8, 128, 128
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    n = 9600 * sms // 148 + 3
    tile, ctas, parts, _ = B.msa_norm_rope_plan(d, hq, heads, heads, n)
    assert tile > 1 and parts == 1 and ctas * tile < n and n % tile != 0
    lens = [(n - 700, 100), (0, 9), (699, 0), (1, 77)]
    kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
    used = [-(-(x + c) // page) for x, c in lens]
    order = torch.randperm(sum(used) + 3, generator=torch.Generator().manual_seed(4)).to(torch.int32)
    table = torch.full((4, max(used)), -7, dtype=torch.int32)
    for s, part in enumerate(order[:sum(used)].split(used)):
        table[s, :used[s]] = part
    pools = [torch.zeros(len(order), page, heads, d, dtype=kind, device=DEV) for _ in range(2)]
    cache = api.PagedCache(pools[0], pools[1], table.to(DEV), torch.tensor([x + c for x, c in lens], dtype=torch.int32, device=DEV),
                           torch.tensor([0, n - 700, n - 700, n - 1, n], dtype=torch.int32, device=DEV))
    extra = 5  # rows of a padded batch
    q, k, v = [rows_of(n + extra, h, d, s) for s, h in ((1, hq), (2, heads), (3, heads))]
    wq, wk = [(1 + 0.3 * torch.randn(d, device=DEV)).bfloat16() for _ in range(2)]
    freqs = api.rope_frequencies(64, 1e6)
    q_out = torch.full((n + extra, hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
    api.paged_append(cache, k, v, q, api.Rope(freqs, False, 1.1), wq, wk, 1e-5, q_out)
    assert B.check_async_status() == (0, 0) and (q_out[n:] == 7).all()
    positions = torch.cat([torch.arange(c, c + x) for x, c in lens])
    seq = torch.repeat_interleave(torch.arange(4), torch.tensor([x for x, _ in lens]))
    at = (table[seq, positions // page].long() * page + positions % page).to(DEV)
    positions = positions.to(DEV)
    stored = pools[0].view(torch.uint8).flatten(0, 1)[at].view(kind)
    for lo in range(0, n, 4096):
        part = slice(lo, min(lo + 4096, n))
        close(q_out[part], turn(q[part].double(), wq.double(), positions[part], freqs, False, 1.1, 1e-5))
        close(stored[part], turn(k[part].double(), wk.double(), positions[part], freqs, False, 1.1, 1e-5),
              *((2.0 ** -4, 2.0 ** -10) if fp8 else ()))
    assert torch.equal(pools[1].view(torch.uint8).flatten(0, 1)[at], v[:n].to(kind).contiguous().view(torch.uint8))
    untouched = torch.ones(len(order) * page, dtype=torch.bool, device=DEV)
    untouched[at] = False
    assert not any(p.view(torch.uint8).flatten(0, 1)[untouched].any() for p in pools)
