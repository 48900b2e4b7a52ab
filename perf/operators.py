"""Cases on which the serving and training operators around sparse attention are measured: norms of queries and
keys with the position rotation (forward and gradient), appending to a paged K/V cache, and attention of new
tokens over that cache.  `own = False` computes them with elementary torch operations, `own = True` with the
kernels of this package."""
import math
import random

import torch

own = False

EPS = 1e-6


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a decode step of 32 sequences deep in their contexts: latency
        dict(name="rope-decode32", op="rope", tokens=32, hq=64, hkv=8, d=128, rot=64, inter=False, norm=True, yarn=1.0),
        # a prefill chunk of a model that was stretched to long contexts
        dict(name="rope-prefill32k", op="rope", tokens=32768, hq=64, hkv=8, d=128, rot=128, inter=False, norm=True, yarn=8.0),
        # the index branch's heads (8 query heads, one key head of 64), rotation alone, odd row count
        dict(name="rope-index10007", op="rope", tokens=10007, hq=8, hkv=1, d=64, rot=32, inter=True, norm=False, yarn=1.0),
        # training: gradients of a micro-batch of 8192 tokens
        dict(name="grad-8k", op="grad", tokens=8192, hq=64, hkv=4, d=128, rot=128, inter=False, norm=True, yarn=1.0),
        # training: a short ragged micro-batch, other pair layout, half of the head turned
        dict(name="grad-1537", op="grad", tokens=1537, hq=64, hkv=8, d=128, rot=64, inter=True, norm=True, yarn=4.0),
        # a decode step's append: one token for each of 32 sequences
        dict(name="append-decode32", op="append", batch=32, qmin=1, qmax=1, kvmin=1, kvmax=8192, page=64, fp8=False, hq=64, hkv=8,
             d=128, rot=64, inter=False, norm=True, yarn=1.0, lens=3),
        # a ragged batch of prefill chunks onto an fp8 cache of small pages
        dict(name="append-chunks-fp8", op="append", batch=6, qmin=700, qmax=2500, kvmin=0, kvmax=1500, page=16, fp8=True, hq=64, hkv=8,
             d=128, rot=128, inter=True, norm=True, yarn=8.0, lens=4),
        # one token of one sequence: the smallest call
        dict(name="attn-one-2k", op="attn", batch=1, qmin=1, qmax=1, kvmin=2047, kvmax=2047, page=64, fp8=False, hq=64, hkv=8, d=128, lens=5),
        # a decode step of a large ragged batch
        dict(name="attn-decode64", op="attn", batch=64, qmin=1, qmax=1, kvmin=1, kvmax=32000, page=64, fp8=False, hq=64, hkv=8, d=128, lens=6),
        # the same on an fp8 cache with four KV heads
        dict(name="attn-decode32-fp8", op="attn", batch=32, qmin=1, qmax=1, kvmin=4000, kvmax=32000, page=128, fp8=True, hq=64, hkv=4, d=128,
             lens=7),
        # a few new tokens of every sequence (drafted tokens being verified, odd lengths) on small pages
        dict(name="attn-verify16", op="attn", batch=16, qmin=2, qmax=7, kvmin=500, kvmax=16000, page=16, fp8=False, hq=64, hkv=8, d=128, lens=8),
        # a prefill chunk over a long cache: the largest
        dict(name="attn-chunk4096", op="attn", batch=1, qmin=4096, qmax=4096, kvmin=28672, kvmax=28672, page=64, fp8=False, hq=64, hkv=8,
             d=128, lens=9),
    ]


def _spread(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["rope", "grad", "append", "attn", "attn", "attn"])
    hq, hkv, d = rng.choice([(64, 8, 128), (64, 4, 128), (32, 8, 128), (16, 2, 128), (64, 8, 128)])
    turn = dict(rot=rng.choice([d, d // 2, d // 4]), inter=rng.random() < 0.5, norm=rng.random() < 0.75, yarn=rng.choice([1.0, 4.0, 8.0]))
    if op in ("rope", "grad"):
        if rng.random() < 0.2:
            hq, hkv, d = rng.choice([(8, 1, 64), (4, 1, 64), (4, 1, 128)])
            turn["rot"] = d // 2
        return dict(op=op, tokens=_spread(rng, 1, 32768 if op == "rope" else 8192), hq=hq, hkv=hkv, d=d, **turn)
    case = dict(op=op, page=rng.choice([16, 32, 64, 128]), fp8=rng.random() < 0.4, hq=hq, hkv=hkv, d=d, lens=rng.randrange(1 << 30))
    kind = rng.choice(["decode", "few", "chunk"])
    if kind == "decode":
        case.update(batch=_spread(rng, 1, 64), qmin=1, qmax=1)
    elif kind == "few":
        case.update(batch=_spread(rng, 1, 32), qmin=1, qmax=rng.randint(2, 9))
    else:
        q = _spread(rng, 33, 4096)
        case.update(batch=rng.randint(1, max(1, min(6, 4096 // q))), qmin=max(1, q // 2), qmax=q)
    if op == "append":
        return dict(case, kvmin=0, kvmax=_spread(rng, 64, 4096), **turn)
    top = _spread(rng, 64, 28672)
    return dict(case, kvmin=rng.randint(1, top), kvmax=top)


def _lens(case):
    """(new tokens, tokens before them) of each sequence."""
    r = random.Random(case["lens"])
    return [(r.randint(case["qmin"], case["qmax"]), r.randint(case["kvmin"], case["kvmax"])) for _ in range(case["batch"])]


def work(case):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] in ("rope", "grad"):
        rows = case["tokens"] * (hq + hkv) * d
        small = case["tokens"] * 8 + case["rot"] * 4 + (4 * d if case["norm"] else 0)
        if case["op"] == "rope":
            return {"bytes": 4 * rows + small, "flops": rows * (10 if case["norm"] else 4)}
        return {"bytes": 6 * rows + small + (8 * d if case["norm"] else 0), "flops": rows * (20 if case["norm"] else 4)}
    lens = _lens(case)
    new, elt = sum(n for n, _ in lens), 1 if case["fp8"] else 2
    kv = sum(n + c for n, c in lens)
    if case["op"] == "append":
        return {"bytes": new * d * (4 * hq + 2 * hkv * (2 + elt)) + 4 * (2 * len(lens) + new), "flops": new * d * (hq + hkv) * 10}
    pairs = sum(n * c + n * (n + 1) // 2 for n, c in lens)
    return {"bytes": new * hq * (4 * d + 4) + kv * hkv * d * 2 * elt + 4 * (2 * len(lens) + kv // case["page"]), "flops": 4 * d * hq * pairs}


# ----------------------------------------------------------------------------------------- inputs
def _frequencies(rot, factor, dev):
    """Radians per position of each pair (base 10000 x 500), interpolated between stretched and plain frequencies by
    wavelength as for a context `factor` times the 32768 tokens of training, and the factor on the rotated values."""
    i = torch.arange(rot // 2, dtype=torch.float64, device=dev)
    f = 5e6 ** (-2.0 * i / rot)
    turns = 32768.0 * f / (2 * math.pi)
    keep = ((turns - 1.0) / 31.0).clamp(0.0, 1.0)
    return f * keep + f / factor * (1 - keep), 0.1 * math.log(factor) + 1.0


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed * 7919 + 17)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    s = dict(case=case)
    if "rot" in case:
        s["freqs"], s["mscale"] = _frequencies(case["rot"], case["yarn"], dev)
        w = [(1 + 0.3 * torch.randn(d, generator=g, device=dev)).bfloat16() for _ in range(2)]
        s["wq"], s["wk"] = w if case["norm"] else (None, None)
    if case["op"] in ("rope", "grad"):
        n = case["tokens"]
        start = int(torch.randint(0, (1 << 20) - n, (1,), generator=g, device=dev))
        s["pos"] = torch.arange(start, start + n, device=dev) if n > 64 else torch.randint(0, 1 << 20, (n,), generator=g, device=dev)
    else:
        lens = _lens(case)
        n = sum(x for x, _ in lens)
        s["max_q"] = max(x for x, _ in lens)
        s["cu_q"] = torch.tensor([sum(x for x, _ in lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=dev)
        s["kv_lens"] = torch.tensor([x + c for x, c in lens], dtype=torch.int32, device=dev)
        need = max(-(-(x + c) // case["page"]) for x, c in lens)
        # every sequence has pages of its own up to its length; the rest of its row of the table is unused
        used = [-(-(x + c) // case["page"]) for x, c in lens]
        pages = sum(used) + 3
        order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
        s["table"] = torch.zeros(len(lens), need, dtype=torch.int32, device=dev)
        at = 0
        for i, u in enumerate(used):
            s["table"][i, :u] = order[at:at + u]
            at += u
        shape = (pages, case["page"], hkv, d)
        kind = torch.float8_e4m3fn if case["fp8"] else torch.bfloat16
        s["k_pool"], s["v_pool"] = [torch.randn(shape, generator=g, device=dev, dtype=torch.bfloat16).to(kind) for _ in range(2)]
    if case["op"] == "attn":
        s["q"] = (2 * torch.randn(n, hq, d, generator=g, device=dev)).bfloat16()
        return s
    # queries, keys and values come as slices of one projection's output
    qkv = torch.randn(n, (hq + 2 * hkv) * d, generator=g, device=dev, dtype=torch.bfloat16)
    s["q"], s["k"], s["v"] = [x.unflatten(1, (-1, d)) for x in qkv.split([hq * d, hkv * d, hkv * d], 1)]
    if case["op"] == "grad":
        s["dq"] = torch.randn(n, hq, d, generator=g, device=dev, dtype=torch.bfloat16)
        s["dk"] = torch.randn(n, hkv, d, generator=g, device=dev, dtype=torch.bfloat16)
    return s


# ------------------------------------------------------------------------------------- plain forms
def _pairs(x, rot, inter):
    return (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])


def _joined(a, b, rest, inter):
    return torch.cat([torch.stack([a, b], -1).flatten(-2) if inter else torch.cat([a, b], -1), rest], -1)


def _cos_sin(pos, s):
    angle = pos.double()[:, None] * s["freqs"]
    return (angle.cos() * s["mscale"]).float()[:, None], (angle.sin() * s["mscale"]).float()[:, None]


def _rope(x, w, pos, s):
    rot, inter = s["case"]["rot"], s["case"]["inter"]
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    cos, sin = _cos_sin(pos, s)
    a, b = _pairs(x, rot, inter)
    return _joined(a * cos - b * sin, a * sin + b * cos, x[..., rot:], inter)


def _rope_grad(dy, x, w, pos, s):
    rot, inter = s["case"]["rot"], s["case"]["inter"]
    dy = dy.float()
    cos, sin = _cos_sin(pos, s)
    a, b = _pairs(dy, rot, inter)
    g = _joined(a * cos + b * sin, b * cos - a * sin, dy[..., rot:], inter)
    if w is None:
        return g.bfloat16(), None
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    x = x * r
    gw = g * w.float()
    return (r * (gw - x * (gw * x).mean(-1, keepdim=True))).bfloat16(), (g * x).sum((0, 1))


def _rows(s):
    """Sequence and position of each new token."""
    cu = s["cu_q"].long()
    i = torch.arange(s["q"].shape[0], device=cu.device)
    seq = torch.searchsorted(cu[1:], i, right=True)
    return seq, i - cu[1:][seq] + s["kv_lens"].long()[seq]


def _append(s):
    seq, pos = _rows(s)
    page = s["case"]["page"]
    at = s["table"].long()[seq, pos // page] * page + pos % page
    # (only the bytes are stored below: an fp8 value is stored as the nearest one, the largest where it is beyond)
    for pool, x in ((s["k_pool"], _rope(s["k"], s["wk"], pos, s)), (s["v_pool"], s["v"].float())):
        x = x.clamp(-448, 448) if s["case"]["fp8"] else x
        pool.view(torch.uint8).flatten(0, 1).index_copy_(0, at, x.to(pool.dtype).view(torch.uint8))
    return {"q": _rope(s["q"], s["wq"], pos, s).bfloat16(), "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _attn(s):
    c, (seq, pos) = s["case"], _rows(s)
    b, g = c["batch"], c["hq"] // c["hkv"]
    table = s["table"].long()
    length = table.shape[1] * c["page"]
    k, v = [pool.view(torch.uint8)[table].view(pool.dtype).float().reshape(b, length, c["hkv"], c["d"]) for pool in (s["k_pool"], s["v_pool"])]
    at = (seq, torch.arange(pos.shape[0], device=pos.device) - s["cu_q"].long()[seq])
    q = torch.zeros(b, s["max_q"], c["hkv"], g, c["d"], device=k.device)
    q[at] = s["q"].float().unflatten(1, (c["hkv"], g)) * c["d"] ** -0.5
    last = torch.full((b, s["max_q"]), length, device=k.device)
    last[at] = pos
    score = torch.matmul(q.permute(0, 2, 3, 1, 4).reshape(b, c["hkv"], -1, c["d"]), k.permute(0, 2, 3, 1))
    score = score.view(b, c["hkv"], g, s["max_q"], length)
    score.masked_fill_((torch.arange(length, device=k.device) > last[..., None])[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    total = score.sub_(top).exp_().sum(-1, keepdim=True)
    out = torch.matmul(score.view(b, c["hkv"], -1, length), v.transpose(1, 2)).view(b, c["hkv"], g, s["max_q"], c["d"]) / total
    lse = (top + total.log()).squeeze(-1)
    return {"out": out.permute(0, 3, 1, 2, 4)[at].flatten(1, 2).bfloat16(), "lse": lse.permute(0, 3, 1, 2)[at].flatten(1, 2)}


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2606_13392_b200 import api
        if op == "attn":
            out, lse = api.paged_attn(api.PagedCache(s["k_pool"], s["v_pool"], s["table"], s["kv_lens"], s["cu_q"]), s["q"])
            return {"out": out, "lse": lse}
        rope = api.Rope(s["freqs"], s["case"]["inter"], s["mscale"])
        if op == "append":
            cache = api.PagedCache(s["k_pool"], s["v_pool"], s["table"], s["kv_lens"], s["cu_q"])
            q = api.paged_append(cache, s["k"], s["v"], s["q"], rope, s["wq"], s["wk"], EPS)
            return {"q": q, "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
        if op == "rope":
            q, k = api.qk_norm_rope(s["q"], s["k"], s["pos"], rope, s["wq"], s["wk"], EPS)
            return {"q": q, "k": k}
        dq, dk, dwq, dwk = api.qk_norm_rope_backward(s["dq"], s["dk"], s["q"], s["k"], s["pos"], rope, s["wq"], s["wk"], EPS)
        return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}
    if op == "attn":
        return _attn(s)
    if op == "append":
        return _append(s)
    if op == "rope":
        return {"q": _rope(s["q"], s["wq"], s["pos"], s).bfloat16(), "k": _rope(s["k"], s["wk"], s["pos"], s).bfloat16()}
    dq, dwq = _rope_grad(s["dq"], s["q"], s["wq"], s["pos"], s)
    dk, dwk = _rope_grad(s["dk"], s["k"], s["wk"], s["pos"], s)
    return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}


# ------------------------------------------------------------------------------------ definition
def exact(case, seed):
    """The operators' definitions in 64 bits: a pair (a, b) at position p becomes (a + ib) exp(i p f), gradients come
    from the definition by automatic differentiation, attention goes sequence by sequence and head by head."""
    s = prepare(case, seed)
    d = case["d"]

    def turned(x, w, pos):
        if w is not None:
            x = w.double() * x / (x.square().sum(-1, keepdim=True) / d + EPS).sqrt()
        half = case["rot"] // 2
        first = torch.arange(half, device=x.device) * (2 if case["inter"] else 1)
        second = first + (1 if case["inter"] else half)
        z = torch.complex(x[..., first], x[..., second])
        angle = pos.double().unsqueeze(1) * s["freqs"]
        z = z * torch.polar(torch.full_like(angle, s["mscale"]), angle).unsqueeze(1)
        y = x.clone()
        y[..., first], y[..., second] = z.real, z.imag
        return y

    if case["op"] == "rope":
        return {"q": turned(s["q"].double(), s["wq"], s["pos"]), "k": turned(s["k"].double(), s["wk"], s["pos"])}
    if case["op"] == "grad":
        found = {}
        for n in "qk":
            x = s[n].double().requires_grad_()
            w = None if s["w" + n] is None else s["w" + n].double().requires_grad_()
            turned(x, w, s["pos"]).backward(s["d" + n].double())
            found["d" + n], found["dw" + n] = x.grad, None if w is None else w.grad
        return found
    cu, kv, page = s["cu_q"].tolist(), s["kv_lens"].tolist(), case["page"]
    if case["op"] == "append":
        pools = [s["k_pool"].double(), s["v_pool"].double()]
        q = []
        for i in range(case["batch"]):
            rows = slice(cu[i], cu[i + 1])
            pos = torch.arange(kv[i] - (cu[i + 1] - cu[i]), kv[i], device="cuda")
            q.append(turned(s["q"][rows].double(), s["wq"], pos))
            where = s["table"][i].long()[pos // page]
            pools[0][where, pos % page] = turned(s["k"][rows].double(), s["wk"], pos)
            pools[1][where, pos % page] = s["v"][rows].double()
        return {"q": torch.cat(q), "k_pool": pools[0], "v_pool": pools[1]}
    if work(case)["flops"] > 2e13:
        return None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    group = case["hq"] // case["hkv"]
    for i in range(case["batch"]):
        tokens = torch.arange(kv[i], device="cuda")
        hidden = tokens > torch.arange(kv[i] - (cu[i + 1] - cu[i]), kv[i], device="cuda").unsqueeze(1)
        where = s["table"][i].long()[tokens // page]
        for h in range(case["hq"]):
            k = s["k_pool"].view(torch.uint8).view(s["k_pool"].shape[:3] + (-1,))[where, tokens % page, h // group].view(s["k_pool"].dtype).double()
            v = s["v_pool"].view(torch.uint8).view(s["v_pool"].shape[:3] + (-1,))[where, tokens % page, h // group].view(s["v_pool"].dtype).double()
            logit = (s["q"][cu[i]:cu[i + 1], h].double() @ k.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
            lse[cu[i]:cu[i + 1], h] = torch.logsumexp(logit, 1)
            out[cu[i]:cu[i + 1], h] = torch.softmax(logit, 1) @ v
    return {"out": out, "lse": lse}
