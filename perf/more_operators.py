"""Cases on which the operators of a bounded cache and of the end of a decode step are measured: the attention weight
that cached tokens have received (`weigh`), the choice of the tokens that stay (`keep`), their move to the front of
the sequence's pages (`compact`), and the choice of the next token from its logits (`sample`).  `own = False` computes
them with elementary torch operations, `own = True` with the kernels of this package."""
import math
import random

import torch

own = False


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one new token of one sequence: the smallest call
        dict(name="weigh-one-2k", op="weigh", batch=1, qmin=1, qmax=1, kvmin=2047, kvmax=2047, page=64, fp8=False, hq=64, hkv=8, decay=1.0,
             lens=1),
        # a decode step of a large ragged batch, older steps fading
        dict(name="weigh-decode64", op="weigh", batch=64, qmin=1, qmax=1, kvmin=1, kvmax=32000, page=64, fp8=False, hq=64, hkv=8, decay=0.98,
             lens=2),
        # the last tokens of prompts as observers of what goes before them, fp8 cache, uneven windows, pages of 16
        dict(name="weigh-window-fp8", op="weigh", batch=6, qmin=17, qmax=48, kvmin=8000, kvmax=32000, page=16, fp8=True, hq=64, hkv=4, decay=0.0,
             lens=3),
        # all queries of a prefill chunk on a long cache: the largest
        dict(name="weigh-chunk4096", op="weigh", batch=1, qmin=4096, qmax=4096, kvmin=28672, kvmax=28672, page=64, fp8=False, hq=64, hkv=8,
             decay=1.0, lens=4),
        # caches at their budget drop the tokens of the last steps that nobody looked at
        dict(name="keep-decode32", op="keep", batch=32, kvmin=4160, kvmax=4160, page=64, hkv=8, budget=4096, sinks=4, recent=256, lens=5),
        # long prompts are cut down to a small budget
        dict(name="keep-prompts", op="keep", batch=3, kvmin=60000, kvmax=262144, page=128, hkv=8, budget=2048, sinks=16, recent=32, lens=6),
        # the moves that belong to the two choices
        dict(name="compact-decode32", op="compact", batch=32, kvmin=4160, kvmax=4160, page=64, fp8=False, hkv=8, budget=4096, sinks=4, recent=256,
             lens=7),
        dict(name="compact-prompts-fp8", op="compact", batch=3, kvmin=30000, kvmax=65536, page=16, fp8=True, hkv=8, budget=2048, sinks=16, recent=32,
             lens=8),
        # one sequence with the usual filters: latency
        dict(name="sample-one", op="sample", rows=1, vocab=131072, kind="bf16", spread=3.0, temperature=0.8, top_k=50, top_p=0.9, min_p=0.0,
             each=False),
        # a decode step whose requests bring their own settings; odd vocabulary
        dict(name="sample-each96", op="sample", rows=96, vocab=100003, kind="bf16", spread=3.0, temperature=0.9, top_k=200, top_p=0.9, min_p=0.02,
             each=True),
        # nucleus of a flat distribution, no limit on the count
        dict(name="sample-nucleus33", op="sample", rows=33, vocab=50001, kind="fp16", spread=1.5, temperature=1.1, top_k=0, top_p=0.95, min_p=0.0,
             each=False),
        # rollouts: the whole distribution, fp32 logits
        dict(name="sample-rollout256", op="sample", rows=256, vocab=131072, kind="fp32", spread=2.0, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0,
             each=False),
    ]


def _spread(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["weigh", "weigh", "keep", "compact", "sample", "sample"])
    if op == "sample":
        vocab = _spread(rng, 500, 200000)
        return dict(op=op, rows=_spread(rng, 1, min(512, 33554432 // vocab)), vocab=vocab, kind=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                    spread=rng.choice([1.0, 2.0, 3.0, 5.0]), temperature=rng.choice([0.3, 0.7, 1.0, 1.5]),
                    top_k=rng.choice([0, 1, 20, 50, 1000]), top_p=rng.choice([1.0, 0.5, 0.9, 0.99]), min_p=rng.choice([0.0, 0.0, 0.05]),
                    each=rng.random() < 0.5)
    hq, hkv = rng.choice([(64, 8), (64, 4), (32, 8), (16, 2)])
    case = dict(op=op, page=rng.choice([16, 32, 64, 128]), hkv=hkv, lens=rng.randrange(1 << 30))
    if op == "weigh":
        case.update(fp8=rng.random() < 0.4, hq=hq, decay=rng.choice([0.0, 0.9, 1.0]))
        kind = rng.choice(["decode", "few", "chunk"])
        if kind == "decode":
            case.update(batch=_spread(rng, 1, 64), qmin=1, qmax=1)
        elif kind == "few":
            case.update(batch=_spread(rng, 1, 24), qmin=1, qmax=rng.randint(2, 48))
        else:
            q = _spread(rng, 49, 4096)
            case.update(batch=rng.randint(1, max(1, min(6, 4096 // q))), qmin=max(1, q // 2), qmax=q)
        top = _spread(rng, 64, 28672)
        return dict(case, kvmin=rng.randint(0, top), kvmax=top)
    budget = _spread(rng, 64, 4096)
    top = _spread(rng, budget, 16 * budget)
    case.update(batch=_spread(rng, 1, max(1, min(64, 130000 // top))), kvmin=rng.randint(1, top), kvmax=top, budget=budget,
                sinks=rng.choice([0, 1, 4, 16]), recent=rng.choice([0, 1, 31, budget // 4]))
    return dict(case, fp8=rng.random() < 0.4) if op == "compact" else case


D = 128  # head size


def _lens(case):
    """(new tokens, tokens before them) of each sequence."""
    r = random.Random(case["lens"])
    return [(r.randint(case.get("qmin", 0), case.get("qmax", 0)), r.randint(case["kvmin"], case["kvmax"])) for _ in range(case["batch"])]


def work(case):
    if case["op"] == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * (4 if case["kind"] == "fp32" else 2) + case["rows"] * (16 + (16 if case["each"] else 0)), "flops": 4 * n}
    lens, hkv = _lens(case), case["hkv"]
    kv = sum(n + c for n, c in lens)
    lists = 4 * (len(lens) + kv // case["page"])
    if case["op"] == "weigh":
        new = sum(n for n, _ in lens)
        pairs = sum(n * c + n * (n + 1) // 2 for n, c in lens)
        old = 0 if case["decay"] == 0 else sum(c for _, c in lens)
        return {"bytes": new * case["hq"] * (2 * D + 4) + kv * hkv * (D * (1 if case["fp8"] else 2) + 4) + old * hkv * 4 + lists,
                "flops": 2 * D * case["hq"] * pairs}
    kept = sum(min(c, case["budget"]) for _, c in lens)
    if case["op"] == "keep":
        return {"bytes": 4 * hkv * (kv + case["batch"] * case["budget"]) + lists, "flops": kv * hkv}
    # every kept token behind the first dropped one moves; the first of n dropped among m stands at about m / (n + 1)
    moved = 0
    for _, c in lens:
        stay, drop = min(c, case["budget"]), max(0, c - case["budget"])
        first = min(stay, case["sinks"]) + max(0, c - case["recent"] - case["sinks"]) // (drop + 1)
        moved += max(0, stay - first) if drop else 0
    return {"bytes": hkv * (moved * (4 * D * (1 if case["fp8"] else 2) + 8) + 4 * kept) + lists, "flops": 0}


# ----------------------------------------------------------------------------------------- inputs
KINDS = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _take(pool, table):
    """Rows of a pool's pages (any type of element) of every sequence: [batch, pages, ...]."""
    return pool.view(torch.uint8)[table].view(pool.dtype)


def _plain_lse(s):
    """The log-sum-exp that attention has returned for the queries: fp32 [rows, heads]."""
    c, cu, lens = s["case"], s["cu_q"].tolist(), s["kv_lens"].tolist()
    g = c["hq"] // c["hkv"]
    lse = torch.empty(s["q"].shape[:2], device="cuda")
    for i, n in enumerate(lens):
        new = cu[i + 1] - cu[i]
        k = _take(s["k_pool"], s["table"][i].long()).flatten(0, 1)[:n].float()
        hidden = torch.arange(n, device="cuda") > torch.arange(n - new, n, device="cuda")[:, None]
        for h in range(c["hkv"]):
            q = s["q"][cu[i]:cu[i + 1], h * g:(h + 1) * g].float() * D ** -0.5
            score = torch.matmul(q.transpose(0, 1), k[:, h].T).masked_fill_(hidden, -math.inf)
            lse[cu[i]:cu[i + 1], h * g:(h + 1) * g] = score.logsumexp(-1).T
    return lse


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed * 7919 + 29)
    s = dict(case=case)
    if case["op"] == "sample":
        rows = case["rows"]
        # a head of a few likely tokens over the bulk
        x = case["spread"] * torch.randn(rows, case["vocab"], generator=g, device=dev)
        x += 2 * case["spread"] * (torch.rand(rows, case["vocab"], generator=g, device=dev) < 2e-4)
        s["logits"] = x.to(KINDS[case["kind"]])
        s["u"] = torch.rand(rows, generator=g, device=dev)
        for name in ("temperature", "top_k", "top_p", "min_p"):
            s[name] = case[name]
            if case["each"]:  # every request has its own: the case's, or less, or the filter off
                r = torch.rand(rows, generator=g, device=dev)
                off = {"temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0}[name]
                v = torch.where(r < 0.2, torch.full_like(r, off), case[name] * (1 - 0.3 * r))
                s[name] = v.round().to(torch.int32) if name == "top_k" else v
        return s
    lens, hkv = _lens(case), case["hkv"]
    total = [n + c for n, c in lens]
    s["cu_q"] = torch.tensor([sum(n for n, _ in lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device=dev)
    s["kv_lens"] = torch.tensor(total, dtype=torch.int32, device=dev)
    # every sequence has pages of its own up to its length; the rest of its row of the table is unused
    used = [-(-n // case["page"]) for n in total]
    pages = sum(used) + 3
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    s["table"] = torch.zeros(len(lens), max(used), dtype=torch.int32, device=dev)
    at = 0
    for i, u in enumerate(used):
        s["table"][i, :u] = order[at:at + u]
        at += u
    # most tokens have received little, a few a lot
    s["weights"] = torch.rand(pages, hkv, case["page"], generator=g, device=dev).pow_(6).mul_(8)
    kind = torch.float8_e4m3fn if case.get("fp8") else torch.bfloat16
    shape = (pages, case["page"], hkv, D)
    if case["op"] == "keep":
        # the choice reads no keys: a program has the pool all the same
        s["k_pool"] = torch.empty(shape, dtype=kind, device=dev)
        return s
    s["k_pool"] = torch.randn(shape, generator=g, device=dev, dtype=torch.bfloat16).to(kind)
    if case["op"] == "weigh":
        s["q"] = (2 * torch.randn(sum(n for n, _ in lens), case["hq"], D, generator=g, device=dev)).bfloat16()
        s["lse"] = _plain_lse(s)
        return s
    s["v_pool"] = torch.randn(shape, generator=g, device=dev, dtype=torch.bfloat16).to(kind)
    s["keep"] = _keep(s)["keep"]
    return s


# ------------------------------------------------------------------------------------- plain forms
def _weigh(s):
    c = s["case"]
    b, hkv, g = c["batch"], c["hkv"], c["hq"] // c["hkv"]
    table, cu, kv = s["table"].long(), s["cu_q"].long(), s["kv_lens"].long()
    length = table.shape[1] * c["page"]
    dev = table.device
    row = torch.arange(s["q"].shape[0], device=dev)
    seq = torch.searchsorted(cu[1:], row, right=True)
    at = (seq, row - cu[seq])
    new = cu[1:] - cu[:-1]
    q = torch.zeros(b, c["qmax"], hkv, g, D, device=dev)
    q[at] = s["q"].float().unflatten(1, (hkv, g)) * D ** -0.5
    lse = torch.full((b, c["qmax"], hkv, g), math.inf, device=dev)  # (no query: no weight)
    lse[at] = s["lse"].unflatten(1, (hkv, g))
    place = torch.arange(length, device=dev)
    last = kv[:, None] - new[:, None] + torch.arange(c["qmax"], device=dev)  # position of each query
    k = _take(s["k_pool"], table).float().reshape(b, length, hkv, D)
    score = torch.matmul(q.permute(0, 2, 3, 1, 4).reshape(b, hkv, -1, D), k.permute(0, 2, 3, 1)).view(b, hkv, g, c["qmax"], length)
    score.sub_(lse.permute(0, 2, 3, 1)[..., None]).masked_fill_((place > last[..., None])[:, None, None], -math.inf)
    got = score.exp_().sum((2, 3))
    old = s["weights"][table].permute(0, 2, 1, 3).reshape(b, hkv, length)
    fresh = place >= (kv - new)[:, None]  # tokens of this call start at nothing
    old = torch.where(fresh[:, None], torch.zeros_like(old), old) * c["decay"]
    i, j = (place < kv[:, None]).nonzero(as_tuple=True)
    s["weights"][table[i, j // c["page"]], :, j % c["page"]] = (old + got)[i, :, j]
    return {"weights": s["weights"]}


def _keep(s):
    c = s["case"]
    b, hkv, budget = c["batch"], c["hkv"], c["budget"]
    table, kv = s["table"].long(), s["kv_lens"].long()
    w = s["weights"][table].permute(0, 2, 1, 3).reshape(b, hkv, -1)
    place = torch.arange(w.shape[2], device=w.device)
    n = kv.clamp(max=budget)
    recent = n.clamp(max=c["recent"])
    sinks = torch.minimum(n - recent, torch.full_like(n, c["sinks"]))
    w = torch.where(((place < sinks[:, None]) | (place >= (kv - recent)[:, None]))[:, None], torch.full_like(w, math.inf), w)
    w = torch.where((place >= kv[:, None])[:, None], torch.full_like(w, -math.inf), w)
    order = w.sort(dim=-1, descending=True, stable=True).indices[..., :budget]
    order = torch.nn.functional.pad(order, (0, budget - order.shape[-1]))
    order = torch.where((torch.arange(budget, device=w.device) < n[:, None])[:, None], order, torch.full_like(order, w.shape[2]))
    order = order.sort(dim=-1).values
    return {"keep": torch.where(order == w.shape[2], torch.full_like(order, -1), order).to(torch.int32), "lens": n.to(torch.int32)}


def _compact(s):
    c = s["case"]
    b, h, to = (s["keep"] >= 0).nonzero(as_tuple=True)
    source = s["keep"].long()[b, h, to]
    table = s["table"].long()
    src, src_slot, dst, dst_slot = table[b, source // c["page"]], source % c["page"], table[b, to // c["page"]], to % c["page"]
    k, v, w = s["k_pool"].view(torch.uint8), s["v_pool"].view(torch.uint8), s["weights"]
    k[dst, dst_slot, h], v[dst, dst_slot, h], w[dst, h, dst_slot] = k[src, src_slot, h], v[src, src_slot, h], w[src, h, src_slot]
    return {"k_pool": s["k_pool"], "v_pool": s["v_pool"], "weights": s["weights"]}


def _column(v, like):
    """A setting of every row, in 64 bits."""
    return v.double()[:, None] if torch.is_tensor(v) else torch.full((like.shape[0], 1), v, dtype=torch.float64, device=like.device)


def _sample(s):
    x = s["logits"].double()
    temperature, top_k, top_p, min_p = [_column(s[n], x) for n in ("temperature", "top_k", "top_p", "min_p")]
    # (settings are fp32 numbers wherever they come from)
    temperature, top_p, min_p = [v.float().double() for v in (temperature, top_p, min_p)]
    z, index = x.sort(dim=-1, descending=True, stable=True)
    z = (z - z[:, :1]) / temperature
    w = z.exp()
    w = torch.where((top_k > 0) & (torch.arange(x.shape[1], device=x.device) >= top_k), torch.zeros_like(w), w)
    total = w.cumsum(-1)
    w = torch.where((top_p < 1) & (total - w >= top_p * total[:, -1:]), torch.zeros_like(w), w)
    w = torch.where(z < min_p.log(), torch.zeros_like(w), w)
    # back in the order of the vocabulary
    w = torch.zeros_like(w).scatter_(1, index, w)
    upto = w.cumsum(-1)
    total = upto[:, -1:]
    token = (upto <= s["u"].double()[:, None] * total).sum(-1, keepdim=True)
    logprob = (w.gather(1, token) / total).log()
    return {"token": token[:, 0], "logprob": logprob[:, 0].float()}


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2606_13392_b200 import api
        if op == "sample":
            token, logprob = api.sample(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
            return {"token": token, "logprob": logprob}
        cache = api.PagedCache(s["k_pool"], s.get("v_pool"), s["table"], s["kv_lens"], s["cu_q"])
        if op == "weigh":
            return {"weights": api.paged_weights(cache, s["q"], s["lse"], s["weights"], s["case"]["decay"])}
        if op == "keep":
            keep, lens = api.paged_keep(cache, s["weights"], s["case"]["budget"], s["case"]["sinks"], s["case"]["recent"])
            return {"keep": keep, "lens": lens}
        api.paged_compact(cache, s["keep"], s["weights"])
        return {"k_pool": s["k_pool"], "v_pool": s["v_pool"], "weights": s["weights"]}
    return {"weigh": _weigh, "keep": _keep, "compact": _compact, "sample": _sample}[op](s)


# ------------------------------------------------------------------------------------ definition
def exact(case, seed):
    """The operators' definitions in 64 bits, sequence by sequence and head by head, or row by row."""
    s = prepare(case, seed)
    if case["op"] == "sample":
        tokens, logprobs = [], []
        for r in range(case["rows"]):
            t, k, p, m = [float(torch.as_tensor(v[r] if torch.is_tensor(v) else v, dtype=torch.float32))
                          for v in (s["temperature"], s["top_k"], s["top_p"], s["min_p"])]
            x = s["logits"][r].double()
            prob = torch.softmax(x / t, 0)
            live = torch.argsort(x, descending=True, stable=True)
            if k > 0:
                live = live[:int(k)]
            if p < 1:
                mass = prob[live].cumsum(0)
                live = live[:int((mass < p * mass[-1]).sum()) + 1]
            if m > 0:
                live = live[x[live] >= x.max() + t * math.log(m)]
            live = live.sort().values
            mass = prob[live].cumsum(0)
            j = min(int((mass <= float(s["u"][r]) * mass[-1]).sum()), len(live) - 1)
            tokens.append(live[j])
            logprobs.append((prob[live[j]] / mass[-1]).log())
        return {"token": torch.stack(tokens), "logprob": torch.stack(logprobs)}
    lens, table, page = s["kv_lens"].tolist(), s["table"].long(), case["page"]
    if case["op"] == "keep":
        keep = torch.full((case["batch"], case["hkv"], case["budget"]), -1, dtype=torch.int32, device="cuda")
        for i, n in enumerate(lens):
            stay = min(n, case["budget"])
            recent = min(case["recent"], stay)
            sinks = min(case["sinks"], stay - recent)
            for h in range(case["hkv"]):
                w = s["weights"][table[i], h].flatten()[sinks:n - recent].double()
                best = torch.argsort(w, descending=True, stable=True)[:stay - recent - sinks] + sinks
                ends = torch.cat([torch.arange(sinks, device="cuda"), torch.arange(n - recent, n, device="cuda")])
                keep[i, h, :stay] = torch.cat([best, ends]).sort().values.int()
        return {"keep": keep, "lens": torch.tensor([min(n, case["budget"]) for n in lens], dtype=torch.int32)}
    if case["op"] == "compact":
        if work(case)["bytes"] > 2e9 or case["batch"] * case["hkv"] > 600:
            return None
        pools = [s["k_pool"].double(), s["v_pool"].double()]
        weights = s["weights"].double()
        for i in range(case["batch"]):
            for h in range(case["hkv"]):
                source = s["keep"][i, h]
                source = source[source >= 0].long()
                to = torch.arange(len(source), device="cuda")
                moved = [p[table[i][source // page], source % page, h].clone() for p in pools]
                for p, m in zip(pools, moved):
                    p[table[i][to // page], to % page, h] = m
                weights[table[i][to // page], h, to % page] = weights[table[i][source // page], h, source % page].clone()
        return {"k_pool": pools[0], "v_pool": pools[1], "weights": weights}
    if work(case)["flops"] > 2e13:
        return None
    cu, g = s["cu_q"].tolist(), case["hq"] // case["hkv"]
    weights = s["weights"].double()
    for i, n in enumerate(lens):
        new = cu[i + 1] - cu[i]
        place = torch.arange(n, device="cuda")
        k = _take(s["k_pool"], table[i]).flatten(0, 1)[:n]
        seen = place <= torch.arange(n - new, n, device="cuda")[:, None]
        for h in range(case["hkv"]):
            w = weights[table[i][place // page], h, place % page]
            w = torch.where(place < n - new, case["decay"] * w, torch.zeros_like(w))
            kh = k[:, h].double()
            for head in range(h * g, (h + 1) * g):
                logit = s["q"][cu[i]:cu[i + 1], head].double() @ kh.T / math.sqrt(D)
                w += torch.where(seen, torch.exp(logit - s["lse"][cu[i]:cu[i + 1], head].double()[:, None]), 0.0).sum(0)
            weights[table[i][place // page], h, place % page] = w
    return {"weights": weights}
