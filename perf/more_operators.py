"""The operators of a long answer over a bounded cache, case by case.

  weigh   the attention weight that a call's rows give each cached token, summed per KV head and added
          to what the token has gathered so far (over requests' own pages, and over shared prefixes)
  evict   a request's cache cut to a budget: per KV head the first, the last and the heaviest tokens
          stay, in order, at the front of the request's pages
  sample  the next token of every row of logits: temperature, top-k, top-p and min-p, drawn with a
          given uniform number a row

`own` False computes them in elementary torch operations, rounded once at the end (in 32 bits; sampling
in 64, where a cumulated sum stands next to a border); `own` True makes the calls of this package.  Head
counts are those of the library's workloads: 32 over 8 of 128, 28 over 4 of 128, 16 over 2 of 128, 4 over
2 of 64.
"""
import math
import random

import torch

own = False

SHAPES = [(32, 8, 128), (28, 4, 128), (16, 2, 128), (4, 2, 64)]


def _weigh(name, shape, nq, past, block, groups=0, members=(1, 1), prefix=(0, 0)):
    """groups 0: members[1] requests of their own; else groups of requests that share a prefix."""
    hq, hkv, d = SHAPES[shape]
    return {"name": name, "op": "weigh", "hq": hq, "hkv": hkv, "d": d, "block": block, "lens": 1,
            "groups": groups, "mem_lo": members[0], "mem_hi": members[1], "pre_lo": prefix[0], "pre_hi": prefix[1],
            "nq_lo": nq[0], "nq_hi": nq[1], "past_lo": past[0], "past_hi": past[1]}


def _evict(name, shape, n_req, length, keep, first, last, block):
    hq, hkv, d = SHAPES[shape]
    return {"name": name, "op": "evict", "hq": hq, "hkv": hkv, "d": d, "block": block, "lens": 2, "n_req": n_req,
            "len_lo": length[0], "len_hi": length[1], "keep": keep, "first": first, "last": last}


def _sample(name, rows, vocab, dtype, temperature, top_k, top_p, min_p, each=False):
    """each: the filters are given row by row, some rows without one."""
    return {"name": name, "op": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "temperature": temperature,
            "top_k": top_k, "top_p": top_p, "min_p": min_p, "each": each}


def listed():
    return [
        # one answer token over one repaired request of 10 chunks of 512 tokens: latency
        _weigh("weigh_one", 0, (1, 1), (5120, 5120), 16),
        # one answer token of each request of the batched workload: K at bandwidth
        _weigh("weigh_batch", 0, (1, 1), (6144, 10240), 16, members=(16, 16)),
        # one question over one repaired request, odd group of 7 heads
        _weigh("weigh_question", 1, (77, 77), (6411, 6411), 64),
        # a long prompt piece over a cached context: the tensor cores and the exponentials
        _weigh("weigh_prompt", 0, (2048, 2048), (8192, 8192), 16),
        # 64 answers over one shared document set, next token of each
        _weigh("weigh_shared", 0, (1, 1), (30, 250), 16, 1, (64, 64), (5120, 5120)),
        # a small cache of small heads cut by half: latency
        _evict("evict_small", 3, 1, (611, 611), 301, 4, 32, 16),
        # one repaired request cut to 2048 tokens
        _evict("evict_one", 0, 1, (5120, 5120), 2048, 4, 64, 16),
        # the batched workload cut to 4096 tokens each: rows moved at bandwidth
        _evict("evict_batch", 0, 16, (6144, 10240), 4096, 4, 256, 16),
        # one answer token: latency
        _sample("sample_one", 1, 131072, "f32", 0.8, 50, 0.95, 0.0),
        # a step of 64 answers, every filter, row by row
        _sample("sample_batch", 64, 100003, "f32", 0.9, 200, 0.9, 0.05, each=True),
        # plain temperature over a small odd vocabulary in bf16
        _sample("sample_plain", 16, 32003, "bf16", 1.0, 0, 1.0, 0.0),
        # a large batch, top-p alone: every logit counts
        _sample("sample_large", 512, 131072, "f32", 1.0, 0, 0.9, 0.0),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))) - 0.5))))


def _range(rng, lo, hi):
    """(lo, hi) of ragged sizes: one size, or from a part of the largest up to it."""
    top = _log(rng, lo, hi)
    return (top, top) if rng.random() < 0.4 else (max(lo, int(top * rng.uniform(0.2, 0.9))), top)


def draw(rng):
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    while True:
        op = rng.choice(["weigh", "weigh", "evict", "sample"])
        shape, block = rng.randrange(len(SHAPES)), rng.choice([8, 16, 16, 32, 64, 128, 256])
        if op == "weigh":
            nq = (1, 1) if rng.random() < 0.4 else _range(rng, 1, 2048)
            past = _range(rng, 1, 65536)
            if rng.random() < 0.4:
                c = _weigh("", shape, nq, past, block, _log(rng, 1, 8), _range(rng, 1, 64), _range(rng, 16, 65536))
            else:
                n = _log(rng, 1, 128)
                c = _weigh("", shape, nq, past, block, members=(n, n))
            if c["mem_hi"] * max(1, c["groups"]) > 256:
                continue
        elif op == "evict":
            length = _range(rng, 16, 131072)
            c = _evict("", shape, _log(rng, 1, 128), length, max(1, int(length[1] * rng.uniform(0.1, 1.05))),
                       rng.choice([0, 1, 4, 64]), rng.choice([0, 1, 32, 100, 512]), block)
        else:
            temperature = rng.choice([0.0, 0.3, 0.7, 1.0, 1.0, 1.5])
            c = _sample("", _log(rng, 1, 512), _log(rng, 512, 262144), rng.choice(["f32", "f32", "bf16"]), temperature,
                        rng.choice([0, 0, _log(rng, 1, 2000)]), rng.choice([1.0, round(rng.uniform(0.3, 0.99), 3)]),
                        rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.2), 3)]), rng.random() < 0.4)
        del c["name"]
        c["lens"] = rng.randrange(1 << 20)
        w = work(c)
        if any(w[k] > most[k] for k in most) or _held(c) > 12e9:
            continue
        return c


def _lengths(c):
    """The case's ragged sizes: part of the case, the same for every seed of the values."""
    r = random.Random(c["lens"] * 7919 + 17)
    if c["op"] == "evict":
        return {"own": [r.randint(c["len_lo"], c["len_hi"]) for _ in range(c["n_req"])]}
    members = [r.randint(c["mem_lo"], c["mem_hi"]) for _ in range(max(1, c["groups"]))]
    prefix = [r.randint(c["pre_lo"], c["pre_hi"]) for _ in range(c["groups"])]
    nq = [r.randint(c["nq_lo"], c["nq_hi"]) for _ in range(sum(members))]
    return {"members": members, "prefix": prefix, "nq": nq,
            "own": [r.randint(c["past_lo"], c["past_hi"]) + n for n in nq]}


def _held(c):
    """What the plain form and the cache hold at most, so that a drawn case leaves room for three states."""
    if c["op"] == "sample":
        return c["rows"] * c["vocab"] * 60
    n = _lengths(c)
    row = c["hkv"] * c["d"] * 2
    if c["op"] == "evict":
        return 4 * sum(n["own"]) * row
    total = 4 * (sum(n["own"]) + sum(n["prefix"])) * row
    total += len(n["nq"]) * max(n["own"]) * (c["hkv"] * c["d"] * 4 + 2 * max(n["nq"]) * c["hq"] * 4)
    if c["groups"]:
        rows = max(n["members"]) * max(n["nq"])
        total += c["groups"] * max(n["prefix"]) * (c["hkv"] * c["d"] * 4 + 2 * rows * c["hq"] * 4)
    return total


def work(case):
    c = case
    if c["op"] == "sample":
        size = 4 if c["dtype"] == "f32" else 2
        # the logits once; of each a difference, a scaling, an exponential and a sum
        return {"bytes": c["rows"] * (c["vocab"] * size + 16), "flops": 4 * c["rows"] * c["vocab"]}
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    n = _lengths(c)
    if c["op"] == "evict":
        total = 0
        for length in n["own"]:
            keep = min(length, c["keep"])
            total += hkv * 4 * length if keep < length else 0          # the weights
            moved = max(0, keep - c["first"]) if keep < length else 0
            total += hkv * (2 * moved * (4 * d + 4) + 4 * keep)        # K, V and the weight in and out, the index
        return {"bytes": total, "flops": 0}
    seen, rows, request = 0, 0, 0
    for g, m in enumerate(n["members"]):
        for _ in range(m):
            q, o = n["nq"][request], n["own"][request]
            seen += q * ((n["prefix"][g] if c["groups"] else 0) + o) - q * (q - 1) // 2
            rows += q
            request += 1
    keys = sum(n["prefix"]) + sum(n["own"])
    # q and lse of every row, K and the gathered weight of every token
    return {"bytes": rows * hq * (2 * d + 4) + keys * hkv * (2 * d + 8), "flops": (2 * d + 3) * hq * seen}


def _pages(lengths, free, block):
    """Block table [n, most blocks] int32 of lengths' sequences, taken from the shuffled list `free`; -1 past a
    sequence's end."""
    need = [-(-x // block) for x in lengths]
    n = torch.tensor(need, device="cuda")
    at = torch.cumsum(n, 0) - n
    col = torch.arange(max(1, max(need)), device="cuda")
    has = col[None] < n[:, None]
    table = torch.where(has, free[torch.where(has, at[:, None] + col[None], 0)], -1).to(torch.int32)
    return table, free[sum(need):]


def _slots(s, table, most):
    """Slots of the first `most` tokens of each table row [n, most] (0 past a row's end)."""
    at = torch.arange(most, device="cuda")
    block = s["case"]["block"]
    return table.long()[:, at // block].clamp(min=0) * block + at % block


def _normal(gen, *shape, scale=None, dtype=torch.bfloat16):
    x = torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)
    return (x if scale is None else x.mul_(scale)).to(dtype)


def _cache(gen, slots, width):
    """Two planes of a layer: K with a few outlier channels eight times the others, as the library's caches have."""
    k_scale = torch.where(torch.rand(width, generator=gen, device="cuda") < 0.01, 8.0, 1.0)
    cache = torch.empty(2, slots, width, dtype=torch.bfloat16, device="cuda")
    step = max(1, (1 << 26) // width)
    for a in range(0, slots, step):         # in pieces: the 32-bit draws of a large cache are not kept
        b = min(slots, a + step)
        cache[0, a:b] = _normal(gen, b - a, width, scale=k_scale)
        cache[1, a:b] = _normal(gen, b - a, width)
    return cache


def _prepare_sample(c, gen, s):
    n, v = c["rows"], c["vocab"]
    dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    s["logits"] = torch.empty(n, v, dtype=dtype, device="cuda")
    for a in range(0, n, 64):
        b = min(n, a + 64)
        x = torch.randn(b - a, v, generator=gen, device="cuda").mul_(2.0)
        # a few dozen tokens that the context speaks for, and some that the vocabulary does not have
        likely = torch.randint(0, v, (b - a, 48), generator=gen, device="cuda")
        x.scatter_add_(1, likely, torch.randn(b - a, 48, generator=gen, device="cuda").abs_().mul_(5.0))
        x[:, v - v // 97:] = -math.inf
        s["logits"][a:b] = x.to(dtype)
    s["uniform"] = torch.rand(n, generator=gen, device="cuda")
    par = {k: c[k] for k in ("temperature", "top_k", "top_p", "min_p")}
    if c["each"]:
        def some(value, off, kind):
            drop = torch.rand(n, generator=gen, device="cuda") < 0.25
            return torch.where(drop, off, value).to(kind)
        par = {"temperature": some(par["temperature"], 0.0, torch.float32), "top_k": some(par["top_k"], 0, torch.int32),
               "top_p": some(par["top_p"], 1.0, torch.float32), "min_p": some(par["min_p"], 0.0, torch.float32)}
    s["par"] = par
    s["token"] = torch.empty(n, dtype=torch.int64, device="cuda")
    s["logp"] = torch.empty(n, dtype=torch.float32, device="cuda")


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = {"case": c}
    if c["op"] == "sample":
        _prepare_sample(c, gen, s)
        if own:
            from paper_2609_35139_gb300 import AnswerSession, cr
            cache = torch.empty(2, 16, 128, dtype=torch.bfloat16, device="cuda")
            s["session"] = AnswerSession(cr.target_dims(1, 2, 64, 256, "bf16"), 4, cache, max_tokens=c["rows"])
        return s
    hq, hkv, d, block = c["hq"], c["hkv"], c["d"], c["block"]
    n = _lengths(c)
    pre = n.get("prefix", [])
    slots = (sum(-(-x // block) for x in n["own"] + pre) + 7) * block
    free = torch.randperm(slots // block, generator=gen, device="cuda")
    s["cache"] = _cache(gen, slots, hkv * d)
    s["table"], free = _pages(n["own"], free, block)
    s["own_len"] = torch.tensor(n["own"], dtype=torch.int32, device="cuda")
    s["own_most"] = max(n["own"])
    # what the tokens have gathered so far: spread over many octaves, some nothing at all (a few rows' weights,
    # so that what a call adds counts beside it)
    s["weights"] = torch.randn(hkv, slots, generator=gen, device="cuda").mul_(2.0).exp_().div_(s["own_most"])
    s["weights"][torch.rand(hkv, slots, generator=gen, device="cuda") < 0.03] = 0.0
    tokens, requests = 1, len(n["own"])
    if c["op"] == "evict":
        s["keep"] = torch.full((requests,), c["keep"], dtype=torch.int32, device="cuda")
        s["kept"] = torch.full((requests, hkv, c["keep"]), -1, dtype=torch.int32, device="cuda")
        s["new_len"] = torch.empty(requests, dtype=torch.int32, device="cuda")
    else:
        cu = [0]
        for x in n["nq"]:
            cu.append(cu[-1] + x)
        s["cu_q"], tokens = cu, cu[-1]
        s["q"] = _normal(gen, tokens, hq * d, scale=1.5)
        s["scale"] = 1.0 / math.sqrt(d)
        # the batch's shape as index tensors, for the plain form: token of (request, i)
        lo, nq = torch.tensor(cu[:-1], device="cuda"), torch.tensor(n["nq"], device="cuda")
        i = torch.arange(max(n["nq"]), device="cuda")
        s["tok"] = torch.where(i[None] < nq[:, None], lo[:, None] + i[None], -1)
        s["nq"] = nq
        if c["groups"]:
            s["ptable"], free = _pages(pre, free, block)
            s["prefix_len"] = torch.tensor(pre, dtype=torch.int32, device="cuda")
            s["prefix_most"] = max(pre)
            cg = [0]
            for m in n["members"]:
                cg.append(cg[-1] + m)
            s["cu_group"] = cg
            lo_g, hi_g = (torch.tensor([cu[g] for g in x], device="cuda") for x in (cg[:-1], cg[1:]))
            i = torch.arange(int((hi_g - lo_g).max()), device="cuda")
            s["gtok"] = torch.where(i[None] < (hi_g - lo_g)[:, None], lo_g[:, None] + i[None], -1)
        # the rows' log-sum-exp, as the attention call has given it
        s["lse"] = torch.logaddexp(*(_plain_lse(s, w) for w in (0, 1))) if c["groups"] else _plain_lse(s, 0)
    if own:
        from paper_2609_35139_gb300 import AnswerSession, cr
        s["session"] = AnswerSession(cr.target_dims(1, hkv, d, hq * d, "bf16"), hq, s["cache"], block_size=block,
                                     max_tokens=tokens, max_requests=requests)
        if c["op"] == "weigh":
            s["batch"] = s["session"].batch(s["cu_q"], s.get("cu_group"))
    return s


def run(state):
    s, c = state, state["case"]
    if c["op"] == "sample":
        if own:
            s["session"].sample(s["logits"], s["uniform"], **s["par"], out=s["token"], logp=s["logp"])
        else:
            _plain_sample(s)
        return {"token": s["token"], "logp": s["logp"]}
    if c["op"] == "evict":
        if own:
            s["session"].evict(0, s["table"], s["own_len"], s["keep"], s["weights"], c["keep"], first=c["first"],
                               last=c["last"], kept=s["kept"], new_len=s["new_len"])
        else:
            _plain_evict(s)
        return {"k": s["cache"][0], "v": s["cache"][1], "weights": s["weights"], "kept": s["kept"],
                "new_len": s["new_len"]}
    if own:
        more = {"prefix_table": s["ptable"], "prefix_len": s["prefix_len"]} if c["groups"] else {}
        s["session"].weigh(0, s["batch"], s["q"], s["lse"], s["table"], s["own_len"], s["weights"], **more)
    else:
        _plain_weigh(s, 0)
        if c["groups"]:
            _plain_weigh(s, 1)
    return {"weights": s["weights"]}


# ------------------------------------------------------------------ plain forms
def _plain_scores(s, which):
    """Scores of the requests' rows over their own tokens (which 0), or of the groups' over their prefixes (1),
    in 32 bits: [n, hkv, rows, group, most], -inf where a row does not see a token; the rows' tokens; slots."""
    c = s["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    table, tok, most = (s["ptable"], s["gtok"], s["prefix_most"]) if which else (s["table"], s["tok"], s["own_most"])
    n, rows = tok.shape
    slots = _slots(s, table, most)
    k = s["cache"][0][slots].float().view(n, most, hkv, d).permute(0, 2, 3, 1)
    q = s["q"].float().view(-1, hkv, hq // hkv, d)[tok.clamp(min=0)].permute(0, 2, 1, 3, 4)
    score = (q.reshape(n, hkv, -1, d) * s["scale"]) @ k
    j = torch.arange(most, device="cuda")
    if which:
        seen = (j[None, None] < s["prefix_len"][:, None, None]) & (tok >= 0)[:, :, None]
    else:
        limit = (s["own_len"] - s["nq"])[:, None] + torch.arange(rows, device="cuda")[None] + 1
        seen = (j[None, None] < limit[:, :, None]) & (tok >= 0)[:, :, None]
    score = score.view(n, hkv, rows, hq // hkv, most)
    return score.masked_fill_(~seen[:, None, :, None], -math.inf), tok, slots


def _plain_lse(s, which):
    score, tok, _ = _plain_scores(s, which)
    lse = torch.logsumexp(score, 4).permute(0, 2, 1, 3).reshape(*tok.shape, -1)      # [n, rows, hq]
    out = torch.empty(s["q"].shape[0], lse.shape[2], device="cuda")
    out[tok[tok >= 0]] = lse[tok >= 0]
    return out


def _plain_weigh(s, which):
    score, tok, slots = _plain_scores(s, which)
    n, hkv, rows, g, most = score.shape
    lse = s["lse"][tok.clamp(min=0)].view(n, rows, hkv, g).transpose(1, 2)
    w = score.sub_(lse[..., None]).exp_().sum((2, 3))                                 # [n, hkv, most]
    j = torch.arange(most, device="cuda")
    length = s["prefix_len"] if which else s["own_len"]
    there = j[None] < length[:, None]
    old = there if which else j[None] < (s["own_len"] - s["nq"])[:, None]
    at = slots[there]
    base = torch.where(old[there][None], s["weights"][:, at], 0.0)
    s["weights"][:, at] = base + w.transpose(0, 1)[:, there]


def _plain_evict(s):
    c = s["case"]
    hkv, d = c["hkv"], c["d"]
    lengths = _lengths(c)["own"]
    slots = _slots(s, s["table"], s["own_most"])
    s["new_len"].copy_(torch.minimum(s["own_len"], s["keep"]))
    planes = s["cache"].view(2, -1, hkv, d)
    heads = torch.arange(hkv, device="cuda")[:, None]
    for r, n in enumerate(lengths):
        if n <= c["keep"]:
            s["kept"][r, :, :n] = torch.arange(n, dtype=torch.int32, device="cuda")
            continue
        last = min(c["last"], c["keep"])
        first = min(c["first"], c["keep"] - last)
        at = slots[r, :n]
        stays = torch.zeros(hkv, n, dtype=torch.bool, device="cuda")
        stays[:, :first] = True
        stays[:, n - last:] = True
        order = torch.sort(s["weights"][:, at[first:n - last]], dim=1, descending=True, stable=True).indices
        stays[heads, first + order[:, :c["keep"] - first - last]] = True
        kept = stays.nonzero()[:, 1].view(hkv, c["keep"])
        s["kept"][r] = kept.to(torch.int32)
        src, dst = at[kept], at[None, :c["keep"]].expand(hkv, -1)
        for x in (planes[0], planes[1]):
            x[dst, heads] = x[src, heads]
        s["weights"][heads, dst] = s["weights"][heads, src]


def _plain_sample(s):
    n, v = s["logits"].shape
    x = s["logits"].double()
    full = lambda p: (p if torch.is_tensor(p) else torch.full((n,), p, device="cuda"))[:, None]
    temperature, top_k = full(s["par"]["temperature"]).double(), full(s["par"]["top_k"]).long()
    top_p, min_p = full(s["par"]["top_p"]), full(s["par"]["min_p"])
    # (a parameter is a 32-bit number)
    temperature, top_p, min_p = (p.float().double() for p in (temperature, top_p, min_p))
    top, best = x.max(1, keepdim=True)
    best = (x == top).to(torch.int8).argmax(1, keepdim=True)
    w = ((x - top) / torch.where(temperature > 0, temperature, 1.0)).exp_()
    del x
    # ranks: descending, ties by the lowest index
    ranked, order = torch.sort(w, dim=1, descending=True, stable=True)
    rank = torch.arange(v, device="cuda")[None]
    ranked.masked_fill_((top_k > 0) & (rank >= top_k), 0.0)
    before = torch.cumsum(ranked, 1)
    total = before[:, -1:].clone()
    before.sub_(ranked)
    keep = (before < top_p * total) | (top_p >= 1) | (rank == 0)
    keep &= ranked >= min_p
    ranked.masked_fill_(~keep, 0.0)
    w = torch.zeros_like(w).scatter_(1, order, ranked)
    del ranked, order, before, keep
    cum = torch.cumsum(w, 1)
    total = cum[:, -1:]
    hit = (cum > s["uniform"].double()[:, None] * total).to(torch.int8).argmax(1, keepdim=True)
    token = torch.where(temperature > 0, hit, best)
    s["token"].copy_(token[:, 0])
    s["logp"].copy_(torch.where(temperature > 0, (w.gather(1, token) / total).log(), 0.0)[:, 0])


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"weigh": _exact_weigh, "evict": _exact_evict, "sample": _exact_sample}[case["op"]](s)


def _exact_weigh(s):
    c = s["case"]
    if work(c)["flops"] > 2e12:
        return None
    hq, hkv, d, block = c["hq"], c["hkv"], c["d"], c["block"]
    g = hq // hkv
    n = _lengths(c)
    w = s["weights"].double()

    def add(table, length, a, b, causal):
        if length == 0 or a == b:
            return
        at = torch.arange(length, device="cuda")
        slot = table[at.div(block, rounding_mode="floor")].long() * block + at.remainder(block)
        key = s["cache"][0][slot].view(length, hkv, d)
        fresh = b - a if causal else 0
        w[:, slot[length - fresh:]] = 0.0
        step = max(1, int(2e8 // (length * g)))
        for h in range(hkv):
            kh = key[:, h].double()
            for i in range(a, b, step):
                e = min(b, i + step)
                q = s["q"][i:e].view(e - i, hq, d)[:, h * g:(h + 1) * g].double()
                x = torch.einsum("igd,jd->igj", q, kh) / math.sqrt(d) - s["lse"][i:e, h * g:(h + 1) * g].double()[..., None]
                if causal:
                    late = at[None] > (length - b + torch.arange(i, e, device="cuda"))[:, None]
                    x.masked_fill_(late[:, None], -math.inf)
                w[h, slot] += torch.exp(x).sum((0, 1))

    cu, request = s["cu_q"], 0
    for grp, m in enumerate(n["members"]):
        if c["groups"]:
            add(s["ptable"][grp], n["prefix"][grp], cu[request], cu[request + m], False)
        for _ in range(m):
            add(s["table"][request], n["own"][request], cu[request], cu[request + 1], True)
            request += 1
    return {"weights": w}


def _exact_evict(s):
    """Copies: the heaviest by a threshold and a count of its ties instead of a sort."""
    c = s["case"]
    hkv, d, block, keep = c["hkv"], c["d"], c["block"], c["keep"]
    k, v = s["cache"][0].double().view(-1, hkv, d), s["cache"][1].double().view(-1, hkv, d)
    w, kept = s["weights"].double(), s["kept"].clone()
    lens = _lengths(c)["own"]
    for r, n in enumerate(lens):
        at = torch.arange(n, device="cuda")
        slot = s["table"][r][at.div(block, rounding_mode="floor")].long() * block + at.remainder(block)
        if n <= keep:
            kept[r, :, :n] = at.to(torch.int32)
            continue
        last = min(c["last"], keep)
        first = min(c["first"], keep - last)
        rest = keep - first - last
        for h in range(hkv):
            x = w[h, slot].clone()
            x[:first], x[n - last:] = math.inf, math.inf
            if rest:
                least = torch.kthvalue(x, n - keep + 1).values
                chosen = x > least
                ties = x == least
                chosen |= ties & (torch.cumsum(ties.int(), 0) <= keep - int(chosen.sum()))
            else:
                chosen = x == math.inf
            idx = torch.nonzero(chosen).flatten()
            kept[r, h] = idx.to(torch.int32)
            src, dst = slot[idx], slot[:keep]
            k[dst, h], v[dst, h], w[h, dst] = k[src, h].clone(), v[src, h].clone(), w[h, src].clone()
    return {"k": k.view(-1, hkv * d), "v": v.view(-1, hkv * d), "weights": w, "kept": kept,
            "new_len": torch.tensor([min(n, keep) for n in lens], dtype=torch.int32, device="cuda")}


def _exact_sample(s):
    """Row by row, the cuts found as thresholds."""
    n, v = s["logits"].shape
    token, logp = torch.empty(n, dtype=torch.int64), torch.zeros(n, dtype=torch.float64)
    host = {k: (p.tolist() if torch.is_tensor(p) else [torch.tensor(p).item()] * n) for k, p in s["par"].items()}
    u = s["uniform"].tolist()
    for r in range(n):
        x = s["logits"][r].double()
        t, k, p, m = (host[name][r] for name in ("temperature", "top_k", "top_p", "min_p"))
        if t <= 0:
            token[r] = int(torch.nonzero(x == x.max())[0])
            continue
        inside = torch.ones(v, dtype=torch.bool, device="cuda")

        def cut(least, most):
            """Keep what is above `least` and the first of its equals, `most` in all."""
            above, equal = inside & (x > least), inside & (x == least)
            return above | (equal & (torch.cumsum(equal.int(), 0) <= most - int(above.sum())))

        if 0 < k < v:
            inside = cut(torch.topk(x, k).values[-1], k)
        w = torch.softmax(x / t, 0)
        if p < 1:
            has = torch.sort(x[inside], descending=True).values
            mass = torch.cumsum(torch.exp((has - has[0]) / t), 0)
            number = 1 + int((mass[:-1] < p * mass[-1]).sum())       # those whose predecessors stay below p
            inside = cut(has[number - 1], number)
        if m > 0:
            inside &= torch.exp((x - x.max()) / t) >= m
        w = torch.where(inside, w, 0.0)
        cum = torch.cumsum(w, 0)
        token[r] = int(torch.searchsorted(cum, torch.tensor([u[r]], dtype=torch.float64, device="cuda") * cum[-1],
                                          right=True))
        logp[r] = float(torch.log(w[token[r]] / cum[-1]))
    return {"token": token.cuda(), "logp": logp.cuda()}
