"""The answering operators, case by case: what a target model does with a repaired, paged cache.

  append  a question's or an answer's new tokens: K rotated to its position and written with V into
          one layer of the paged cache at each token's slot, Q rotated for the attention
  paged   attention of the requests' new tokens over their own pages (causal among the new tokens)
  prefix  the same for requests that share a long prefix (one document set, many questions): the
          prefix's pages are read once for all requests of a group

`own` False computes them in elementary torch operations in 32 bits, rounded once at the end; `own`
True makes the calls of this package.  Head counts are those of the library's workloads (d_model /
head_dim query heads): 32 over 8 of 128, 28 over 4 of 128, 16 over 2 of 128, 4 over 2 of 64.
"""
import math
import random

import torch

own = False

SHAPES = [(32, 8, 128), (28, 4, 128), (16, 2, 128), (4, 2, 64)]


def _append(name, shape, tokens, dtype, block, max_pos, skip):
    hq, hkv, d = SHAPES[shape]
    return {"name": name, "op": "append", "hq": hq, "hkv": hkv, "d": d, "block": block, "lens": 1,
            "tokens": tokens, "dtype": dtype, "max_pos": max_pos, "skip": skip}


def _paged(name, shape, n_req, nq, past, block):
    hq, hkv, d = SHAPES[shape]
    return {"name": name, "op": "paged", "hq": hq, "hkv": hkv, "d": d, "block": block, "lens": 2,
            "n_req": n_req, "nq_lo": nq[0], "nq_hi": nq[1], "past_lo": past[0], "past_hi": past[1]}


def _prefix(name, shape, groups, members, prefix, nq, past, block):
    hq, hkv, d = SHAPES[shape]
    return {"name": name, "op": "prefix", "hq": hq, "hkv": hkv, "d": d, "block": block, "lens": 3,
            "groups": groups, "mem_lo": members[0], "mem_hi": members[1], "pre_lo": prefix[0],
            "pre_hi": prefix[1], "nq_lo": nq[0], "nq_hi": nq[1], "past_lo": past[0], "past_hi": past[1]}


def listed():
    return [
        # one answer token of one request: nothing but latency
        _append("append_one", 0, 1, "bf16", 16, 5200, 0.0),
        # one answer token of each of 64 requests, a few of them padding (slot -1)
        _append("append_decode_64", 1, 64, "bf16", 16, 8192, 0.1),
        # the questions of a batch, 16 of about 45 tokens, from an fp32 projection
        _append("append_questions", 2, 723, "f32", 32, 2700, 0.0),
        # prompts being prefilled: bandwidth
        _append("append_prompts", 0, 16384, "bf16", 16, 131072, 0.0),
        # one answer token over one repaired request of 10 chunks of 512 tokens
        _paged("decode_one", 0, 1, (1, 1), (5120, 5120), 16),
        # one answer token of each request of the batched workload (16 of 6144 to 10240 tokens)
        _paged("decode_batch", 0, 16, (1, 1), (6144, 10240), 16),
        # one question over one repaired request of 20 ragged chunks, odd group of 7 heads
        _paged("question", 1, 1, (77, 77), (6411, 6411), 64),
        # a long prompt piece over a cached context
        _paged("prompt", 0, 1, (2048, 2048), (8192, 8192), 16),
        # four questions' answers over one small document set, next token of each
        _prefix("shared_small", 2, 1, (4, 4), (2560, 2560), (1, 1), (20, 90), 16),
        # 64 answers over the 10-chunk document set
        _prefix("shared_decode", 0, 1, (64, 64), (5120, 5120), (1, 1), (30, 250), 16),
        # several document sets at once, ragged, up to four tokens a request (drafted tokens)
        _prefix("shared_groups", 1, 4, (9, 17), (2560, 10240), (1, 4), (0, 130), 32),
        # a large batch over a long shared prefix
        _prefix("shared_large", 0, 1, (256, 256), (32768, 32768), (1, 1), (100, 500), 16),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)) ) - 0.5))))


def _range(rng, lo, hi):
    """(lo, hi) of ragged sizes: one size, or from a part of the largest up to it."""
    top = _log(rng, lo, hi)
    return (top, top) if rng.random() < 0.4 else (max(lo, int(top * rng.uniform(0.2, 0.9))), top)


def draw(rng):
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    while True:
        op = rng.choice(["append", "paged", "paged", "prefix", "prefix"])
        shape, block = rng.randrange(len(SHAPES)), rng.choice([8, 16, 16, 32, 64, 128, 256])
        if op == "append":
            c = _append("", shape, _log(rng, 1, 16384), rng.choice(["bf16", "bf16", "f32"]), block,
                        _log(rng, 64, 131072), rng.choice([0.0, 0.0, 0.15]))
        elif op == "paged":
            nq = (1, 1) if rng.random() < 0.5 else _range(rng, 1, 2048)
            c = _paged("", shape, _log(rng, 1, 128), nq, _range(rng, 1, 65536), block)
        else:
            nq = (1, 1) if rng.random() < 0.6 else _range(rng, 1, 64)
            c = _prefix("", shape, _log(rng, 1, 8), _range(rng, 1, 128), _range(rng, 128, 65536), nq,
                        _range(rng, 1, 2048), block)
            if c["mem_hi"] * c["groups"] > 256:
                continue
        del c["name"]
        c["lens"] = rng.randrange(1 << 20)
        w = work(c)
        if any(w[k] > most[k] for k in most) or _plain_bytes(c) > 12e9:
            continue
        return c


def _plain_bytes(c):
    """What the plain form holds at most, so that a drawn case leaves room for three states."""
    if c["op"] == "append":
        return 0
    lens = _lengths(c)
    r, nq, past = len(lens["nq"]), max(lens["nq"]), max(lens["own"])
    total = r * past * c["hkv"] * c["d"] * 8 + 2 * r * nq * c["hq"] * past * 4
    if c["op"] == "prefix":
        g, m, p = c["groups"], max(lens["members"]), max(lens["prefix"])
        total += g * p * c["hkv"] * c["d"] * 8 + 2 * g * m * nq * c["hq"] * p * 4
    return total


def _lengths(c):
    """The case's ragged sizes: part of the case, the same for every seed of the values."""
    r = random.Random(c["lens"] * 7919 + 17)
    if c["op"] == "append":
        return {}
    if c["op"] == "paged":
        members = [1] * c["n_req"]
        prefix = [0] * c["n_req"]
    else:
        members = [r.randint(c["mem_lo"], c["mem_hi"]) for _ in range(c["groups"])]
        prefix = [r.randint(c["pre_lo"], c["pre_hi"]) for _ in range(c["groups"])]
    n = sum(members)
    nq = [r.randint(c["nq_lo"], c["nq_hi"]) for _ in range(n)]
    own_len = [r.randint(c["past_lo"], c["past_hi"]) + nq[i] for i in range(n)]
    return {"members": members, "prefix": prefix, "nq": nq, "own": own_len}


def work(case):
    c = case
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    if c["op"] == "append":
        size = 4 if c["dtype"] == "f32" else 2
        keep = c["tokens"] - int(c["tokens"] * c["skip"])
        # q of every token and k, v of the written ones in and out, position and slot of each
        return {"bytes": c["tokens"] * (hq * d * (size + 2) + 12) + keep * 2 * hkv * d * (size + 2),
                "flops": 3 * d * (c["tokens"] * hq + keep * hkv)}
    n = _lengths(c)
    seen, rows, request = 0, 0, 0
    for g, m in enumerate(n["members"]):
        for _ in range(m):
            q, o = n["nq"][request], n["own"][request]
            seen += q * (n["prefix"][g] + o) - q * (q - 1) // 2
            rows += q
            request += 1
    keys = sum(n["prefix"]) + sum(n["own"])
    return {"bytes": 2 * rows * hq * d * 2 + keys * 2 * hkv * d * 2, "flops": 4 * d * hq * seen}


def _inv_freq(d):
    return [float(torch.tensor(10000.0 ** (-2.0 * i / d), dtype=torch.float32)) for i in range(d // 2)]


def _pages(lengths, free, block, device):
    """Block table [n, most blocks] int32 of lengths' sequences, taken from the shuffled list `free`; -1 past a sequence's end."""
    need = [-(-x // block) for x in lengths]
    width = max(1, max(need))
    n = torch.tensor(need, device=device)
    at = torch.cumsum(n, 0) - n
    col = torch.arange(width, device=device)
    has = col[None] < n[:, None]
    idx = torch.where(has, at[:, None] + col[None], 0)
    table = torch.where(has, free[idx], -1).to(torch.int32)
    return table, free[sum(need):]


def _normal(gen, *shape, scale=None, dtype=torch.bfloat16):
    x = torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)
    return (x if scale is None else x.mul_(scale)).to(dtype)


def prepare(case, seed):
    c = case
    hq, hkv, d, block = c["hq"], c["hkv"], c["d"], c["block"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    width = hkv * d
    # K with a few outlier channels eight times the others, as the library's caches have
    k_scale = torch.where(torch.rand(width, generator=gen, device="cuda") < 0.01, 8.0, 1.0)
    s = {"case": c, "scale": 1.0 / math.sqrt(d), "inv_freq": _inv_freq(d)}
    if c["op"] == "append":
        t = c["tokens"]
        dtype = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        blocks = -(-t // block) + 5
        slots = blocks * block
        s["qkv"] = _normal(gen, t, (hq + 2 * hkv) * d, dtype=dtype)   # one projection's output
        s["qkv"][:, hq * d:(hq + hkv) * d] *= k_scale.to(dtype)
        s["pos"] = torch.randint(0, c["max_pos"], (t,), generator=gen, device="cuda", dtype=torch.int32)
        s["slots"] = torch.randperm(slots, generator=gen, device="cuda")[:t].to(torch.int64)
        drop = int(t * c["skip"])
        s["slots"][torch.randperm(t, generator=gen, device="cuda")[:drop]] = -1
        s["cache"] = _normal(gen, 2, slots, width)
        s["q_out"] = torch.empty(t, hq * d, dtype=torch.bfloat16, device="cuda")
        tokens, requests = t, 1
    else:
        n = _lengths(c)
        need = sum(-(-x // block) for x in n["own"] + n["prefix"])
        blocks = need + 7
        slots = blocks * block
        free = torch.randperm(blocks, generator=gen, device="cuda")
        s["cache"] = torch.empty(2, slots, width, dtype=torch.bfloat16, device="cuda")
        step = max(1, (1 << 26) // width)
        for a in range(0, slots, step):     # in pieces: the 32-bit draws of a large cache are not kept
            b = min(slots, a + step)
            s["cache"][0, a:b] = _normal(gen, b - a, width, scale=k_scale)
            s["cache"][1, a:b] = _normal(gen, b - a, width)
        s["table"], free = _pages(n["own"], free, block, "cuda")
        s["own_len"] = torch.tensor(n["own"], dtype=torch.int32, device="cuda")
        cu = [0]
        for x in n["nq"]:
            cu.append(cu[-1] + x)
        s["cu_q"] = cu
        tokens, requests = cu[-1], len(n["nq"])
        s["q"] = _normal(gen, tokens, hq * d, scale=1.5)
        s["out"] = torch.empty(tokens, hq * d, dtype=torch.bfloat16, device="cuda")
        # the batch's shape as index tensors, for the plain form: token of (request, i), and back
        most = max(n["nq"])
        lo = torch.tensor(cu[:-1], device="cuda")
        nq = torch.tensor(n["nq"], device="cuda")
        i = torch.arange(most, device="cuda")
        s["tok"] = torch.where(i[None] < nq[:, None], lo[:, None] + i[None], 0)
        s["req"] = torch.repeat_interleave(torch.arange(requests, device="cuda"), nq)
        s["idx"] = torch.arange(tokens, device="cuda") - lo[s["req"]]
        s["nq"] = nq
        s["own_most"] = max(n["own"])
        if c["op"] == "prefix":
            s["ptable"], free = _pages(n["prefix"], free, block, "cuda")
            s["prefix_len"] = torch.tensor(n["prefix"], dtype=torch.int32, device="cuda")
            cg = [0]
            for m in n["members"]:
                cg.append(cg[-1] + m)
            s["cu_group"] = cg
            s["prefix_most"] = max(n["prefix"])
            mem = torch.tensor(n["members"], device="cuda")
            first = torch.tensor(cg[:-1], device="cuda")
            j = torch.arange(max(n["members"]), device="cuda")
            s["member"] = torch.where(j[None] < mem[:, None], first[:, None] + j[None], 0)
            s["group"] = torch.repeat_interleave(torch.arange(len(cg) - 1, device="cuda"), mem)
            s["place"] = torch.arange(requests, device="cuda") - first[s["group"]]
    if own:
        from paper_2609_35139_gb300 import AnswerSession, cr
        target = cr.target_dims(1, hkv, d, hq * d, "bf16")
        s["session"] = AnswerSession(target, hq, s["cache"], block_size=block, max_tokens=tokens,
                                     max_requests=requests, inv_freq_target=s["inv_freq"])
        if c["op"] != "append":
            s["batch"] = s["session"].batch(s["cu_q"], s.get("cu_group"))
    return s


def run(state):
    s, c = state, state["case"]
    if c["op"] == "append":
        hq, hkv, d = c["hq"], c["hkv"], c["d"]
        q, k, v = s["qkv"].split([hq * d, hkv * d, hkv * d], dim=1)
        if own:
            s["session"].append(0, q, k, v, s["pos"], s["slots"], s["q_out"])
        else:
            _plain_append(s, q, k, v)
        return {"k": s["cache"][0], "v": s["cache"][1], "q": s["q_out"]}
    if not own:
        return {"out": _plain_attend(s)}
    if c["op"] == "paged":
        return {"out": s["session"].attend(0, s["batch"], s["q"], s["table"], s["own_len"], s["out"])}
    return {"out": s["session"].attend(0, s["batch"], s["q"], s["table"], s["own_len"], s["out"],
                                       prefix_table=s["ptable"], prefix_len=s["prefix_len"])}


# ------------------------------------------------------------------ plain forms
def _rotate(x, cos, sin):
    """Rotate-half pairs (i, i + d/2) of x [T, heads, d]."""
    a, b = x.chunk(2, dim=-1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _plain_append(s, q, k, v):
    c = s["case"]
    t, hq, hkv, d = c["tokens"], c["hq"], c["hkv"], c["d"]
    ang = s["pos"].float()[:, None] * torch.tensor(s["inv_freq"], device="cuda")[None]
    cos, sin = ang.cos()[:, None], ang.sin()[:, None]
    s["q_out"].copy_(_rotate(q.float().reshape(t, hq, d), cos, sin).reshape(t, hq * d))
    kr = _rotate(k.float().reshape(t, hkv, d), cos, sin).reshape(t, hkv * d)
    keep = s["slots"] >= 0
    to = s["slots"][keep]
    s["cache"][0, to] = kr[keep].to(torch.bfloat16)
    s["cache"][1, to] = v[keep].to(torch.bfloat16)


def _gather(cache, table, most, block, hkv, d):
    """The first `most` tokens' rows of each table row, in 32 bits: [n, hkv, most, d]."""
    at = torch.arange(most, device="cuda")
    slot = table.long()[:, at // block].clamp(min=0) * block + at % block
    return cache[slot].float().view(table.shape[0], most, hkv, d).transpose(1, 2)


def _plain_attend(s):
    c = s["case"]
    hq, hkv, d, block = c["hq"], c["hkv"], c["d"], c["block"]
    g = hq // hkv
    r, most = s["tok"].shape
    q = s["q"].float().view(-1, hkv, g, d)[s["tok"]]                       # [r, i, hkv, g, d]
    q = q.permute(0, 2, 1, 3, 4).reshape(r, hkv, most * g, d) * s["scale"]
    n_own = s["own_most"]
    score = q @ _gather(s["cache"][0], s["table"], n_own, block, hkv, d).transpose(2, 3)
    i = torch.arange(most, device="cuda")
    limit = (s["own_len"] - s["nq"])[:, None] + i[None] + 1                # [r, i]: keys j < limit are seen
    seen = torch.arange(n_own, device="cuda")[None, None] < limit[:, :, None]
    score = score.view(r, hkv, most, g, n_own).masked_fill_(~seen[:, None, :, None], -math.inf).view(r, hkv, most * g, n_own)
    top = score.amax(3, keepdim=True)
    if c["op"] == "prefix":
        n_pre = s["prefix_most"]
        groups, members = s["member"].shape
        qm = q[s["member"]].transpose(1, 2).reshape(groups, hkv, members * most * g, d)
        ps = qm @ _gather(s["cache"][0], s["ptable"], n_pre, block, hkv, d).transpose(2, 3)
        past = torch.arange(n_pre, device="cuda")[None] >= s["prefix_len"][:, None]
        ps.masked_fill_(past[:, None, None], -math.inf)
        back = lambda x: x.view(groups, hkv, members, most * g, -1)[s["group"], :, s["place"]]   # [r, hkv, i g, .]
        top = torch.maximum(top, back(ps.amax(3, keepdim=True)))
        ptop = top[s["member"]].transpose(1, 2).reshape(groups, hkv, members * most * g, 1)
        ps = ps.sub_(ptop).exp_()
        psum, pout = back(ps.sum(3, keepdim=True)), back(ps @ _gather(s["cache"][1], s["ptable"], n_pre, block, hkv, d))
        del ps
    p = score.sub_(top).exp_()
    total, o = p.sum(3, keepdim=True), p @ _gather(s["cache"][1], s["table"], n_own, block, hkv, d)
    if c["op"] == "prefix":
        total, o = total + psum, o + pout
    o = (o / total).view(r, hkv, most, g, d)[s["req"], :, s["idx"]]        # [T, hkv, g, d]
    return o.reshape(-1, hq * d).to(torch.bfloat16)


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c = case
    hq, hkv, d, block = c["hq"], c["hkv"], c["d"], c["block"]
    if c["op"] == "append":
        t = c["tokens"]
        x = s["qkv"].double().view(t, hq + 2 * hkv, d)
        freq = torch.tensor(s["inv_freq"], dtype=torch.float32, device="cuda").double()
        turn = torch.polar(torch.ones(t, d // 2, dtype=torch.float64, device="cuda"), s["pos"].double()[:, None] * freq)
        z = torch.complex(x[..., :d // 2].contiguous(), x[..., d // 2:].contiguous()) * turn[:, None]
        rot = torch.cat([z.real, z.imag], 2)
        k, v = s["cache"][0].double(), s["cache"][1].double()
        for token in torch.nonzero(s["slots"] >= 0).flatten().split(4096):
            k[s["slots"][token]] = rot[token, hq:hq + hkv].reshape(len(token), -1)
            v[s["slots"][token]] = x[token, hq + hkv:].reshape(len(token), -1)
        return {"k": k, "v": v, "q": rot[:, :hq].reshape(t, -1)}
    if work(case)["flops"] > 2e12:
        return None
    n = _lengths(c)
    out = torch.zeros(s["cu_q"][-1], hq, d, dtype=torch.float64, device="cuda")
    request = 0

    def rows(which, table, length):
        at = torch.arange(length, device="cuda")
        blk = table[at.div(block, rounding_mode="floor")].long()
        return s["cache"][which][blk * block + at.remainder(block)].view(length, hkv, d)

    for grp, m in enumerate(n["members"]):
        pre = n["prefix"][grp]
        pk = [rows(w, s["ptable"][grp], pre) for w in (0, 1)] if pre else None
        for _ in range(m):
            a, b, length = s["cu_q"][request], s["cu_q"][request + 1], n["own"][request]
            kv = [rows(w, s["table"][request], length) for w in (0, 1)]
            for h in range(hkv):
                key, val = ((kv[w][:, h] if pk is None else torch.cat([pk[w][:, h], kv[w][:, h]])).double() for w in (0, 1))
                q = s["q"][a:b].view(b - a, hkv, hq // hkv, d)[:, h].double()
                sc = torch.einsum("igd,jd->gij", q, key) / math.sqrt(d)
                j = torch.arange(pre + length, device="cuda")
                allowed = j[None] <= (pre + length - (b - a) + torch.arange(b - a, device="cuda"))[:, None]
                w = torch.softmax(torch.where(allowed[None], sc, -math.inf), dim=2)
                out[a:b].view(b - a, hkv, hq // hkv, d)[:, h] = torch.einsum("gij,jd->igd", w, val)
            request += 1
    return {"out": out.view(-1, hq * d)}
