"""The answering calls (cr_paged_append, cr_paged_attention, cr_prefix_attention) against
plain float64 computations of their definitions.

Tolerances, derived before any run.  Append: the rotation is fp32 (angles exact to ~2^-23
of the pair's size) and rounded once, so a value is within half a bf16 ulp of the exact one
plus 2^-20 of the pair's magnitude.  Attention: the output is a convex combination of V rows
rounded to bf16 (relative 2^-9 of the value), with P rounded to bf16 in the tile path: each
weight off by at most 2^-9 relative, so the output is off by at most 2^-9 sum_j p_j |v_j| <=
2^-9 max|v| beyond its own rounding; the fp32 scores (exact bf16 products, |s| <= ~40, d = 128
terms) are off by at most ~40 * 128 * 2^-24 = 3e-4 absolute in the worst case, a relative
error of each weight that again multiplies max|v|.  Bound: |err| <= 2^-8 max|v| + 2^-8 |exact|,
max|v| over the row's visible keys; lse: absolute 1e-3 (the score's error)."""
import math

import numpy as np
import pytest
import torch

from paper_2609_35139_gb300 import AnswerSession, cr

pytestmark = pytest.mark.gpu

SHAPES = {"8b": (32, 8, 128), "7b": (28, 4, 128), "3b": (16, 2, 128), "tiny": (4, 2, 64), "mqa": (40, 1, 64),
          "mha": (3, 3, 128)}


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2609_35139_gb300 import build
    build.build()
    cr.lib()
    cr.cr_clear_device_status()
    yield
    st, word = cr.cr_get_device_status()
    assert st == cr.CR_OK, f"device status {word}"


def _inv_freq(d):
    return (10000.0 ** (-2.0 * np.arange(d // 2) / d)).astype(np.float32)


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("shape", ["8b", "7b", "tiny", "mha"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,rope", [(1, True), (3, True), (157, True), (64, False), (1300, True)])
def test_append_matches_float64(shape, dtype, n, rope):
    hq, hkv, d = SHAPES[shape]
    g = torch.Generator(device="cuda").manual_seed(n + d)
    pad = 8                                        # columns that belong to nobody: a row stride of its own
    qkv = torch.randn(n, (hq + 2 * hkv) * d + pad, generator=g, device="cuda").to(dtype)
    q, k, v = (qkv[:, a:b] for a, b in ((0, hq * d), (hq * d, (hq + hkv) * d),
                                        ((hq + hkv) * d, (hq + 2 * hkv) * d)))
    slots_total = n + 37
    cache = torch.randn(4, slots_total, hkv * d, generator=g, device="cuda").to(torch.bfloat16)
    before = cache.clone()
    slots = torch.randperm(slots_total, generator=g, device="cuda")[:n].to(torch.int64)
    if n > 2:
        slots[n // 2] = -1
    pos = torch.randint(0, 131072, (n,), generator=g, device="cuda", dtype=torch.int32)
    freq = _inv_freq(d)
    sess = AnswerSession(cr.target_dims(2, hkv, d, hq * d, "bf16"), hq, cache, block_size=8, max_tokens=n,
                         inv_freq_target=freq if rope else None)
    q_out = sess.append(1, q, k, v, pos, slots)
    torch.cuda.synchronize()
    ang = pos.double()[:, None] * torch.from_numpy(freq).cuda().double()[None] * (1.0 if rope else 0.0)
    c, s = ang.cos()[:, None], ang.sin()[:, None]

    def rot(x, heads):
        x = x.double().reshape(n, heads, d)
        a, b = x[..., :d // 2], x[..., d // 2:]
        size = torch.sqrt(a * a + b * b).repeat(1, 1, 2)
        return torch.cat([a * c - b * s, b * c + a * s], -1).reshape(n, -1), size.reshape(n, -1)

    def close(got, exact, size):
        half_ulp = torch.exp2(torch.floor(torch.log2(exact.abs().clamp(min=1e-30))) - 8)
        assert bool(((got.double() - exact).abs() <= half_ulp + 2.0 ** -20 * size).all())

    close(q_out, *rot(q, hq))
    keep = slots >= 0
    ke, ksize = rot(k, hkv)
    close(cache[2][slots[keep]], ke[keep], ksize[keep])
    assert torch.equal(cache[3][slots[keep]], v[keep].to(torch.bfloat16))
    untouched = torch.ones(slots_total, dtype=torch.bool, device="cuda")
    untouched[slots[keep]] = False
    assert torch.equal(cache[:2], before[:2])                     # the other layer
    assert torch.equal(cache[2:, untouched], before[2:, untouched])


def test_append_in_place_and_without_queries():
    hq, hkv, d, n = 4, 2, 64, 50
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn(n, hq * d, generator=g, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn(n, hkv * d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    slots = torch.arange(n, dtype=torch.int64, device="cuda")
    t = cr.target_dims(1, hkv, d, hq * d, "bf16")
    caches = [torch.zeros(2, 64, hkv * d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    s0, s1 = (AnswerSession(t, hq, c, max_tokens=n, inv_freq_target=_inv_freq(d)) for c in caches)
    want = s0.append(0, q, k, v, pos, slots)
    mine = q.clone()
    assert s0.append(0, mine, k, v, pos, slots, mine) is mine and torch.equal(mine, want)
    assert s1.append(0, None, k, v, pos, slots) is None
    assert torch.equal(caches[0], caches[1])


def test_append_slot_out_of_range_is_reported_and_skipped():
    hkv, d = 2, 64
    cache = torch.zeros(2, 16, hkv * d, dtype=torch.bfloat16, device="cuda")
    sess = AnswerSession(cr.target_dims(1, hkv, d, 256, "bf16"), 4, cache, max_tokens=2)
    k = torch.ones(2, hkv * d, dtype=torch.bfloat16, device="cuda")
    sess.append(0, None, k, k, torch.zeros(2, dtype=torch.int32, device="cuda"),
                torch.tensor([16, 3], dtype=torch.int64, device="cuda"))
    st, word = cr.cr_get_device_status()
    cr.cr_clear_device_status()
    assert st == cr.CR_ERR_DEVICE_INDEX, word
    assert float(cache.float().sum()) == 2 * hkv * d and bool((cache[:, 3] == 1).all())


# ------------------------------------------------------------------ attention
class Case:
    """A batch with its cache: blocks in shuffled order, every slot that no token owns NaN."""

    def __init__(self, shape, nq, own, members=None, prefix=None, block=16, layers=1, layer=0, seed=0,
                 q_std=1.5, extra_blocks=3):
        self.hq, self.hkv, self.d = SHAPES[shape]
        self.nq, self.own, self.block, self.layer = list(nq), list(own), block, layer
        self.members, self.prefix = members, prefix
        g = torch.Generator(device="cuda").manual_seed(seed)
        width = self.hkv * self.d
        seqs = self.own + list(prefix or [])
        need = [-(-n // block) for n in seqs]
        blocks = sum(need) + extra_blocks
        order = torch.randperm(blocks, generator=g, device="cuda").cpu().numpy()
        self.cache = torch.full((2 * layers, blocks * block, width), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.rows, tables, at = [], [], 0
        for n, b in zip(seqs, need):
            mine = order[at:at + b]
            at += b
            tables.append(mine)
            slots = (mine[:, None] * block + np.arange(block)[None]).reshape(-1)[:n]
            slots = torch.from_numpy(slots.astype(np.int64)).cuda()
            k = torch.randn(n, width, generator=g, device="cuda")
            k[:, ::37] *= 8.0 / max(1.0, 8.0 * q_std)
            v = torch.randn(n, width, generator=g, device="cuda")
            self.cache[2 * layer, slots] = k.to(torch.bfloat16)
            self.cache[2 * layer + 1, slots] = v.to(torch.bfloat16)
            self.rows.append(slots)

        def table(parts):
            t = np.full((len(parts), max(1, max(len(x) for x in parts))), -1, np.int32)
            for i, x in enumerate(parts):
                t[i, :len(x)] = x
            return torch.from_numpy(t).cuda()

        self.table = table(tables[:len(self.own)])
        self.own_len = torch.tensor(self.own, dtype=torch.int32, device="cuda")
        self.cu_q = np.concatenate([[0], np.cumsum(self.nq)]).astype(np.int32)
        self.cu_group = None
        if members:
            self.ptable = table(tables[len(self.own):])
            self.prefix_len = torch.tensor(list(prefix), dtype=torch.int32, device="cuda")
            self.cu_group = np.concatenate([[0], np.cumsum(members)]).astype(np.int32)
        n = int(self.cu_q[-1])
        self.q = torch.randn(n, self.hq * self.d, generator=g, device="cuda").mul_(q_std).to(torch.bfloat16)
        self.scale = 1.0 / math.sqrt(self.d)

    def session(self):
        return AnswerSession(cr.target_dims(self.cache.shape[0] // 2, self.hkv, self.d, self.hq * self.d, "bf16"),
                             self.hq, self.cache, block_size=self.block, max_tokens=int(self.cu_q[-1]),
                             scale=self.scale)

    def run(self, sess=None, batch=None, lse=True):
        sess = sess or self.session()
        batch = batch or sess.batch(self.cu_q, self.cu_group)
        kw = {} if self.cu_group is None else {"prefix_table": self.ptable, "prefix_len": self.prefix_len}
        n = batch.n_tokens
        out = torch.full((n, self.hq * self.d), float("nan"), dtype=torch.bfloat16, device="cuda")
        ls = torch.full((n, self.hq), float("nan"), device="cuda") if lse else None
        sess.attend(self.layer, batch, self.q, self.table, self.own_len, out, lse=ls, **kw)
        torch.cuda.synchronize()
        return out, ls

    def exact(self):
        """(out, lse, max |v| of each row) in float64."""
        hq, hkv, d = self.hq, self.hkv, self.d
        n = int(self.cu_q[-1])
        out = torch.zeros(n, hq, d, dtype=torch.float64, device="cuda")
        lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device="cuda")
        vmax = torch.zeros(n, hq, 1, dtype=torch.float64, device="cuda")
        K, V = (self.cache[2 * self.layer + i] for i in (0, 1))
        group = [0] * len(self.nq)
        if self.cu_group is not None:
            for gi in range(len(self.cu_group) - 1):
                for r in range(self.cu_group[gi], self.cu_group[gi + 1]):
                    group[r] = gi
        for r, nr in enumerate(self.nq):
            for i in range(nr):
                seen = max(0, self.own[r] - nr + i + 1)
                slots = self.rows[r][:seen]
                if self.cu_group is not None:
                    slots = torch.cat([self.rows[len(self.own) + group[r]], slots])
                if len(slots) == 0:
                    continue
                t = int(self.cu_q[r]) + i
                k = K[slots].double().view(-1, hkv, d).repeat_interleave(hq // hkv, 1)
                v = V[slots].double().view(-1, hkv, d).repeat_interleave(hq // hkv, 1)
                s = torch.einsum("hd,jhd->hj", self.q[t].double().view(hq, d), k) * self.scale
                lse[t] = torch.logsumexp(s, 1)
                out[t] = torch.einsum("hj,jhd->hd", torch.exp(s - lse[t][:, None]), v)
                vmax[t] = v.abs().amax(dim=(0, 2))[:, None]
        return out.view(n, -1), lse, vmax.expand(n, hq, d).reshape(n, -1)

    def check(self, **kw):
        out, lse = self.run(**kw)
        e, el, vmax = self.exact()
        o = out.double()
        assert bool(torch.isfinite(o).all())
        bad = (o - e).abs() - (2.0 ** -8 * vmax + 2.0 ** -8 * e.abs())
        assert float(bad.max()) <= 0.0, f"worst excess {float(bad.max()):.3e}"
        if lse is not None:
            empty = torch.isinf(el)
            assert torch.equal(torch.isinf(lse), empty) and bool((lse[empty] < 0).all())
            assert float((lse.double() - el)[~empty].abs().max() if bool((~empty).any()) else 0.0) <= 1e-3
        return out


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("own", [[1], [15, 16, 17], [0, 5, 0, 130], [127, 128, 129, 1], [1000, 3, 513]])
def test_decode(shape, own):
    """One new token a request; a request whose cache is empty sees nothing and gets zeros."""
    Case(shape, [1] * len(own), own, seed=len(own) + sum(own)).check()


@pytest.mark.parametrize("shape", ["8b", "7b", "tiny", "mqa"])
@pytest.mark.parametrize("nq,past", [([2], [0]), ([5, 1, 0, 33], [7, 0, 12, 100]), ([130, 64], [0, 300]),
                                     ([257], [1000]), ([3, 3], [-2, 50])])
def test_new_tokens_are_causal(shape, nq, past):
    """Several new tokens a request (none in one; past -2: the cache holds fewer tokens than
    there are rows, the first of which see nothing)."""
    own = [max(0, a + b) for a, b in zip(nq, past)]
    Case(shape, nq, own, seed=sum(nq)).check()


@pytest.mark.parametrize("block", [8, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("shape", ["3b", "tiny"])
def test_block_sizes(shape, block):
    Case(shape, [1, 4, 40], [700, 4, 333], block=block, layers=2, layer=1, seed=block).check()


@pytest.mark.parametrize("shape", ["8b", "7b", "tiny", "mha"])
@pytest.mark.parametrize("members,prefix,nq,own", [
    ([1], [300], [1], [1]),
    ([3], [17], [1, 1, 1], [1, 40, 0]),
    ([40], [513], [1] * 40, [1 + (7 * i) % 90 for i in range(40)]),
    ([2, 5, 1], [1000, 0, 129], [1, 3, 1, 2, 1, 1, 4, 9], [5, 3, 200, 2, 1, 0, 4, 30]),
    ([4, 0, 2], [64, 5, 128], [1] * 6, [0] * 6),
    ([9], [257], [33] * 9, [33 + i for i in range(9)]),
])
def test_shared_prefix(shape, members, prefix, nq, own):
    Case(shape, nq, own, members, prefix, seed=sum(prefix)).check()


@pytest.mark.parametrize("shape,requests,prefix,own", [("7b", 100, 20000, 3), ("tiny", 200, 9001, 30)])
def test_long_prefix_of_several_row_tiles(shape, requests, prefix, own):
    """Row tiles that are cut in different places and start in the middle of their pieces."""
    Case(shape, [1] * requests, [1 + i % own for i in range(requests)], [requests], [prefix], seed=prefix).check()


@pytest.mark.parametrize("shape,nq", [("7b", 4), ("8b", 32), ("tiny", 50), ("mqa", 1)])
@pytest.mark.parametrize("past", [100, 129, 300, 5000])
def test_one_row_tile(shape, nq, past):
    """Units of 17 to 128 rows, whose chunks (one, odd and even numbers of them) go to two groups."""
    Case(shape, [nq, 1, nq], [nq + past, 700, nq], seed=past + nq).check()


def test_two_batches_on_two_streams():
    """Batches with plans (and workspaces) of their own run side by side."""
    cases = [Case("8b", [1] * 9, [700 + 31 * i for i in range(9)], seed=1),
             Case("8b", [1] * 30, [5 + i for i in range(30)], [30], [4000], seed=2)]
    want = [c.run(lse=False)[0] for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    outs = []
    for c, st in zip(cases, streams):
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            sess = c.session()
            batch = sess.batch(c.cu_q, c.cu_group)
            kw = {} if c.cu_group is None else {"prefix_table": c.ptable, "prefix_len": c.prefix_len}
            outs.append([sess.attend(0, batch, c.q, c.table, c.own_len, **kw) for _ in range(20)])
    torch.cuda.synchronize()
    for got, w in zip(outs, want):
        assert all(torch.equal(o, w) for o in got)


def test_shared_prefix_equals_its_copy_in_every_request():
    """The same keys as a shared prefix and as the head of each request's own sequence."""
    c = Case("8b", [1] * 6, [40] * 6, [6], [640], seed=9)
    a, _ = c.run()
    d = Case("8b", [1] * 6, [40] * 6, [6], [640], seed=9)
    blocks = [torch.cat([d.ptable[0], d.table[r]]) for r in range(6)]
    d.table, d.cu_group = torch.stack(blocks).contiguous(), None
    d.own_len = torch.full((6,), 680, dtype=torch.int32, device="cuda")
    b, _ = d.run()
    assert float((a.double() - b.double()).abs().max()) <= 2.0 ** -7 * float(a.abs().max())


@pytest.mark.parametrize("n_req", [1, 255, 256])
def test_many_requests(n_req):
    Case("tiny", [1 + (i % 3 == 0) for i in range(n_req)], [2 + (i * 13) % 70 for i in range(n_req)], seed=n_req).check()


SHAPES["one"] = (5, 1, 128)      # one KV head: a sequence's keys lie in one line


@pytest.mark.parametrize("shape,nq", [("8b", [1, 4, 2]), ("one", [1, 3, 2]), ("7b", [2, 1, 1]), ("mqa", [1, 1, 1]), ("tiny", [8, 1, 5])])
def test_one_plan_over_changing_lengths(shape, nq):
    """Calls of one plan depend on their own lengths alone, whatever ran before; equal calls give equal bits."""
    most = [5000, 2000, 4000]
    c = Case(shape, nq, most, seed=21)
    sess = c.session()
    batch = sess.batch(c.cu_q)
    seen = {}
    for own in ([5000, 0, 17], [0, 0, 0], most, [40, 1999, 3], [0, 8, 0], most, [5000, 0, 17]):
        c.own = list(own)
        c.own_len = torch.tensor(own, dtype=torch.int32, device="cuda")
        out = c.check(sess=sess, batch=batch)
        assert torch.equal(out, seen.setdefault(tuple(own), out))


def test_strided_queries_and_output_and_repeatability():
    c = Case("8b", [1, 7], [90, 300], seed=4)
    want, _ = c.run()
    wide = torch.zeros(8, c.hq * c.d + 64, dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + c.hq * c.d] = c.q
    big = torch.full((8, c.hq * c.d + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    sess = c.session()
    sess.attend(0, sess.batch(c.cu_q), wide[:, 8:8 + c.hq * c.d], c.table, c.own_len, big[:, :c.hq * c.d])
    torch.cuda.synchronize()
    assert torch.equal(big[:, :c.hq * c.d], want) and bool((big[:, c.hq * c.d:] == 7.0).all())
    again, _ = c.run()
    assert torch.equal(again, want)                 # sums in a fixed order


def test_large_scores_do_not_overflow():
    """Scores of several hundred: the running maximum keeps every exponential in range."""
    c = Case("3b", [1, 20], [400, 900], seed=6, q_std=1.0)
    c.q.mul_(60.0)
    out, lse = c.run()
    e, el, vmax = c.exact()
    # a score's fp32 error grows with it: |s| up to ~1500 of 128 terms, 1500 * 128 * 2^-24 = 1.2e-2
    assert float(((out.double() - e).abs() - (1.5e-2 * 2 * vmax + 2.0 ** -8 * e.abs())).max()) <= 0
    assert float((lse.double() - el).abs().max()) <= 1.5e-2


def test_slots_past_two_gib_offsets():
    """A cache whose rows lie past 2^31 elements and 2^32 bytes from its start."""
    hq, hkv, d = SHAPES["8b"]
    block, blocks = 16, (1 << 31) // (1024 * 16) + 400          # 2^31 elements and some
    cache = torch.zeros(2, blocks * block, hkv * d, dtype=torch.bfloat16, device="cuda")
    sess = AnswerSession(cr.target_dims(1, hkv, d, hq * d, "bf16"), hq, cache, block_size=block, max_tokens=40,
                         inv_freq_target=_inv_freq(d))
    g = torch.Generator(device="cuda").manual_seed(1)
    n = 40
    qkv = torch.randn(n, (hq + 2 * hkv) * d, generator=g, device="cuda").to(torch.bfloat16)
    q, k, v = qkv.split([hq * d, hkv * d, hkv * d], 1)
    table = torch.tensor([[blocks - 1, 3, blocks - 7]], dtype=torch.int32, device="cuda")
    j = torch.arange(n, device="cuda")
    slots = table[0].long()[j // block] * block + j % block
    pos = j.to(torch.int32)
    qr = sess.append(0, q, k, v, pos, slots)
    out = sess.attend(0, sess.batch([0, n]), qr, table, torch.tensor([n], dtype=torch.int32, device="cuda"))
    assert torch.equal(cache[1][slots], v)
    kk = cache[0][slots].double().view(n, hkv, d).repeat_interleave(hq // hkv, 1)
    vv = v.double().reshape(n, hkv, d).repeat_interleave(hq // hkv, 1)
    s = torch.einsum("ihd,jhd->hij", qr.double().view(n, hq, d), kk) / math.sqrt(d)
    s = s.masked_fill(torch.ones(n, n, device="cuda").triu(1).bool(), -math.inf)
    e = torch.einsum("hij,jhd->ihd", torch.softmax(s, 2), vv).reshape(n, -1)
    assert float(((out.double() - e).abs() - 2.0 ** -8 * (float(v.abs().max()) + e.abs())).max()) <= 0


def test_bad_tables_and_lengths_are_reported():
    c = Case("tiny", [1, 1], [40, 20], seed=2)
    sess, cases = c.session(), []
    c.table[0, 1] = c.cache.shape[1] // c.block + 4              # a block outside the cache: zeros
    cases.append(c.own_len.clone())
    cases.append(torch.tensor([-3, 20], dtype=torch.int32, device="cuda"))
    cases.append(torch.tensor([40, 16 * c.table.shape[1] + 1], dtype=torch.int32, device="cuda"))
    for i, lens in enumerate(cases):
        if i == 1:
            c.table[0, 1] = 0
        if i == 2:
            c.table[1] = torch.arange(c.table.shape[1], dtype=torch.int32, device="cuda")
        sess.attend(0, sess.batch(c.cu_q), c.q, c.table, lens)
        st, word = cr.cr_get_device_status()
        cr.cr_clear_device_status()
        assert st == cr.CR_ERR_DEVICE_INDEX, (i, word)


def test_captured_decode_follows_growing_sequences():
    """One captured append and attention, replayed as kv_len, pos and the slots move on."""
    hq, hkv, d, block, steps = 16, 2, 128, 16, 20
    g = torch.Generator(device="cuda").manual_seed(8)
    start = [30, 5, 64]
    cache = torch.randn(2, 40 * block, hkv * d, generator=g, device="cuda").to(torch.bfloat16)
    table = torch.randperm(40, generator=g, device="cuda")[:21].to(torch.int32).view(3, 7).contiguous()
    twin = cache.clone()
    t = cr.target_dims(1, hkv, d, hq * d, "bf16")
    s0, s1 = (AnswerSession(t, hq, c, block_size=block, max_tokens=3, inv_freq_target=_inv_freq(d))
              for c in (cache, twin))
    qkv = torch.empty(3, (hq + 2 * hkv) * d, dtype=torch.bfloat16, device="cuda")
    q, k, v = qkv.split([hq * d, hkv * d, hkv * d], 1)
    pos = torch.tensor(start, dtype=torch.int32, device="cuda")
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    kv_len = torch.zeros(3, dtype=torch.int32, device="cuda")
    qr, out = (torch.empty(3, hq * d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    b0, b1 = s0.batch([0, 1, 2, 3]), s1.batch([0, 1, 2, 3])

    def step(sess, batch, qr, out):
        sess.append(0, q, k, v, pos, slots, qr)
        sess.attend(0, batch, qr, table, kv_len, out)

    side = torch.cuda.Stream()
    graph = None
    for i in range(steps):
        qkv.copy_(torch.randn(qkv.shape, generator=g, device="cuda").to(torch.bfloat16))
        pos.copy_(torch.tensor([x + i for x in start], dtype=torch.int32))
        j = pos.long()
        slots.copy_(table.long().gather(1, (j // block)[:, None])[:, 0] * block + j % block)
        kv_len.copy_(pos + 1)
        want_q, want = torch.empty_like(qr), torch.empty_like(out)
        step(s1, b1, want_q, want)
        torch.cuda.synchronize()
        if graph is None:
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                step(s0, b0, qr, out)
            torch.cuda.current_stream().wait_stream(side)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step(s0, b0, qr, out)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(cache, twin), i
