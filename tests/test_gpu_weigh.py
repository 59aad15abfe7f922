"""cr_attention_weights (AnswerSession.weigh) against a plain float64 computation of its definition.

Tolerance, derived before any run: a score is a sum of d <= 128 exact bf16 products in fp32, off by at
most 128 * 2^-23 * sum |q k| scale, and that sum stays below 25 here (|q| about 1.5, |k| about 1): 3.9e-4,
which is the relative error of its exponential; the scaling, the subtraction of lse and ex2 add at most
2^-22 * (25 + 25) = 1.2e-5.  Terms are positive, so their fp32 sum of n terms is off by at most n * 2^-24 of
itself in any order (n <= 6000 here: 3.6e-4) and adding to what was gathered by 2^-24 of that.  Bound:
1e-3 of the new part + 2^-23 of the whole."""
import math

import numpy as np
import pytest
import torch

from paper_2609_35139_gb300 import cr
from test_gpu_answer import SHAPES, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2609_35139_gb300 import build
    build.build()
    cr.cr_clear_device_status()
    yield
    st, word = cr.cr_get_device_status()
    assert st == cr.CR_OK, f"device status {word}"


def prefix_of(c):
    return {} if c.cu_group is None else {"prefix_table": c.ptable, "prefix_len": c.prefix_len}


def start(c, seed=0):
    """What the tokens have gathered: NaN where no old token lies (new ones' slots included)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.full((c.hkv, c.cache.shape[1]), float("nan"), device="cuda")
    fill = lambda slots: w.__setitem__((slice(None), slots), torch.rand(c.hkv, len(slots), generator=g, device="cuda"))
    for r, n in enumerate(c.nq):
        fill(c.rows[r][:max(0, c.own[r] - n)])
    for i in range(len(c.prefix or [])):
        fill(c.rows[len(c.own) + i])
    return w


def exact(c, lse, weights):
    """(old part, new part) in float64, [hkv, slots]."""
    hq, hkv, d = c.hq, c.hkv, c.d
    g = hq // hkv
    old = weights.double()
    new = torch.zeros_like(old)
    K = c.cache[2 * c.layer]

    def add(slots, a, b, causal):
        n = len(slots)
        if n == 0 or a == b:
            return
        q = c.q[a:b].double().view(b - a, hkv, g, d)
        s = torch.einsum("ihgd,jhd->hgij", q, K[slots].double().view(n, hkv, d)) * c.scale
        l = lse[a:b].double().view(b - a, hkv, g).permute(1, 2, 0)[..., None]
        p = torch.exp(s - l)
        p = torch.where(l == -math.inf, 0.0, p)
        if causal:
            i = torch.arange(b - a, device="cuda")
            p = torch.where(torch.arange(n, device="cuda")[None] < (n - (b - a) + i + 1)[:, None], p, 0.0)
            fresh = slots[max(0, n - (b - a)):]
            old[:, fresh] = 0.0
        new[:, slots] += p.sum((1, 2))

    cu = [int(x) for x in c.cu_q]
    for r in range(len(c.nq)):
        add(c.rows[r], cu[r], cu[r + 1], True)
    if c.cu_group is not None:
        for i in range(len(c.cu_group) - 1):
            add(c.rows[len(c.own) + i], cu[c.cu_group[i]], cu[c.cu_group[i + 1]], False)
    return old, new


def check(c, lse=None, sess=None, batch=None):
    sess = sess or c.session()
    batch = batch or sess.batch(c.cu_q, c.cu_group)
    if lse is None:
        _, lse = c.run(sess, batch)
    w = start(c)
    old, new = exact(c, lse, w)
    got = sess.weigh(c.layer, batch, c.q, lse, c.table, c.own_len, w.clone(), **prefix_of(c))
    torch.cuda.synchronize()
    want = old + new
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = ~torch.isnan(want)
    bad = (got.double() - want).abs() - (1e-3 * new + 2.0 ** -23 * want.abs())
    assert not bool(fine.any()) or float(bad[fine].max()) <= 0.0, f"worst excess {float(bad[fine].max()):.3e}"
    return got, lse, w, sess, batch


@pytest.mark.parametrize("shape", list(SHAPES))
@pytest.mark.parametrize("own", [[1], [15, 16, 17], [0, 5, 0, 130], [127, 128, 129, 1], [255, 256, 257], [1000, 3, 513]])
def test_one_new_token(shape, own):
    """A decode step; a request without tokens has nothing to gather."""
    check(Case(shape, [1] * len(own), own, seed=len(own) + sum(own)))


@pytest.mark.parametrize("shape", ["8b", "7b", "tiny", "mqa"])
@pytest.mark.parametrize("nq,own", [([3], [3]), ([2, 5, 4], [700, 5, 260]), ([17, 1, 40], [17, 300, 900]),
                                    ([130], [130]), ([128], [385]), ([300, 20], [811, 20]), ([0, 33, 0], [12, 70, 0])])
def test_many_new_tokens(shape, nq, own):
    check(Case(shape, nq, own, seed=sum(nq)))


@pytest.mark.parametrize("block", [8, 32, 256, 1024])
@pytest.mark.parametrize("nq,own", [([1, 1], [300, 2049]), ([70], [1500])])
def test_blocks(block, nq, own):
    check(Case("8b", nq, own, block=block, layers=2, layer=1, seed=block))


@pytest.mark.parametrize("shape", ["8b", "7b", "tiny"])
@pytest.mark.parametrize("members,prefix,nq,own", [([4], [512], [1] * 4, [20, 1, 33, 90]),
                                                   ([3, 1, 2], [1000, 0, 17], [1, 2, 1, 60, 1, 3], [5, 2, 40, 60, 1, 300]),
                                                   ([40], [300], [2] * 40, list(range(2, 42))),
                                                   ([2, 0, 1], [129, 64, 255], [1, 1, 1], [0, 1, 1])])
def test_prefixes(shape, members, prefix, nq, own):
    """A prefix gathers over all rows of its group (of an empty group: nothing)."""
    check(Case(shape, nq, own, members, prefix, seed=sum(own)))


def test_more_rows_than_tokens_cached():
    """kv_len below the number of new tokens: the first rows see nothing, every token is new."""
    c = Case("8b", [9, 1], [4, 0], seed=5)
    check(c)


@pytest.mark.parametrize("nq,own", [([1], [200]), ([50], [300])])
def test_rows_that_see_nothing_and_nan_rows(nq, own):
    c = Case("8b", nq, own, seed=7)
    _, lse = c.run()
    lse[0, 3] = -math.inf                  # (of KV head 0)
    got, *_ = check(c, lse)
    lse[0, 9] = float("nan")               # (of KV head 2: every token that row 0 sees)
    got, *_ = check(c, lse)
    seen = c.rows[0][:own[0] - nq[0] + 1]
    assert bool(torch.isnan(got[2, seen]).all()) and not bool(torch.isnan(got[0, seen]).any())
    # a query that holds NaN but whose row saw nothing gives nothing
    lse[0, 8:12] = -math.inf
    c.q[0, 8 * c.d:12 * c.d] = float("nan")
    got, *_ = check_masked(c, lse)
    assert not bool(torch.isnan(got[2, seen]).any())


def check_masked(c, lse):
    """check for queries that are NaN where lse is -inf."""
    q = c.q
    c.q = torch.nan_to_num(q)
    w = start(c)
    old, new = exact(c, lse, w)
    c.q = q
    sess = c.session()
    got = sess.weigh(c.layer, sess.batch(c.cu_q, c.cu_group), c.q, lse, c.table, c.own_len, w.clone())
    want = old + new
    fine = ~torch.isnan(want)
    assert torch.equal(torch.isnan(got), ~fine)
    assert float(((got.double() - want).abs() - 1e-3 * new - 2.0 ** -23 * want)[fine].max()) <= 0.0
    return got, want


def test_nan_key_stays_with_its_token():
    c = Case("8b", [3], [400], seed=11)
    sess = c.session()
    batch = sess.batch(c.cu_q)
    _, lse = c.run(sess, batch)
    want = sess.weigh(0, batch, c.q, lse, c.table, c.own_len, start(c))
    j = c.rows[0][123]
    c.cache[0, j, 2 * c.d + 5] = float("nan")             # KV head 2
    got = sess.weigh(0, batch, c.q, lse, c.table, c.own_len, start(c))
    assert bool(torch.isnan(got[2, j]))
    got[2, j] = want[2, j]
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


def test_equal_calls_give_equal_bits():
    c = Case("8b", [600, 1, 3], [2500, 700, 3], [3], [900], seed=13)
    got, lse, w, sess, batch = check(c)
    for _ in range(3):
        again = sess.weigh(0, batch, c.q, lse, c.table, c.own_len, w.clone(), **prefix_of(c))
        assert torch.equal(torch.nan_to_num(again, nan=-1.0), torch.nan_to_num(got, nan=-1.0))


def test_q_may_be_a_column_of_a_wider_tensor():
    c = Case("7b", [3, 40], [60, 300], seed=17)
    got, lse, w, sess, batch = check(c)
    wide = torch.randn(43, c.hq * c.d + 64, device="cuda").to(torch.bfloat16)
    wide[:, 32:32 + c.hq * c.d] = c.q
    again = sess.weigh(0, batch, wide[:, 32:32 + c.hq * c.d], lse, c.table, c.own_len, w.clone())
    assert torch.equal(torch.nan_to_num(again, nan=-1.0), torch.nan_to_num(got, nan=-1.0))


def test_captured_and_replayed_as_sequences_grow():
    c = Case("8b", [1, 1], [40, 300], seed=19)
    sess = c.session()
    batch = sess.batch(c.cu_q)
    lens = torch.tensor([30, 280], dtype=torch.int32, device="cuda")
    lse = torch.randn(2, c.hq, device="cuda") + 5
    w = torch.zeros(c.hkv, c.cache.shape[1], device="cuda")
    sess.weigh(0, batch, c.q, lse, c.table, lens, w.clone())
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        sess.weigh(0, batch, c.q, lse, c.table, lens, w)
    by_hand = torch.zeros_like(w)
    for a, b in ((30, 280), (31, 281), (40, 300)):
        lens.copy_(torch.tensor([a, b], dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        sess.weigh(0, batch, c.q, lse, c.table, lens, by_hand)
        assert torch.equal(w, by_hand)


def test_bad_blocks_and_lengths_are_reported():
    c = Case("8b", [1, 20], [100, 90], seed=23)
    sess = c.session()
    batch = sess.batch(c.cu_q)
    _, lse = c.run(sess, batch)
    good = sess.weigh(0, batch, c.q, lse, c.table, c.own_len, start(c))
    cr.cr_clear_device_status()
    table = c.table.clone()
    table[0, 1], table[1, 2] = 10 ** 6, -7
    got = sess.weigh(0, batch, c.q, lse, table, c.own_len, start(c))
    st, word = cr.cr_get_device_status()
    cr.cr_clear_device_status()
    assert st == cr.CR_ERR_DEVICE_INDEX, word
    old = start(c)
    for r, b in ((0, 1), (1, 2)):               # the bad blocks' tokens have gathered nothing
        at = c.rows[r][16 * b:16 * (b + 1)]
        assert torch.equal(got[:, at], old[:, at])
        got[:, at] = good[:, at]
    assert torch.equal(torch.nan_to_num(got, nan=-1.0), torch.nan_to_num(good, nan=-1.0))
    for bad in ([-5, 90], [100, 10 ** 6]):
        sess.weigh(0, batch, c.q, lse, c.table, torch.tensor(bad, dtype=torch.int32, device="cuda"), start(c))
        st, word = cr.cr_get_device_status()
        cr.cr_clear_device_status()
        assert st == cr.CR_ERR_DEVICE_INDEX, word


def test_on_another_stream_and_with_two_batches_at_once():
    c = Case("8b", [1, 33], [500, 800], seed=29)
    got, lse, w, sess, batch = check(c)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    torch.cuda.synchronize()
    for s in streams:
        b = sess.batch(c.cu_q, stream=s)
        mine = w.clone()
        s.wait_stream(torch.cuda.current_stream())
        outs.append((sess.weigh(0, b, c.q, lse, c.table, c.own_len, mine, stream=s), b))
    torch.cuda.synchronize()
    for x, _ in outs:
        assert torch.equal(torch.nan_to_num(x, nan=-1.0), torch.nan_to_num(got, nan=-1.0))


@pytest.mark.parametrize("heads", [(100, 1, 64), (160, 1, 64), (300, 1, 64), (129, 1, 128), (65, 1, 128)])
@pytest.mark.parametrize("nq,own", [([1], [300]), ([3, 40], [3, 700])])
def test_groups_of_any_size(monkeypatch, heads, nq, own):
    """Groups that fill a tile of rows badly, and ones that no tile holds."""
    monkeypatch.setitem(SHAPES, "wide", heads)
    check(Case("wide", nq, own, seed=heads[0]))


def test_single_tokens_beside_a_prompt():
    """Segments of few rows in a call that has one of many."""
    check(Case("8b", [1] * 20 + [150] + [2] * 5, [1, 700, 30] * 6 + [5, 5, 600] + [300, 2, 9, 2000, 3], seed=31))


@pytest.mark.parametrize("shape", ["8b", "tiny"])
def test_a_long_prompt(shape):
    """Units cut between CTAs, and the join of their parts."""
    check(Case(shape, [1300], [4000], seed=37))
