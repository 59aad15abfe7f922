"""cr_attention_weights against float64, to a bound that no row can be lost below.

Tolerance, derived before any run, of a term p = exp(s - l), s = scale q . k, l the row's lse (given, so exact):
- s: the d / 16 MMAs of a score add exact products to a sum of 24 bits.  An MMA loses at most two last bits of its
  largest partial sum, which is no larger than A = scale sum |q k|: d / 16 * 2^-22 A in all.  Where all partial sums
  fit 24 bits (whole numbers and halves, below) nothing.
- the scale's correction for what MMAs cut off: 1.5e-7 of s, below 2^-22 |s|;
- the rounded scale, alike for s and l: 2^-24 |s - l|; the FMAs that form s - l: twice that; l in log2 units: 2^-23 |l|;
- 2^x: 2^-22.
A token's sum of positive terms: 32 + 3 additions a tile of rows, one carry, one exchange, and a part for each CTA
that a unit goes through (28 allowed): 64 * 2^-24 of itself.  Adding it to what the token had: 2^-24 of the whole.

With whole and half numbers that is about 1e-5 of a sum, where a row of 1300 is 8e-4 of it and one head of a row
2e-4: each test asserts, from the float64 terms alone, that every row and head has a token that would show its loss."""
import math

import numpy as np
import pytest
import torch

from test_gpu_answer import Case
from test_gpu_weigh import lib, prefix_of, start  # noqa: F401  (lib: fixture)

pytestmark = pytest.mark.gpu


def fill(c, kind, seed):
    """Q, and K of every token, anew."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, d = c.q.shape[0], c.d
    whole = lambda lo, hi, *shape: torch.randint(lo, hi + 1, shape, generator=g, device="cuda").float()
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    if kind == "whole":
        q = whole(-3, 3, n, c.hq, d) / 2
    elif kind == "cancelling":             # s is what two large halves leave
        half = normal(n, c.hq, d // 2) * 6
        q = torch.cat([half, 0.3 * normal(n, c.hq, d // 2) - half], 2)
    else:                                  # negative: every score far below 0
        q = -(normal(n, c.hq, d).abs() * 0.5 + 1.0)
    c.q.copy_(q.reshape(n, c.hq * d))
    for slots in c.rows:
        m = len(slots)
        if kind == "whole":
            k = whole(-1, 1, m, c.hkv, d)
        elif kind == "cancelling":
            half = normal(m, c.hkv, d // 2)
            k = torch.cat([half, half], 2)
        else:
            k = normal(m, c.hkv, d).abs() + 0.5
        c.cache[2 * c.layer, slots] = k.reshape(m, c.hkv * d).to(torch.bfloat16)


def exact(c, lse, weights, whole):
    """(old part, new part, tolerance) in float64, [hkv, slots]."""
    hq, hkv, d = c.hq, c.hkv, c.d
    g, scale = hq // hkv, float(np.float32(c.scale))
    old = weights.double()
    new, tol = torch.zeros_like(old), torch.zeros_like(old)
    seen = []                               # (rows' terms, slots, head) for the assertion at the end

    def add(slots, a, b, causal):
        n = len(slots)
        if n == 0 or a == b:
            return
        if causal:
            old[:, slots[max(0, n - (b - a)):]] = 0.0
        for h in range(hkv):
            k = c.cache[2 * c.layer][slots].view(n, hkv, d)[:, h].double()
            q = c.q[a:b].view(b - a, hq, d)[:, h * g:(h + 1) * g].double()
            l = lse[a:b, h * g:(h + 1) * g].double()[..., None]
            s = torch.einsum("igd,jd->igj", q, k) * scale
            p = torch.exp(s - l)
            if causal:
                i = torch.arange(b - a, device="cuda")
                p.mul_((torch.arange(n, device="cuda")[None] < (n - (b - a) + i + 1)[:, None])[:, None])
            rel = s.abs() * 2.0 ** -22 + (s - l).abs() * (3 * 2.0 ** -24) + l.abs() * 2.0 ** -23 + 2.0 ** -22
            if not whole:
                rel += torch.einsum("igd,jd->igj", q.abs(), k.abs()) * (scale * d / 16 * 2.0 ** -22)
            new[h, slots] += p.sum((0, 1))
            tol[h, slots] += (p * rel).sum((0, 1))
            if whole:
                seen.append((p, slots, h))

    cu = [int(x) for x in c.cu_q]
    for r in range(len(c.nq)):
        add(c.rows[r], cu[r], cu[r + 1], True)
    if c.cu_group is not None:
        for i in range(len(c.cu_group) - 1):
            add(c.rows[len(c.own) + i], cu[c.cu_group[i]], cu[c.cu_group[i + 1]], False)
    tol += 64 * 2.0 ** -24 * new + 2.0 ** -24 * (old + new).abs()
    for p, slots, h in seen:
        assert bool((p > 2 * torch.nan_to_num(tol[h, slots], nan=math.inf)).any(2).all()), "a lost row could pass"
    return old, new, tol


def check(c, kind, seed=0):
    fill(c, kind, seed)
    sess = c.session()
    batch = sess.batch(c.cu_q, c.cu_group)
    _, lse = c.run(sess, batch)
    w = start(c)
    old, new, tol = exact(c, lse, w, kind == "whole")
    got = sess.weigh(c.layer, batch, c.q, lse, c.table, c.own_len, w.clone(), **prefix_of(c))
    want = old + new
    fine = ~torch.isnan(want)
    assert torch.equal(torch.isnan(got), ~fine)
    worst = ((got.double() - want).abs() / tol)[fine & (tol > 0)].max()
    assert float(worst) <= 1.0, f"{float(worst):.2f} of the tolerance"
    assert torch.equal(got[fine & (tol == 0)], w[fine & (tol == 0)])


KINDS = ["whole", "cancelling", "negative"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape,nq,own", [("8b", [1300], [4000]), ("tiny", [1300], [4000]), ("7b", [300, 77, 1], [2000, 900, 500]),
                                          ("mqa", [90], [5000]), ("3b", [128, 129, 257], [128, 1029, 3000])])
def test_many_rows(kind, shape, nq, own):
    """Units whole and cut between CTAs, tiles full and ragged, masked by causality and not."""
    check(Case(shape, nq, own, seed=sum(nq)), kind, seed=sum(own))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape,nq,own", [("8b", [1] * 5, [1, 17, 300, 2500, 9]), ("tiny", [3, 8, 1], [3, 700, 64]),
                                          ("3b", [2, 1], [1111, 2])])
def test_few_rows(kind, shape, nq, own):
    check(Case(shape, nq, own, seed=sum(own)), kind, seed=sum(nq))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", ["8b", "tiny"])
def test_prefixes_and_a_prompt_beside_single_tokens(kind, shape):
    check(Case(shape, [1, 2, 1, 60, 1, 300], [5, 2, 40, 60, 1, 700], [3, 1, 2], [1000, 0, 333], seed=41), kind, seed=43)
