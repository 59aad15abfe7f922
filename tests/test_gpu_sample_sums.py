"""cr_sample's sums against float64 where many logits weigh the same: an error that they share adds up.

Tolerance, derived before any run: a weight is off by 2^-26.8 of itself at most (the bound stands at the
kernel's weight_parts), and what is cut off below 2^-44 of the largest is 2^-26 of weights above 2^-18, as all
are here.  A sum's share S of another is then off by S (1 - S) <= 1/4 of the difference of two such errors: by
(2 * 2^-26.8 + 2^-26) / 4 < 2^-26, which is test_gpu_sample.py's EDGE.  Every u and top_p below stands at least that
far from a border, so the token is the one that float64 gives."""
import math

import numpy as np
import pytest
import torch

from test_gpu_sample import EDGE, check, lib, logits, plain, sess  # noqa: F401  (lib, sess: fixtures)

pytestmark = pytest.mark.gpu

# top, the others' value, temperature: the difference of the two does not fit fp32
ROWS = [(10.3, 0.1, 1.0), (8.45, 0.013, 0.7), (60.3, 0.7, 5.4), (-0.3, -10.7, 1.0), (0.3, -10.1, 1.0), (11.9, 1.1, 1.0)]


def beside(border, up):
    """The fp32 number next to a border that lies EDGE or more above (below) it."""
    at = border + EDGE if up else border - EDGE
    f = np.float32(at)
    if up and float(f) < at:
        f = np.nextafter(f, np.float32(2))
    if not up and float(f) > at:
        f = np.nextafter(f, np.float32(-1))
    return float(f)


def row(top, value, temperature, top_at):
    """A peak and a flat rest that weighs about as much."""
    a, b, t = (float(np.float32(x)) for x in (top, value, temperature))
    lost = abs(float(np.float32(b) - np.float32(a)) - (b - a)) / t
    assert lost > 2.0 ** -24, lost
    n = round(math.exp((a - b) / t))
    x = torch.full((n + 1,), b, device="cuda")
    x[top_at] = a
    return x, n, math.exp((b - a) / t), t


@pytest.mark.parametrize("top,value,temperature", ROWS)
def test_tokens_beside_borders_of_a_flat_rest(sess, top, value, temperature):
    x, n, w, t = row(top, value, temperature, -1)
    js = sorted({int(n * (0.55 + 0.44 * i / 23)) for i in range(24)})
    borders = [j * w / (1.0 + n * w) for j in js]
    u = [beside(b, up) for b in borders for up in (False, True)]
    want = [j - 1 + up for j in js for up in (False, True)]
    u = torch.tensor(u, device="cuda")
    rows = x.expand(len(want), -1).contiguous()
    assert plain(x, u[0].item(), t, 0, 1.0, 0.0)[0] == want[0]
    assert sess.sample(rows, u, temperature=temperature).tolist() == want
    assert sess.sample(rows, u, temperature=temperature, min_p=2.0 ** -19).tolist() == want
    for r in (0, len(want) // 2, len(want) - 1):          # one row of many CTAs
        assert sess.sample(rows[r:r + 1], u[r:r + 1].clone(), temperature=temperature).tolist() == want[r:r + 1]


@pytest.mark.parametrize("top,value,temperature", ROWS)
@pytest.mark.parametrize("top_k", [0, 1])
def test_the_cut_of_top_p_in_a_flat_rest(sess, top, value, temperature, top_k):
    """top_p beside a border: which of the equal ones is the last that stays (drawn by u = 1).  top_k 1: a
    top_k that leaves three quarters of them."""
    x, n, w, t = row(top, value, temperature, 0)
    m = n * 3 // 4 if top_k else n                        # of the rest
    js = sorted({int(m * (0.3 + 0.6 * i / 15)) for i in range(16)})
    p = [beside((1.0 + j * w) / (1.0 + m * w), up) for j in js for up in (False, True)]
    want = [j + up for j in js for up in (False, True)]   # (before token j + 1 stand the top and j others)
    p = torch.tensor(p, device="cuda")
    rows = x.expand(len(want), -1).contiguous()
    u = torch.ones(len(want), device="cuda")
    k = m + 1 if top_k else 0
    assert plain(x, 1.0, t, k, p[0].item(), 0.0)[0] == want[0]
    assert sess.sample(rows, u, temperature=temperature, top_k=k, top_p=p).tolist() == want
    r = len(want) // 2
    assert sess.sample(rows[r:r + 1], u[:1], temperature=temperature, top_k=k, top_p=p[r].item()).tolist() == want[r:r + 1]


@pytest.mark.parametrize("middle,temperature", [(1e4, 0.05), (9e4, 1.0), (90848.0, 1.0), (90856.0, 1.0), (-1e4, 0.1), (-1e6, 1.0),
                                                (3e-5, 1e-6), (2.5e30, 1e25)])
@pytest.mark.parametrize("kw", [dict(), dict(top_p=0.8), dict(top_k=60, top_p=0.9), dict(min_p=0.01)])
def test_logits_far_from_zero_in_units_of_the_temperature(sess, middle, temperature, kw):
    """Either side of where the weights are told from the largest logit instead of from zero."""
    x, u = logits(6, 5003, seed=17, std=2.5 * temperature)
    check(sess, x + middle, u, temperature=temperature, **kw)


@pytest.mark.parametrize("value", [0.0, 0.0433, 0.7, -3.3, 33.3])
def test_sums_of_the_most_equal_logits(sess, value):
    """2^20 - 1 largest weights: the sum stays below 2^64, and a token's place is u times their number."""
    v = 1048575
    u = torch.tensor([0.0, 0.1, 0.5, 0.99, 0.99999994], device="cuda")
    x = torch.full((5, v), value, device="cuda")
    assert sess.sample(x, u).tolist() == [int(a * v) for a in u.double().tolist()]
    assert sess.sample(x, u, top_p=0.9999).max() < v
