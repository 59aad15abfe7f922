"""cr_sample over rows of which a mask leaves few tokens, as constrained decoding gives them: fewer
than top_k, in lists short and long, beside every other filter.  The checks are those of
test_gpu_sample.py, with its tolerance."""
import math

import pytest
import torch

from test_gpu_sample import check, lib, logits, sess  # noqa: F401  (lib, sess: fixtures)

pytestmark = pytest.mark.gpu


def masked(n, v, allowed, seed, dtype=torch.float32):
    """Rows of v logits with allowed[r] of them, anywhere, above -inf, and a u for each."""
    x, u = logits(n, v, dtype, seed=seed, std=1.5)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    rank = torch.rand(n, v, generator=g, device="cuda").argsort(1).argsort(1)
    return x.masked_fill_(rank >= torch.tensor(allowed, device="cuda")[:, None], -math.inf), u


def used_before(sess):
    """Calls whose rows leave sums of many sizes behind in the SMs' shared memory."""
    x, u = logits(600, 3001, seed=99)
    sess.sample(x, u, top_k=100, top_p=0.9)
    sess.sample(x[:40], u[:40].clone(), top_k=100, top_p=0.9, temperature=0.05)


@pytest.mark.parametrize("top_p", [0.5, 0.95, 1.0])
@pytest.mark.parametrize("top_k", [50, 128, 200, 1000])
@pytest.mark.parametrize("v", [1500, 32003, 131072])
def test_fewer_tokens_than_top_k_in_a_short_list(sess, v, top_k, top_p):
    """1 to 256 tokens: those that are left are compared each with each."""
    used_before(sess)
    allowed = [1, 2, 3, 5, 10, 29, 30, 49, 50, 51, 100, 127, 128, 129, 199, 200, 201, 255, 256] + list(range(4, 256, 6))
    x, u = masked(len(allowed), v, allowed, seed=v + top_k)
    check(sess, x, u, top_k=top_k, top_p=top_p)
    for r in range(2, 14):
        used_before(sess)
        check(sess, x[r:r + 1], u[r:r + 1].clone(), top_k=top_k, top_p=top_p)
    check(sess, x, u, top_k=top_k, top_p=top_p, min_p=0.1, temperature=0.6)


@pytest.mark.parametrize("top_p", [0.5, 0.95, 1.0])
@pytest.mark.parametrize("top_k,v", [(128, 1500), (128, 4000), (1000, 131072), (1000, 262144), (512, 100003)])
def test_fewer_tokens_than_top_k_in_a_long_list(sess, v, top_k, top_p):
    """More tokens left than are compared each with each, fewer than top_k; and just as many, and more."""
    used_before(sess)
    allowed = [257, 258, 290, 300, 333, 400, 499, 500, 501, 511, 512, 513, 700, 900, 998, 999, 1000, 1001, 1100]
    allowed = [a for a in allowed if a <= v // 2]
    x, u = masked(len(allowed), v, allowed, seed=v + top_k)
    check(sess, x, u, top_k=top_k, top_p=top_p)
    check(sess, x, u, top_k=top_k, top_p=top_p, min_p=0.05, temperature=1.7)
    for r in range(0, len(allowed), 2):
        used_before(sess)
        check(sess, x[r:r + 1], u[r:r + 1].clone(), top_k=top_k, top_p=top_p)
        check(sess, x[r:r + 1].to(torch.bfloat16), u[r:r + 1].clone(), top_k=top_k, top_p=top_p)


@pytest.mark.parametrize("kw", [dict(top_k=50, top_p=0.9), dict(top_k=1000, top_p=0.9), dict(top_k=1000), dict(top_p=0.9)])
def test_masked_rows_by_the_batch(sess, kw):
    """Clusters of every size, a CTA a row among them; all that a mask leaves in one place of the vocabulary."""
    for n, v in ((1, 40000), (30, 40000), (64, 40000), (100, 40000), (160, 9000)):
        x, u = masked(n, v, [1 + (37 * r) % 700 for r in range(n)], seed=n)
        check(sess, x, u, **kw)
        used_before(sess)
        together = torch.full_like(x, -math.inf)
        together[:, 5000:5600] = x[:, :600].nan_to_num(neginf=-1.5)
        check(sess, together, u, **kw)


def test_equal_calls_give_equal_tokens_whatever_ran_before(sess):
    """Rows short of top_k, behind calls that leave other sums behind."""
    x, u = masked(24, 131072, [3 + 29 * r for r in range(24)], seed=3)
    want = [sess.sample(x, u, top_k=k, top_p=0.9).clone() for k in (50, 1000)]
    for t in (0.03, 1.0, 8.0):
        y, _ = logits(600, 3001, seed=int(10 * t))
        sess.sample(y, torch.rand(600, device="cuda"), top_k=100, top_p=0.9, temperature=t)
        for k, w in zip((50, 1000), want):
            assert torch.equal(sess.sample(x, u, top_k=k, top_p=0.9), w)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("low", [None, -1e9, -1e4])
@pytest.mark.parametrize("kw", [dict(top_k=50, top_p=0.95), dict(top_k=50), dict(top_k=1000, top_p=0.9), dict(top_p=0.9),
                                dict(top_k=5, min_p=0.05), dict(temperature=0.4), dict()])
def test_masks_of_finite_values(sess, dtype, low, kw):
    """The type's lowest value, or another far down: never drawn, though it counts among top_k's."""
    low = torch.finfo(dtype).min if low is None else low
    for n, v in ((1, 131072), (9, 32003), (40, 1500)):
        x, u = masked(n, v, [1 + (53 * r + 10) % 700 for r in range(n)], seed=n, dtype=dtype)
        token = check(sess, x.clamp(min=low), u, **kw)
        assert bool((x.gather(1, token[:, None]) > -math.inf).all())
        x, u = logits(n, v, dtype, seed=n)
        x[:, v - v // 9:] = low
        token = check(sess, x, u, **kw)
        assert int(token.max()) < v - v // 9
