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
