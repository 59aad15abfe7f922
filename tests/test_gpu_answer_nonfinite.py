"""Queries and keys that are not finite, in the attention over a paged cache.  A row that sees
nothing gets zeros; every other row gets what the definition gives, NaN where a score that it
sees is NaN or +inf or where all of them are -inf, and what it does not see does not reach it.

Tolerance: that of test_gpu_answer.py (derived there) for the finite rows."""
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


# one batch for each way in which a row ends: joined by a CTA, by a warp, in blocks (eight partials
# deep and one), finished by the kernel of tiles, and joined with a prefix
WAYS = {"cta": ("8b", [1], [300], None, None), "warp": ("3b", [1] * 20, [50] * 20, None, None),
        "deep": ("8b", [1] * 100, [9] * 100, None, None), "blocks": ("8b", [1] * 200, [5] * 200, None, None),
        "tiles": ("7b", [130], [500], None, None), "finished": ("8b", [33] * 20, [45] * 20, None, None),
        "prefix_cta": ("tiny", [1, 2], [5, 9], [2], [130]), "prefix": ("8b", [33] * 9, [45] * 9, [9], [257])}


def _check(c):
    """The finite outputs within the bound, the others NaN; the log-sum-exp finite in the same places."""
    out, lse = c.run()
    e, el, vmax = c.exact()
    o = out.double()
    assert torch.equal(torch.isnan(o), torch.isnan(e)), (int(torch.isnan(o).sum()), int(torch.isnan(e).sum()))
    ok = torch.isfinite(e)
    assert float(((o - e).abs() - (2.0 ** -8 * vmax + 2.0 ** -8 * e.abs()))[ok].max()) <= 0.0
    ok = torch.isfinite(el)
    assert torch.equal(torch.isfinite(lse), ok)
    assert float((lse.double() - el)[ok].abs().max()) <= 1e-3
    return out, lse, e, el


@pytest.mark.parametrize("way", list(WAYS))
def test_a_nan_query_gives_nan(way):
    shape, nq, own, members, prefix = WAYS[way]
    c = Case(shape, nq + [2], own + [30], members and members[:-1] + [members[-1] + 1], prefix, seed=5)
    n, d = c.q.shape[0], c.d
    c.q[0] = float("nan")                       # a whole token, and one head of the last
    c.q[n - 1, d] = float("nan")
    out, lse, e, _ = _check(c)
    assert bool(torch.isnan(out[0]).all()) and bool(torch.isnan(lse[0]).all())
    assert bool(torch.isnan(out[n - 1, d:2 * d]).all()) and bool(torch.isfinite(out[n - 1, :d]).all())


@pytest.mark.parametrize("way", list(WAYS))
def test_a_key_that_is_not_finite_reaches_the_rows_that_see_it(way):
    """NaN in one KV head of a request's last key, +inf in a component of another's middle key: by the
    sign of the row's query there its score is +inf (the row is NaN) or -inf (the key has no weight)."""
    shape, nq, own, members, prefix = WAYS[way]
    c = Case(shape, nq + [2], own + [30], members and members[:-1] + [members[-1] + 1], prefix, seed=6)
    width, d = c.hkv * c.d, c.d
    c.cache[0, c.rows[len(nq)][-1], width - d:] = float("nan")
    c.cache[0, c.rows[0][own[0] // 2], 5] = float("inf")
    out, _, e, _ = _check(c)
    assert bool(torch.isfinite(e[-2]).all()) and bool(torch.isnan(e[-1]).any())
    seen = c.q[nq[0] - 1].view(c.hq, d)[:c.hq // c.hkv, 5].float()
    assert torch.equal(torch.isnan(out[nq[0] - 1].view(c.hq, d)[:c.hq // c.hkv, 0]), seen > 0)


@pytest.mark.parametrize("shape,nq,own", [("8b", [1, 1], [1, 40]), ("7b", [40, 1], [40, 3]), ("mqa", [2], [2])])
def test_all_scores_minus_infinity(shape, nq, own):
    """A row whose only key has the score -inf: 0 / 0, and the logarithm of a sum of nothing but zeros."""
    c = Case(shape, nq, own, seed=7)
    c.cache[0, c.rows[0][0], 5] = float("inf")
    c.q[0].view(c.hq, c.d)[:, 5] = -1.0
    out, lse, _, _ = _check(c)
    heads = c.hq // c.hkv
    assert bool(torch.isnan(out[0].view(c.hq, c.d)[:heads]).all()) and bool(torch.isneginf(lse[0, :heads]).all())


@pytest.mark.parametrize("shape,nq,own", [("8b", [4, 1], [1, 9]), ("7b", [40], [3]), ("8b", [33] * 20, [1] * 20)])
def test_a_row_that_sees_nothing_gets_zeros_whatever_its_query_is(shape, nq, own):
    c = Case(shape, nq, own, seed=8)
    c.q[0] = float("nan")
    out, lse, _, _ = _check(c)
    assert bool((out[0] == 0).all()) and bool(torch.isneginf(lse[0]).all())
