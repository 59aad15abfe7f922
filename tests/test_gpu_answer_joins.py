"""Joins of partial results with heads of 64: batches on both sides of 2500 and 6000 rows (tokens
times query heads), where the join goes by rows, by blocks with eight partials in flight and by
blocks, with and without shared prefixes, and groups whose rows start at any offset.

Tolerance: that of test_gpu_answer.py, derived there."""
import pytest
import torch

from paper_2609_35139_gb300 import cr
from test_gpu_answer import SHAPES, Case

pytestmark = pytest.mark.gpu

SHAPES.setdefault("odd", (7, 1, 64))          # a group's rows start at multiples of 7
SHAPES.setdefault("odd3", (9, 3, 64))


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


def _ragged(tokens):
    """Requests of 1 to 5 new tokens (as many as asked for in all), with 0 to 60 cached before them."""
    nq = []
    while sum(nq) < tokens:
        nq.append(min(1 + (3 * len(nq)) % 5, tokens - sum(nq)))
    return nq, [n + (17 * i) % 61 for i, n in enumerate(nq)]


@pytest.mark.parametrize("prefix", [False, True])
@pytest.mark.parametrize("shape,tokens", [("mqa", 62), ("mqa", 63), ("mqa", 150), ("mqa", 151), ("odd", 357), ("odd", 358),
                                          ("odd", 600), ("odd3", 280), ("odd3", 500)])
def test_rows_on_both_sides_of_the_joins(shape, tokens, prefix):
    nq, own = _ragged(tokens)
    groups = ([3, len(nq) - 4, 1], [700, 129, 33]) if prefix else (None, None)
    Case(shape, nq, own, *groups, seed=tokens).check()


@pytest.mark.parametrize("shape,tokens", [("odd", 870), ("odd3", 690)])
def test_many_rows_over_prefixes(shape, tokens):
    """More than 6000 rows; requests of up to 40 tokens, so that some fill tiles."""
    nq = []
    while sum(nq) < tokens:
        nq.append(min(1 + (11 * len(nq)) % 40, tokens - sum(nq)))
    own = [n + (17 * i) % 61 for i, n in enumerate(nq)]
    for groups in (([1, 2, len(nq) - 3], [40, 300, 1000]), (None, None)):
        Case(shape, nq, own, *groups, seed=tokens).check()
