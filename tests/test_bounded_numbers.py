"""Numbers of AnswerSession.evict and .sample that 32 bits do not hold are refused, not cut (no GPU needed)."""
import pytest
import torch

from test_bounded_refusals import elsewhere  # noqa: F401  (a fixture)


@pytest.fixture
def session(elsewhere):  # noqa: F811
    """Its tensors lie on the CPU; calls whose arguments are in order end where a current CUDA device is asked for."""
    elsewhere._device_index = -1
    return elsewhere


@pytest.mark.parametrize("x", [2 ** 31, 2 ** 32, 2 ** 32 + 5, -2 ** 31 - 1, 2 ** 70])
def test_evict(session, x):
    a = dict(block_table=torch.zeros(2, 4, dtype=torch.int32), kv_len=torch.zeros(2, dtype=torch.int32),
             keep=torch.zeros(2, dtype=torch.int32), weights=torch.zeros(2, 64), max_keep=5)
    for name in ("first", "last", "max_keep"):
        with pytest.raises(ValueError, match=name):
            session.evict(0, **{**a, name: x})
    for name in ("first", "last"):
        with pytest.raises(ValueError, match="current CUDA device"):
            session.evict(0, **{**a, name: 2 ** 31 - 1})


@pytest.mark.parametrize("x", [2 ** 31, 2 ** 32, 2 ** 32 + 5, -2 ** 31 - 1, 2 ** 70])
def test_sample(session, x):
    logits, u = torch.zeros(3, 100), torch.zeros(3)
    with pytest.raises(ValueError, match="top_k"):
        session.sample(logits, u, top_k=x)
    for good in (0, -1, 2 ** 31 - 1, -2 ** 31):
        with pytest.raises(ValueError, match="current CUDA device"):
            session.sample(logits, u, top_k=good)
