"""cr_paged_append at its edges: a cache of canonical K takes values as they are."""
import pytest
import torch

from paper_2609_35139_gb300 import AnswerSession, cr

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


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_without_rotation_every_value_is_rounded_alone(d, dtype):
    """An infinity or NaN in one half of a head leaves its partner in the other half as it is."""
    hq, hkv, n = 4, 2, 9
    g = torch.Generator(device="cuda").manual_seed(d)
    q = torch.randn(n, hq * d, generator=g, device="cuda").to(dtype)
    k, v = (torch.randn(n, hkv * d, generator=g, device="cuda").to(dtype) for _ in range(2))
    for x in (q, k, v):
        x[0, 3], x[1, d // 2 + 5], x[2, d - 1] = float("inf"), float("-inf"), float("nan")
    cache = torch.zeros(2, 16, hkv * d, dtype=torch.bfloat16, device="cuda")
    sess = AnswerSession(cr.target_dims(1, hkv, d, hq * d, "bf16"), hq, cache, max_tokens=n)
    out = sess.append(0, q, k, v, torch.arange(n, dtype=torch.int32, device="cuda"),
                      torch.arange(n, dtype=torch.int64, device="cuda"))
    for got, x in ((out, q), (cache[0, :n], k), (cache[1, :n], v)):
        assert torch.equal(torch.isnan(got), torch.isnan(x))
        assert torch.equal(got.nan_to_num(0.5, 9e3, -9e3), x.to(torch.bfloat16).nan_to_num(0.5, 9e3, -9e3))
