"""cr_paged_append at its edges: a cache of canonical K takes values as they are, and positions go
through the whole range of 32 bits.

Tolerance for positions: that of test_gpu_answer.py's append (half a bf16 ulp and 2^-20 of the
pair's size), the angle being exact to within some 2^-23 at every position."""
import numpy as np
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


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("top", [2 ** 17, 2 ** 20, 2 ** 22, 2 ** 24, 2 ** 27, 2 ** 31 - 1])
def test_positions_of_any_size(d, top):
    hq, n = 2, 64
    g = torch.Generator(device="cuda").manual_seed(top % 1000 + d)
    pos = torch.randint(top - top // 8, top, (n,), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    pos[0], pos[1], pos[2] = top, top - 1, -top
    freq = (10000.0 ** (-2.0 * np.arange(d // 2) / d)).astype(np.float32)
    q = torch.randn(n, hq * d, generator=g, device="cuda").to(torch.bfloat16)
    k = torch.zeros(n, d, dtype=torch.bfloat16, device="cuda")
    sess = AnswerSession(cr.target_dims(1, 1, d, hq * d, "bf16"), hq,
                         torch.zeros(2, 64, d, dtype=torch.bfloat16, device="cuda"), max_tokens=n, inv_freq_target=freq)
    got = sess.append(0, q, k, k, pos, torch.arange(n, dtype=torch.int64, device="cuda")).double().view(n, hq, d)
    # pos f has up to 55 bits: the position in two parts, so that both products are exact in 64
    f = freq.astype(np.float64)
    p = pos.cpu().numpy().astype(np.int64)
    hi, lo = (p >> 16 << 16).astype(np.float64), (p & 0xffff).astype(np.float64)
    a, b = (torch.from_numpy(x[:, None] * f[None]) for x in (hi, lo))      # 15 + 24 and 16 + 24 bits
    ca, sa, cb, sb = a.cos(), a.sin(), b.cos(), b.sin()
    c, s = (ca * cb - sa * sb).cuda()[:, None], (sa * cb + ca * sb).cuda()[:, None]
    x = q.double().view(n, hq, d)
    u, w = x[..., :d // 2], x[..., d // 2:]
    exact = torch.cat([u * c - w * s, w * c + u * s], -1)
    size = torch.sqrt(u * u + w * w).repeat(1, 1, 2)
    half_ulp = torch.exp2(torch.floor(torch.log2(exact.abs().clamp(min=1e-30))) - 8)
    assert float(((got - exact).abs() - half_ulp - 2.0 ** -20 * size).max()) <= 0.0
