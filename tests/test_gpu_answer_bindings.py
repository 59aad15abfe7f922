"""The answering calls by their bindings of the C ABI (cr.cr_paged_append, cr.cr_attention_plan,
cr.cr_paged_attention, cr.cr_prefix_attention) give what AnswerSession gives, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2609_35139_gb300 import AnswerSession, cr
from test_gpu_answer import Case

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


@pytest.mark.parametrize("members,prefix", [(None, None), ([2, 1], [200, 33])])
def test_attention(members, prefix):
    c = Case("8b", [1, 40, 2], [90, 100, 7], members, prefix, layers=2, layer=1, seed=41)
    want, want_lse = c.run()
    layer = cr.paged_layer(c.cache, 1, c.hkv, c.d, c.block)
    heads = (c.hq, c.hkv, c.d)
    ws = torch.empty(cr.cr_attention_workspace_bytes(*heads, c.cu_q, c.cu_group), dtype=torch.uint8, device="cuda")
    batch = cr.cr_attention_plan(*heads, c.cu_q, ws, c.cu_group)
    out, lse = torch.empty_like(want), torch.empty_like(want_lse)
    if members:
        cr.cr_prefix_attention(layer, batch, c.q, c.table, c.own_len, c.ptable, c.prefix_len, c.scale, out, lse)
    else:
        cr.cr_paged_attention(layer, batch, c.q, c.table, c.own_len, c.scale, out, lse)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append(dtype):
    hq, hkv, d, n = 4, 2, 64, 21
    g = torch.Generator(device="cuda").manual_seed(42)
    q, k, v = (torch.randn(n, h * d, generator=g, device="cuda").to(dtype) for h in (hq, hkv, hkv))
    pos = torch.arange(100, 100 + n, dtype=torch.int32, device="cuda")
    slots = torch.randperm(32, generator=g, device="cuda")[:n]
    freq = (10000.0 ** (-2.0 * np.arange(d // 2) / d)).astype(np.float32)
    for f, mode in ((freq, cr.CR_ROPE_GLOBAL), (None, cr.CR_ROPE_NONE)):
        a, b = (torch.zeros(2, 32, hkv * d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        sess = AnswerSession(cr.target_dims(1, hkv, d, hq * d, "bf16"), hq, a, max_tokens=n, inv_freq_target=f)
        want = sess.append(0, q, k, v, pos, slots)
        out = torch.empty_like(want)
        layer = cr.paged_layer(b, 0, hkv, d, 16)
        cr.cr_paged_append(layer, k, v, pos, slots, f, mode, q, hq, out)
        assert torch.equal(out, want) and torch.equal(a, b)
        b.zero_()
        cr.cr_paged_append(layer, k, v, pos, slots, f, mode)
        assert torch.equal(a, b)
