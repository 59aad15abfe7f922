"""Weighing, evicting and sampling at their largest: offsets past 2^31 elements, the longest requests."""
import pytest
import torch

from paper_2609_35139_gb300 import AnswerSession, cr
from test_gpu_answer import Case
from test_gpu_evict import Pages
from test_gpu_weigh import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2609_35139_gb300 import build
    build.build()
    cr.cr_clear_device_status()
    yield
    torch.cuda.empty_cache()
    st, word = cr.cr_get_device_status()
    assert st == cr.CR_OK, f"device status {word}"


@pytest.mark.parametrize("nq,own", [([1, 1], [700, 33]), ([40], [600])])
def test_weights_of_a_plane_of_more_than_2_31_values(nq, own):
    c = Case("8b", nq, own, extra_blocks=(1 << 31) // (1024 * 16) + 999, seed=41)
    assert max(int(x.max()) for x in c.rows) * 1024 > 1 << 31
    check(c)


def test_eviction_behind_2_31_values():
    p = Pages([700, 300], hkv=8, d=128, layers=1, layer=0, seed=42)
    width, slots = 1024, p.cache.shape[1]
    more = (1 << 31) // (width * p.block) + 1
    behind = more * p.block
    cache = torch.zeros(2, behind + slots, width, dtype=torch.bfloat16, device="cuda")
    cache[:, behind:] = p.cache
    weights = torch.zeros(8, behind + slots, device="cuda")
    weights[:, behind:] = p.weights
    p.cache, p.weights = cache, weights
    p.table = torch.where(p.table >= 0, p.table + more, p.table)
    p.slots = [x + behind for x in p.slots]
    p.session = AnswerSession(cr.target_dims(1, 8, 128, 4096, "bf16"), 32, cache, block_size=p.block, max_tokens=1)
    p.check(250, first=4, last=32)


@pytest.mark.parametrize("n", [380000, 400003])
def test_eviction_of_the_longest_requests(n):
    """The keys of eight CTAs fill their shared memory, or do not fit it and are read again."""
    Pages([n], hkv=2, d=64, block=64, kind="ties", seed=n).check(100001, first=4, last=256)


@pytest.mark.parametrize("kw", [dict(top_k=30), dict(top_p=0.8), dict()])
def test_rows_of_logits_behind_2_31_values(kw):
    rows, vocab, ld = 2100, 5000, (1 << 20) + 24
    g = torch.Generator(device="cuda").manual_seed(43)
    x = torch.empty(rows, ld, dtype=torch.bfloat16, device="cuda")[:, :vocab]
    x.copy_(torch.randn(rows, vocab, generator=g, device="cuda").mul_(3.0))
    u = torch.rand(rows, generator=g, device="cuda")
    s = AnswerSession(cr.target_dims(1, 2, 64, 256, "bf16"), 4, torch.empty(2, 16, 128, dtype=torch.bfloat16, device="cuda"), max_tokens=1)
    assert torch.equal(s.sample(x, u, **kw), s.sample(x.contiguous(), u, **kw))
