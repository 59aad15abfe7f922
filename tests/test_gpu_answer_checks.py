"""AnswerSession refuses a tensor of the host among those of the GPU, each argument by itself,
before anything is launched."""
import pytest
import torch

from paper_2609_35139_gb300 import cr
from test_gpu_answer import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2609_35139_gb300 import build
    build.build()


@pytest.mark.parametrize("which", range(6))
def test_append_with_one_tensor_of_the_host(which):
    c = Case("tiny", [3], [9], seed=1)
    k = torch.zeros(3, c.hkv * c.d, dtype=torch.bfloat16, device="cuda")
    args = [c.q, k, k.clone(), torch.zeros(3, dtype=torch.int32, device="cuda"),
            torch.full((3,), -1, dtype=torch.int64, device="cuda"), torch.empty_like(c.q)]
    sess = c.session()
    sess.append(0, *args)
    args[which] = args[which].cpu()
    with pytest.raises(ValueError, match="cuda:0"):
        sess.append(0, *args)
    torch.cuda.synchronize()


@pytest.mark.parametrize("which", ["q", "block_table", "kv_len", "out", "lse", "prefix_table", "prefix_len"])
def test_attend_with_one_tensor_of_the_host(which):
    c = Case("tiny", [3, 1], [9, 4], [2], [40], seed=2)
    sess = c.session()
    batch = sess.batch(c.cu_q, c.cu_group)
    kw = dict(q=c.q, block_table=c.table, kv_len=c.own_len, out=torch.empty_like(c.q),
              lse=torch.empty(4, c.hq, device="cuda"), prefix_table=c.ptable, prefix_len=c.prefix_len)
    sess.attend(0, batch, **kw)
    kw[which] = kw[which].cpu()
    with pytest.raises(ValueError, match="cuda:0"):
        sess.attend(0, batch, **kw)
    torch.cuda.synchronize()


def test_one_row_may_have_any_row_stride():
    """A single row is contiguous whatever torch says that the next would be (here one value on)."""
    c = Case("tiny", [1], [20], seed=3)
    sess = c.session()
    want, _ = c.run(sess=sess, lse=False)
    q = torch.empty(c.hq * c.d, 1, dtype=torch.bfloat16, device="cuda").copy_(c.q.t()).t()
    assert q.stride() == (1, 1)
    out = torch.empty(c.hq * c.d, 1, dtype=torch.bfloat16, device="cuda").t()
    assert torch.equal(sess.attend(0, sess.batch(c.cu_q), q, c.table, c.own_len, out), want) and torch.equal(out, want)
    k = torch.zeros(c.hkv * c.d, 1, dtype=torch.bfloat16, device="cuda").t()
    got = sess.append(0, q, k, k, torch.zeros(1, dtype=torch.int32, device="cuda"),
                      torch.full((1,), -1, dtype=torch.int64, device="cuda"), torch.empty_like(out))
    assert torch.equal(got, q)
