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
