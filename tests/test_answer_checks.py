"""What AnswerSession refuses before anything is launched (no GPU needed)."""
import pytest
import torch

from paper_2609_35139_gb300 import AnswerBatch, AnswerSession, build, cr


@pytest.fixture(scope="module")
def sess():
    build.build()
    cache = torch.zeros(2, 64, 128, dtype=torch.bfloat16)
    return AnswerSession(cr.target_dims(1, 2, 64, 256, "bf16"), 4, cache, max_tokens=8, max_requests=2)


def _batch(n_q_heads=4, groups=0):
    b = cr.cr_attention_batch(n_q_heads=n_q_heads, n_kv_heads=2, head_dim=64, n_req=2, n_groups=groups, n_tokens=3,
                              workspace=0x10000, workspace_bytes=1 << 30)
    return AnswerBatch(b, None)


def _args(q_heads=4):
    q = torch.zeros(3, 64 * q_heads, dtype=torch.bfloat16)
    return q, torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)


@pytest.mark.parametrize("groups", [0, 1])
@pytest.mark.parametrize("heads", [2, 6, 8])
def test_a_batch_of_other_query_heads(sess, heads, groups):
    """Heads would meet other KV heads, and columns of the output past the plan's stay as they were."""
    q, table, lens = _args()
    with pytest.raises(ValueError, match="query heads"):
        sess.attend(0, _batch(heads, groups), q, table, lens, prefix_table=table[:1] if groups else None,
                    prefix_len=lens[:1] if groups else None)


@pytest.fixture
def elsewhere(sess):
    """A session whose cache counts as the first GPU's, with every tensor on the CPU."""
    was, sess._device_index = sess._device_index, 0
    yield sess
    sess._device_index = was


@pytest.mark.parametrize("q_out", [False, True])
def test_append_refuses_tensors_of_another_device(elsewhere, q_out):
    q = torch.zeros(3, 256, dtype=torch.bfloat16)
    k = torch.zeros(3, 128, dtype=torch.bfloat16)
    pos, slots = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="cuda:0"):
        elsewhere.append(0, q, k, k, pos, slots, q if q_out else None)
    with pytest.raises(ValueError, match="cuda:0"):
        elsewhere.append(0, None, k, k, pos, slots)


@pytest.mark.parametrize("groups", [0, 1])
def test_attend_refuses_tensors_of_another_device(elsewhere, groups):
    q, table, lens = _args()
    kw = dict(prefix_table=table[:1], prefix_len=lens[:1]) if groups else {}
    with pytest.raises(ValueError, match="cuda:0"):
        elsewhere.attend(0, _batch(4, groups), q, table, lens, torch.zeros_like(q), **kw)


def test_a_cache_that_is_not_on_a_gpu_is_never_launched_on(sess):
    q, table, lens = _args()
    k = torch.zeros(3, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current CUDA device"):
        sess.attend(0, _batch(), q, table, lens)
    with pytest.raises(ValueError, match="current CUDA device"):
        sess.append(0, q, k, k, lens.repeat(2)[:3], torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="current CUDA device"):
        sess.batch([0, 1, 3])


def test_the_append_binding_takes_one_type_for_all():
    layer = cr.cr_paged_layer(0x10000, 0x10000, 64, 2, 64, 16)
    k, q = torch.zeros(3, 128, dtype=torch.bfloat16), torch.zeros(3, 256, dtype=torch.bfloat16)
    pos, slots = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    for kk, vv, qq in ((k.half(), k.half(), None), (k.float(), k, None), (k, k.float(), None), (k, k, q.float()),
                       (k.double(), k.double(), q.double())):
        with pytest.raises(ValueError, match="alike"):
            cr.cr_paged_append(layer, kk, vv, pos, slots, None, cr.CR_ROPE_NONE, qq, 4, q)
