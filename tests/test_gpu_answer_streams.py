"""The answering calls with a stream of their own given by `stream=`: what they allocate is that
stream's, neither still in use by earlier work of another stream nor given back to one too early."""
import pytest
import torch

from paper_2609_35139_gb300 import cr
from test_gpu_answer import Case

pytestmark = pytest.mark.gpu

BUSY = 100_000_000        # clocks: some 50 ms of a stream


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


def _case():
    c = Case("8b", [1] * 30, [5 + i for i in range(30)], [30], [4000], seed=2)
    want, _ = c.run(lse=False)
    return c, c.session(), {"prefix_table": c.ptable, "prefix_len": c.prefix_len}, want


def _late_fill(like, value):
    """Memory like that of a tensor that is about to be allocated, given back while the current
    stream, which is busy, has still to write it."""
    junk = torch.empty_like(like)
    torch.cuda._sleep(BUSY)
    junk.fill_(value)


@pytest.mark.parametrize("raw", [False, True])
def test_outputs_belong_to_the_given_stream(raw):
    c, sess, kw, want = _case()
    batch = sess.batch(c.cu_q, c.cu_group)
    n = c.q.shape[0]
    k = torch.ones(n, c.hkv * c.d, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(n, dtype=torch.int32, device="cuda")
    skip = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    st = side.cuda_stream if raw else side
    _late_fill(want, 7.0)
    out = sess.attend(0, batch, c.q, c.table, c.own_len, stream=st, **kw)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    _late_fill(want, 7.0)
    q = sess.append(0, c.q, k, k, pos, skip, stream=st)       # no rotation: a copy
    torch.cuda.synchronize()
    assert torch.equal(q, c.q)


@pytest.mark.parametrize("raw", [False, True])
def test_a_batch_belongs_to_the_given_stream(raw):
    """Planned on a stream of its own: its workspace is neither one that the current stream has still
    to write, nor, once the batch is dropped, the current stream's to write before the call is done."""
    c, sess, kw, want = _case()
    need = sess.batch(c.cu_q, c.cu_group).workspace.numel()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    st = side.cuda_stream if raw else side
    _late_fill(torch.empty(need, dtype=torch.uint8, device="cuda"), 255)
    batch = sess.batch(c.cu_q, c.cu_group, stream=st)
    out = torch.empty_like(want)
    side.synchronize()                                  # the plan is made, the fill still waits
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
    sess.attend(0, batch, c.q, c.table, c.own_len, out, stream=st, **kw)
    del batch
    junk = [torch.empty(need, dtype=torch.uint8, device="cuda").fill_(255) for _ in range(2)]
    torch.cuda.synchronize()
    assert torch.equal(out, want) and len(junk) == 2


@pytest.mark.parametrize("how", ["given", "current"])
def test_a_dropped_batch_outlasts_its_calls_on_another_stream(how):
    """Planned on the current stream, used on another: the workspace does not come back before the
    other stream is done with it."""
    c, sess, kw, want = _case()
    batch = sess.batch(c.cu_q, c.cu_group)
    need, at = batch.workspace.numel(), batch.workspace.data_ptr()
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
        if how == "current":
            sess.attend(0, batch, c.q, c.table, c.own_len, out, **kw)
    if how == "given":
        sess.attend(0, batch, c.q, c.table, c.own_len, out, stream=side, **kw)
    del batch
    junk = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert junk.data_ptr() != at
    junk.fill_(255)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_a_dropped_batch_of_another_stream_outlasts_its_calls_on_the_default_one():
    c, sess, kw, want = _case()
    side = torch.cuda.Stream()
    batch = sess.batch(c.cu_q, c.cu_group, stream=side)
    need, at = batch.workspace.numel(), batch.workspace.data_ptr()
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    sess.attend(0, batch, c.q, c.table, c.own_len, out, **kw)
    del batch
    with torch.cuda.stream(side):
        junk = torch.empty(need, dtype=torch.uint8, device="cuda")
        assert junk.data_ptr() != at
        junk.fill_(255)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
