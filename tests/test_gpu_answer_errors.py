"""What the attention over a paged cache gives when an index is out of range: a block outside the
cache is read as zeros, a length is clamped, both are recorded, and nothing else changes, neither
in that call nor in a later one.

Tolerance: that of test_gpu_answer.py, derived there."""
import time

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


def _reported():
    st, word = cr.cr_get_device_status()
    cr.cr_clear_device_status()
    assert st == cr.CR_ERR_DEVICE_INDEX, word


BATCHES = {"rows": ("8b", [1] * 12, [3000 + 37 * i for i in range(12)], None, None),
           "tiles": ("8b", [90, 200], [4000, 700], None, None),
           "both": ("7b", [1, 60, 2], [2000, 900, 800], [2, 1], [3000, 500])}


@pytest.mark.parametrize("batch", list(BATCHES))
def test_an_index_error_recorded_before_changes_nothing(batch):
    """An append that met a slot outside its cache has set the status word; it has not been cleared."""
    c = Case(*BATCHES[batch], seed=31)
    sess = c.session()
    small = torch.zeros(1, c.hkv * c.d, dtype=torch.bfloat16, device="cuda")
    sess.append(0, None, small, small, torch.zeros(1, dtype=torch.int32, device="cuda"),
                torch.tensor([c.cache.shape[1]], dtype=torch.int64, device="cuda"))
    c.check(sess=sess)
    _reported()


@pytest.mark.parametrize("batch", list(BATCHES))
def test_a_bad_block_reads_as_zeros_and_the_rest_is_unchanged(batch):
    c = Case(*BATCHES[batch], seed=32)
    j = 5                                               # of the first request's blocks
    spare = sorted(set(range(c.cache.shape[1] // c.block)) -
                   {int(s) // c.block for r in c.rows for s in r.tolist()})[0]
    c.cache[:, spare * c.block:(spare + 1) * c.block] = 0.0
    c.rows[0][j * c.block:(j + 1) * c.block] = torch.arange(spare * c.block, (spare + 1) * c.block, device="cuda")
    for bad in (c.cache.shape[1] // c.block + 4, -7, 2 ** 31 - 1):
        c.table[0, j] = bad
        c.check()
        _reported()


@pytest.mark.parametrize("batch", list(BATCHES))
def test_lengths_are_clamped_and_the_rest_is_unchanged(batch):
    c = Case(*BATCHES[batch], seed=33)
    own, last = list(c.own), len(c.own) - 1
    c.own_len[last] = -3                                # nothing of its own
    c.own[last] = 0
    c.check()
    _reported()
    # a length past the table: all of the table's blocks (the longest request's, its last one brought to full)
    longest, width = own.index(max(own)), c.table.shape[1] * c.block
    c.cache[torch.isnan(c.cache)] = 0.0
    c.table[last] = c.table[longest]
    k = torch.arange(width, device="cuda")
    c.rows[last] = c.table[last].long()[k // c.block] * c.block + k % c.block
    c.own_len[last] = width + 1
    c.own[last] = width
    c.check()
    _reported()


def test_a_wait_goes_on_after_an_index_error():
    """Only a timeout ends other waits: one that nothing satisfies runs to its limit of 2 s although an
    index error stands in the status word, and is then what the word tells."""
    cache = torch.zeros(2, 16, 128, dtype=torch.bfloat16, device="cuda")
    sess = AnswerSession(cr.target_dims(1, 2, 64, 256, "bf16"), 4, cache, max_tokens=1)
    k = torch.ones(1, 128, dtype=torch.bfloat16, device="cuda")
    sess.append(0, None, k, k, torch.zeros(1, dtype=torch.int32, device="cuda"),
                torch.tensor([16], dtype=torch.int64, device="cuda"))
    assert cr.cr_get_device_status()[0] == cr.CR_ERR_DEVICE_INDEX
    t0 = time.perf_counter()
    cr.cr_wait_selftest()
    st, word = cr.cr_get_device_status()
    took = time.perf_counter() - t0
    cr.cr_clear_device_status()
    assert st == cr.CR_ERR_TIMEOUT and list(word[:2]) == [1, 900], word
    assert 1.5 < took < 30.0, took


@pytest.mark.parametrize("batch", list(BATCHES))
def test_lengths_that_change_during_a_call_end_it_all_the_same(batch):
    """Another stream writes kv_len and prefix_len while calls run: their results are undefined, but
    each ends, records nothing, and leaves the plan fit for the calls that follow."""
    c = Case(*BATCHES[batch], seed=34)
    sess = c.session()
    b = sess.batch(c.cu_q, c.cu_group)
    want, _ = c.run(sess=sess, batch=b, lse=False)
    c.check(sess=sess, batch=b)
    kw = {} if c.cu_group is None else {"prefix_table": c.ptable, "prefix_len": c.prefix_len}
    lens = [c.own_len] + ([] if c.cu_group is None else [c.prefix_len])
    full = [x.clone() for x in lens]
    others = [[(x * f).to(torch.int32) for f in (0.0, 1.0, 0.01, 0.6)] for x in full]
    out = torch.empty_like(want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(400):
        with torch.cuda.stream(side):
            for k in range(4):
                for x, values in zip(lens, others):
                    x.copy_(values[(i + k) % 4])
        sess.attend(0, b, c.q, c.table, c.own_len, out, **kw)
    torch.cuda.synchronize()
    assert cr.cr_get_device_status()[0] == cr.CR_OK
    for x, value in zip(lens, full):
        x.copy_(value)
    again, _ = c.run(sess=sess, batch=b, lse=False)
    assert torch.equal(again, want)
