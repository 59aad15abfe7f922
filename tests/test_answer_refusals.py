"""The answering calls check their arguments on the host before any device work, and the
workspace query follows the batch (no GPU needed)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2609_35139_gb300 import AnswerBatch, AnswerSession, build, cr

FAKE = 0x10000   # 256-byte aligned, never dereferenced: validation fails first
BAD, NO = cr.CR_ERR_INVALID_ARG, cr.CR_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def L():
    build.build()
    return cr.lib()


def _layer(**kw):
    a = dict(k=FAKE, v=FAKE, num_slots=1024, n_kv_heads=8, head_dim=128, block_size=16)
    a.update(kw)
    return cr.cr_paged_layer(**a)


BAD_LAYERS = [(dict(k=None), BAD), (dict(v=FAKE + 8), BAD), (dict(num_slots=15), BAD), (dict(num_slots=0), BAD),
              (dict(num_slots=2 ** 30), BAD), (dict(n_kv_heads=0), BAD), (dict(block_size=0), BAD),
              (dict(block_size=-16), BAD), (dict(block_size=4), NO), (dict(block_size=24), NO),
              (dict(head_dim=96), NO), (dict(head_dim=256), NO)]


def test_append_refusals(L):
    freq = np.ones(64, np.float32)

    def call(layer=None, k=FAKE, ldk=1024, v=FAKE, ldv=1024, q=FAKE, ldq=4096, hq=32, dtype=cr.CR_BF16, n=4, pos=FAKE,
             f=freq.ctypes.data, rope=cr.CR_ROPE_GLOBAL, slots=FAKE, qo=FAKE + 4096, ldqo=4096):
        return L.cr_paged_append(ctypes.byref(layer or _layer()), k, ldk, v, ldv, q, ldq, hq, dtype, n, pos, f, rope,
                                 slots, qo, ldqo, None)

    for kw, want in BAD_LAYERS:
        assert call(_layer(**kw)) == want, kw
    for kw in (dict(k=None), dict(v=None), dict(k=FAKE + 2), dict(ldk=1016), dict(ldk=1028), dict(ldv=1000),
               dict(n=0), dict(n=-1), dict(pos=None), dict(pos=FAKE + 4), dict(f=None), dict(rope=2), dict(slots=None),
               dict(slots=FAKE + 8), dict(dtype=2), dict(hq=0), dict(ldq=4088), dict(ldq=4100), dict(qo=None),
               dict(qo=FAKE + 2), dict(ldqo=4095), dict(qo=FAKE, ldqo=8192), dict(qo=FAKE, dtype=cr.CR_F32),
               dict(dtype=cr.CR_F32, ldk=1026)):
        assert call(**kw) == BAD, kw
    assert L.cr_paged_append(None, FAKE, 1024, FAKE, 1024, None, 0, 0, 1, 4, FAKE, freq.ctypes.data, 1, FAKE, None, 0,
                             None) == BAD


def _plan(L, heads=(32, 8, 128), cu=(0, 1, 3), group=None, ws=FAKE, wsb=1 << 40, n_req=None, batch=True):
    cu = np.array(cu, np.int32)
    g = None if group is None else np.array(group, np.int32)
    b = cr.cr_attention_batch()
    return L.cr_attention_plan(*heads, cu.ctypes.data, len(cu) - 1 if n_req is None else n_req,
                               None if g is None else g.ctypes.data, 0 if g is None else len(g) - 1, ws, wsb,
                               ctypes.byref(b) if batch else None, None)


def test_plan_refusals(L):
    for kw in (dict(cu=(1, 2, 3)), dict(cu=(0, 2, 1)), dict(cu=(0, 0, 0)), dict(n_req=0), dict(n_req=257),
               dict(heads=(0, 8, 128)), dict(heads=(12, 8, 128)), dict(heads=(8, 0, 128)), dict(ws=None),
               dict(ws=FAKE + 128), dict(wsb=1000), dict(batch=False), dict(group=(0, 1)), dict(group=(1, 2)),
               dict(group=(0, 3, 2)), dict(group=(0,))):
        assert _plan(L, **kw) == BAD, kw
    assert _plan(L, heads=(32, 8, 96)) == NO
    assert _plan(L, cu=(0, 1, 2 ** 30)) == NO


def _batch(groups=0, **kw):
    a = dict(n_q_heads=32, n_kv_heads=8, head_dim=128, n_req=2, n_groups=groups, n_tokens=3, workspace=FAKE,
             workspace_bytes=1 << 40)
    a.update(kw)
    b = cr.cr_attention_batch(**a)
    b.n_units[0], b.n_units[1], b.n_ctas, b.n_row_blocks = 16, 16, 1, 16
    return b


def _attend(L, prefix, layer=None, batch=None, q=FAKE, ldq=4096, table=FAKE, mb=64, lens=FAKE, scale=0.1, out=FAKE,
            ldo=4096, lse=None, ptable=FAKE, mpb=64, plens=FAKE):
    b = batch if batch is not None else _batch(1 if prefix else 0)
    head = (ctypes.byref(layer or _layer()), ctypes.byref(b), q, ldq, table, mb, lens)
    tail = (scale, out, ldo, lse, None)
    return L.cr_prefix_attention(*head, ptable, mpb, plens, *tail) if prefix else L.cr_paged_attention(*head, *tail)


@pytest.mark.parametrize("prefix", [False, True])
def test_attention_refusals(L, prefix):
    for kw, want in BAD_LAYERS:
        assert _attend(L, prefix, _layer(**kw)) == want, kw
    for kw in (dict(q=None), dict(q=FAKE + 2), dict(ldq=4000), dict(ldq=4097), dict(table=None), dict(table=FAKE + 4),
               dict(mb=0), dict(lens=None), dict(lens=FAKE + 4), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(out=None), dict(ldo=4088), dict(ldo=4100),
               dict(lse=FAKE + 4)):
        assert _attend(L, prefix, **kw) == BAD, kw
    # a batch planned for other heads, with or without groups where the call wants the other, or never planned
    for kw in (dict(n_kv_heads=4), dict(head_dim=64), dict(groups=0 if prefix else 1), dict(workspace=None),
               dict(n_tokens=0), dict(n_req=0), dict(n_req=257), dict(n_q_heads=4), dict(n_q_heads=36)):
        assert _attend(L, prefix, batch=_batch(**{"groups": 1 if prefix else 0, **kw})) == BAD, kw
    assert _attend(L, prefix, batch=cr.cr_attention_batch()) == BAD
    assert _attend(L, prefix, mb=2 ** 28) == NO           # a longest sequence past 2^30 tokens


def test_prefix_refusals(L):
    for kw in (dict(ptable=None), dict(plens=None), dict(mpb=0), dict(ptable=FAKE + 4)):
        assert _attend(L, True, **kw) == BAD, kw
    assert _attend(L, True, mpb=2 ** 28) == NO


def test_workspace_follows_the_batch(L):
    size = lambda *a: cr.cr_attention_workspace_bytes(*a)
    one = size(32, 8, 128, [0, 1])
    assert 0 < one <= size(32, 8, 128, [0, 1, 2]) <= size(32, 8, 128, [0, 1, 40])
    assert size(32, 8, 128, [0, 1, 2], [0, 2]) >= size(32, 8, 128, [0, 1, 2])
    for bad in ((32, 8, 96, [0, 1]), (30, 8, 128, [0, 1]), (32, 8, 128, [0, 0]), (32, 8, 128, [0, 2, 1]),
                (32, 8, 128, [0, 1], [0, 2]), (32, 0, 128, [0, 1])):
        assert size(*bad) == 0, bad
    # a workspace one byte short is refused
    assert _plan(L, cu=(0, 1), wsb=one - 1) == BAD


def test_session_refusals(L):
    t = cr.target_dims(1, 2, 64, 256, "bf16")
    cache = torch.zeros(2, 64, 128, dtype=torch.bfloat16)
    ok = AnswerSession(t, 4, cache, max_tokens=8, max_requests=2)
    for bad in (cache.float(), cache[:1], cache[:, :, :64], cache.transpose(0, 1)):
        with pytest.raises(ValueError):
            AnswerSession(t, 4, bad, max_tokens=8)
    with pytest.raises(ValueError):
        AnswerSession(cr.target_dims(1, 2, 64, 256, "f32"), 4, cache, max_tokens=8)
    with pytest.raises(ValueError):
        AnswerSession(t, 4, cache, max_tokens=8, inv_freq_target=np.ones(31, np.float32))
    for cu in ([0, 1, 2, 3], [0, 9]):                       # past the session's sizes
        with pytest.raises(ValueError):
            ok.batch(cu)
    with pytest.raises(cr.CrError):
        ok.batch([0, 2, 1])
    b, g = (AnswerBatch(_batch(n, n_q_heads=4, n_kv_heads=2, head_dim=64), None) for n in (0, 1))
    q = torch.zeros(3, 256, dtype=torch.bfloat16)
    table, lens = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for args in ((b, q[:2], table, lens), (b, q.float(), table, lens), (b, q[:, :128], table, lens),
                 (b, q, table[:1], lens), (b, q, table.long(), lens), (b, q, table, lens[:1]), (b, q, table, lens, q[:, :8]),
                 (g, q, table, lens)):
        with pytest.raises(ValueError):
            ok.attend(0, *args)
    with pytest.raises(ValueError):
        ok.attend(0, b, q, table, lens, prefix_table=table, prefix_len=lens)
    with pytest.raises(ValueError):
        ok.attend(0, b, q, table, lens, lse=torch.zeros(3, 2))
    k = torch.zeros(3, 128, dtype=torch.bfloat16)
    pos, slots = torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int64)
    for args in ((q, k, k.float(), pos, slots), (q.float(), k, k, pos, slots), (q, k[:, :64], k, pos, slots),
                 (q, k, k, pos.long(), slots), (q, k, k, pos, slots.int()), (q, k, k, pos[:2], slots),
                 (q, k, k, pos, slots, q.float())):
        with pytest.raises(ValueError):
            ok.append(0, *args)
