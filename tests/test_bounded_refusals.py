"""The weighing, evicting and sampling calls check their arguments on the host before any device
work (no GPU needed)."""
import ctypes
import math

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


BAD_LAYERS = [(dict(k=None), BAD), (dict(v=FAKE + 8), BAD), (dict(num_slots=15), BAD), (dict(n_kv_heads=0), BAD),
              (dict(block_size=24), NO), (dict(block_size=4), NO), (dict(head_dim=96), NO)]


def _batch(groups=0, **kw):
    a = dict(n_q_heads=32, n_kv_heads=8, head_dim=128, n_req=2, n_groups=groups, n_tokens=3, workspace=FAKE,
             workspace_bytes=1 << 40)
    a.update(kw)
    return cr.cr_attention_batch(**a)


def test_weights_refusals(L):
    def call(layer=None, batch=None, q=FAKE, ldq=4096, lse=FAKE, table=FAKE, blocks=8, lens=FAKE, ptable=None, pblocks=0,
             plen=None, scale=0.1, w=FAKE):
        return L.cr_attention_weights(ctypes.byref(layer or _layer()), ctypes.byref(batch or _batch()), q, ldq, lse, table,
                                      blocks, lens, ptable, pblocks, plen, scale, w, None)

    for kw, want in BAD_LAYERS:
        assert call(_layer(**kw)) == want, kw
    for kw in (dict(q=None), dict(q=FAKE + 2), dict(ldq=4088), dict(ldq=4100), dict(lse=None), dict(lse=FAKE + 4), dict(table=None),
               dict(table=FAKE + 4), dict(blocks=0), dict(lens=None), dict(lens=FAKE + 8), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=math.nan), dict(scale=math.inf), dict(w=None), dict(w=FAKE + 4),
               dict(ptable=FAKE, pblocks=2, plen=FAKE), dict(batch=_batch(1)), dict(batch=_batch(n_kv_heads=4)),
               dict(batch=_batch(head_dim=64)), dict(batch=_batch(n_q_heads=12)), dict(batch=_batch(workspace=None)),
               dict(batch=_batch(1), ptable=FAKE, pblocks=0, plen=FAKE), dict(batch=_batch(1), ptable=FAKE, pblocks=2),
               dict(batch=_batch(1), ptable=FAKE + 4, pblocks=2, plen=FAKE)):
        assert call(**kw) == BAD, kw
    assert call(blocks=2 ** 31) == NO
    assert L.cr_attention_weights(None, ctypes.byref(_batch()), FAKE, 4096, FAKE, FAKE, 8, FAKE, None, 0, None, 0.1, FAKE,
                                  None) == BAD


def test_evict_refusals(L):
    def call(layer=None, table=FAKE, blocks=8, n=2, lens=FAKE, keep=FAKE + 64, most=100, first=0, last=0, w=FAKE, kept=FAKE,
             new=FAKE + 128, ws=FAKE, wsb=1 << 30):
        return L.cr_paged_evict(ctypes.byref(layer or _layer()), table, blocks, n, lens, keep, most, first, last, w, kept, new,
                                ws, wsb, None)

    for kw, want in BAD_LAYERS:
        assert call(_layer(**kw)) == want, kw
    for kw in (dict(table=None), dict(table=FAKE + 4), dict(blocks=0), dict(n=0), dict(n=257), dict(lens=None), dict(keep=None),
               dict(keep=FAKE + 4), dict(most=0), dict(most=-1), dict(first=-1), dict(last=-1), dict(w=None), dict(w=FAKE + 4),
               dict(kept=None), dict(kept=FAKE + 8), dict(new=None), dict(new=FAKE), dict(new=FAKE + 64), dict(ws=None),
               dict(ws=FAKE + 8), dict(wsb=100)):
        assert call(**kw) == BAD, kw
    assert call(blocks=2 ** 31) == NO
    assert call(_layer(n_kv_heads=4096), n=256, most=2 ** 20, wsb=1 << 50) == NO
    assert L.cr_paged_evict(None, FAKE, 8, 2, FAKE, FAKE, 100, 0, 0, FAKE, FAKE, FAKE + 128, FAKE, 1 << 30, None) == BAD


def test_evict_workspace(L):
    assert [cr.cr_evict_workspace_bytes(*a) for a in ((0, 1, 1), (8, 0, 1), (8, 257, 1), (8, 1, 0), (4097, 1, 1))] == [0] * 5
    one = cr.cr_evict_workspace_bytes(8, 16, 4096)
    assert 0 < one < cr.cr_evict_workspace_bytes(8, 32, 4096) and one <= cr.cr_evict_workspace_bytes(8, 16, 5000)


def test_sample_refusals(L):
    def call(x=FAKE, dtype=cr.CR_F32, ld=1000, n=3, v=1000, how=None, u=FAKE, token=FAKE, logp=None, none=False, **kw):
        a = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
        a.update(kw)
        h = cr.cr_sampling(**a)
        return L.cr_sample(x, dtype, ld, n, v, None if none else ctypes.byref(h), u, token, logp, None)

    for kw in (dict(x=None), dict(x=FAKE + 2), dict(dtype=2), dict(x=FAKE + 1, dtype=cr.CR_BF16), dict(ld=999), dict(n=0),
               dict(n=-1), dict(v=0), dict(none=True), dict(u=None), dict(u=FAKE + 4), dict(token=None), dict(token=FAKE + 8),
               dict(logp=FAKE + 4), dict(temperature=-0.5), dict(temperature=math.nan), dict(temperature=math.inf),
               dict(top_p=math.nan), dict(min_p=math.nan), dict(temperature_rows=FAKE + 4), dict(top_k_rows=FAKE + 8),
               dict(top_p_rows=FAKE + 4), dict(min_p_rows=FAKE + 4)):
        assert call(**kw) == BAD, kw
    assert call(v=1048576, ld=1048576) == NO


@pytest.fixture
def elsewhere():
    """A session whose cache counts as the first GPU's, with every tensor on the CPU."""
    build.build()
    cache = torch.zeros(2, 64, 128, dtype=torch.bfloat16)
    s = AnswerSession(cr.target_dims(1, 2, 64, 256, "bf16"), 4, cache, max_tokens=8, max_requests=2)
    return s


def _on(sess, device):
    sess._device_index = device
    return sess


def _weigh_args(groups=0, heads=4):
    b = cr.cr_attention_batch(n_q_heads=heads, n_kv_heads=2, head_dim=64, n_req=2, n_groups=groups, n_tokens=3,
                              workspace=FAKE, workspace_bytes=1 << 30)
    return dict(batch=AnswerBatch(b, None), q=torch.zeros(3, 256, dtype=torch.bfloat16), lse=torch.zeros(3, 4),
                block_table=torch.zeros(2, 4, dtype=torch.int32), kv_len=torch.zeros(2, dtype=torch.int32),
                weights=torch.zeros(2, 64))


def test_session_weigh_refuses(elsewhere):
    a = _weigh_args()
    with pytest.raises(ValueError, match="cuda:0"):
        _on(elsewhere, 0).weigh(0, **a)
    _on(elsewhere, -1)
    for name, x, match in (("q", torch.zeros(2, 256, dtype=torch.bfloat16), "q"), ("lse", torch.zeros(3, 5), "lse"),
                           ("lse", torch.zeros(3, 4, dtype=torch.bfloat16), "lse"), ("weights", torch.zeros(64, 2), "weights"),
                           ("weights", torch.zeros(2, 63), "weights"), ("kv_len", torch.zeros(2), "kv_len"),
                           ("block_table", torch.zeros(8, dtype=torch.int32), "block_table")):
        with pytest.raises(ValueError, match=match):
            elsewhere.weigh(0, **{**a, name: x})
    with pytest.raises(ValueError, match="groups"):
        elsewhere.weigh(0, **a, prefix_table=a["block_table"][:1], prefix_len=a["kv_len"][:1])
    with pytest.raises(ValueError, match="groups"):
        elsewhere.weigh(0, **_weigh_args(1))
    with pytest.raises(ValueError, match="query heads"):
        elsewhere.weigh(0, **_weigh_args(heads=8))
    with pytest.raises(ValueError, match="current CUDA device"):
        elsewhere.weigh(0, **a)


def test_session_evict_refuses(elsewhere):
    a = dict(block_table=torch.zeros(2, 4, dtype=torch.int32), kv_len=torch.zeros(2, dtype=torch.int32),
             keep=torch.zeros(2, dtype=torch.int32), weights=torch.zeros(2, 64), max_keep=5)
    with pytest.raises(ValueError, match="cuda:0"):
        _on(elsewhere, 0).evict(0, **a)
    _on(elsewhere, -1)
    for name, x, match in (("block_table", torch.zeros(2, 4), "block_table"), ("keep", torch.zeros(3, dtype=torch.int32), "keep"),
                           ("kv_len", torch.zeros(2, dtype=torch.int64), "kv_len"), ("weights", torch.zeros(2, 65), "weights"),
                           ("max_keep", 0, "max_keep"), ("block_table", torch.zeros(8, dtype=torch.int32), "block_table")):
        with pytest.raises(ValueError, match=match):
            elsewhere.evict(0, **{**a, name: x})
    with pytest.raises(ValueError, match="current CUDA device"):
        elsewhere.evict(0, **a)


def test_session_sample_refuses(elsewhere):
    x, u = torch.zeros(3, 100), torch.zeros(3)
    with pytest.raises(ValueError, match="cuda:0"):
        _on(elsewhere, 0).sample(x, u)
    _on(elsewhere, -1)
    for args, kw, match in (((x.half(), u), {}, "logits"), ((x[0], u), {}, "logits"), ((x.t(), u), {}, "logits"),
                            ((x, u[:2]), {}, "uniform"), ((x, u.double()), {}, "uniform"),
                            ((x, u), dict(temperature=torch.zeros(2)), "temperature"),
                            ((x, u), dict(top_k=torch.zeros(3, dtype=torch.int64)), "top_k"),
                            ((x, u), dict(top_p=torch.zeros(3, dtype=torch.bfloat16)), "top_p"),
                            ((x, u), dict(min_p=torch.zeros(1)), "min_p")):
        with pytest.raises(ValueError, match=match):
            elsewhere.sample(*args, **kw)
    with pytest.raises(ValueError, match="current CUDA device"):
        elsewhere.sample(x, u)
