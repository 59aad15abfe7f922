"""The answering path as a user runs it (examples/answer.py): repair into a paged cache, a
question pass over the shared prefix, captured answer steps.  Checked against a float64 decoder
over the same weights and the same repaired rows.

Tolerance, derived before any run: each layer rounds to bf16 about six times on the way into the
residual stream (LayerNorm, QKV, rotation, attention, MLP input and hidden), each a relative 2^-9;
over four layers that is sqrt(24) 2^-9 = 1 % of the stream's RMS, and the largest of some 10^6
logits lies about five standard deviations out: 8e-2 of the logits' RMS bounds it."""
import importlib.util
import math
import os

import pytest
import torch

import fixtures as F
from paper_2609_35139_gb300 import cr

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2609_35139_gb300 import build
    build.build()
    cr.cr_clear_device_status()
    spec = importlib.util.spec_from_file_location("example_answer", os.path.join(ROOT, "examples", "answer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    yield m
    st, word = cr.cr_get_device_status()
    assert st == cr.CR_OK, f"device status {word}"


def _plain(run, prefix_rows, ids, inv_freq):
    """Logits of one request's own tokens, in float64, over the prefix rows [2 L, P, W]."""
    m, t = run.model, run.t
    hq, hkv, d = run.n_q_heads, t.n_kv_heads, t.head_dim
    n = len(ids)
    ln = lambda x: (x - x.mean(1, keepdim=True)) / torch.sqrt(x.var(1, unbiased=False, keepdim=True) + 1e-5)
    ang = (run.prefix + torch.arange(n, device="cuda")).double()[:, None] * inv_freq
    c, s = ang.cos()[:, None], ang.sin()[:, None]

    def rot(x):
        a, b = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    x = m.emb[ids].double()
    for i, w in enumerate(m.layers):
        w = {k: v.double() for k, v in w.items()}
        qkv = ln(x) @ w["qkv"].T
        q, k, v = qkv.split([m.qw, m.kvw, m.kvw], 1)
        q, k, v = rot(q.view(n, hq, d)), rot(k.view(n, hkv, d)), v.view(n, hkv, d)
        k = torch.cat([prefix_rows[2 * i].double().view(-1, hkv, d), k]).repeat_interleave(hq // hkv, 1)
        v = torch.cat([prefix_rows[2 * i + 1].double().view(-1, hkv, d), v]).repeat_interleave(hq // hkv, 1)
        sc = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(d)
        late = torch.arange(run.prefix + n, device="cuda")[None] > run.prefix + torch.arange(n, device="cuda")[:, None]
        p = torch.softmax(sc.masked_fill(late[None], -math.inf), 2)
        x = x + torch.einsum("hij,jhd->ihd", p, v).reshape(n, -1) @ w["o"].T
        x = x + torch.nn.functional.gelu(ln(x) @ w["up"].T) @ w["down"].T
    return ln(x) @ m.emb.double().T


def test_questions_and_answers_over_a_repaired_prefix(example):
    case = F.make_case("small")
    steps = 6
    run = example.Answers(case, [5, 1, 18, 33], steps)
    prefix_rows = run.cache[:, :run.prefix].clone()
    inv = torch.from_numpy(case.inv_freq_target).cuda().double()
    logits = run.question_pass()
    tokens = run.answer(logits, steps)
    torch.cuda.synchronize()
    assert torch.equal(run.cache[:, :run.prefix], prefix_rows)          # the shared pages are read only
    at, worst = 0, 0.0
    for r, n in enumerate(run.question_len):
        # the question's tokens and the answer's, forced to what the run chose
        ids = torch.cat([run.ids[at:at + n], tokens[r, :-1]])
        want = _plain(run, prefix_rows, ids, inv)
        rms = float(want.square().mean().sqrt())
        worst = max(worst, float((logits[at:at + n].double() - want[:n]).abs().max()) / rms)
        # each chosen token is the plain decoder's best, or as good up to the tolerance
        for k in range(steps):
            row = want[n - 1 + k]
            assert float(row.max() - row[tokens[r, k]]) <= 2 * 8e-2 * rms, (r, k)
        at += n
    print(f"question logits: worst error {worst:.3e} x RMS")
    assert worst <= 8e-2
