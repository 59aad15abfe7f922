"""Weighing, evicting and sampling as a user runs them together (examples/answer.py): the question pass
gathers the weight of the documents' tokens, the lightest leave every layer's cache, and the answers'
tokens are drawn over what is left, one captured step replayed.

Checked: the gathered weights of a layer add up to the rows that gave them (a row's weights sum to one, but
for what the scores and lse are off by in fp32, some 1e-4 at most; 2^-10 bounds it); the rows that stay are
the ones named; the steps' logits against a float64 decoder that sees, head by head, the tokens that stayed
(tolerance as for the uncut path: 8e-2 of the logits' RMS); the drawn tokens against a float64 draw from
the steps' own logits."""
import math

import pytest
import torch

import fixtures as F
from paper_2609_35139_gb300 import cr
from test_gpu_answer_path import example  # noqa: F401  (the fixture)
from test_gpu_sample import EDGE, plain

pytestmark = pytest.mark.gpu


def decoder(run, full, cut, ids, nq, inv_freq):
    """Logits of one request's tokens in float64: the first nq see the rows `full` [2 L, P, W] before their own
    tokens, the others the rows `cut`."""
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
        q, k, v = (ln(x) @ w["qkv"].T).split([m.qw, m.kvw, m.kvw], 1)
        q, k, v = rot(q.view(n, hq, d)), rot(k.view(n, hkv, d)), v.view(n, hkv, d)
        out = []
        for rows, lo, hi in ((full, 0, nq), (cut, nq, n)):
            p = rows.shape[1]
            kk = torch.cat([rows[2 * i].double().view(p, hkv, d), k]).repeat_interleave(hq // hkv, 1)
            vv = torch.cat([rows[2 * i + 1].double().view(p, hkv, d), v]).repeat_interleave(hq // hkv, 1)
            sc = torch.einsum("ihd,jhd->hij", q[lo:hi], kk) / math.sqrt(d)
            late = torch.arange(p + n, device="cuda")[None] > p + torch.arange(lo, hi, device="cuda")[:, None]
            out.append(torch.einsum("hij,jhd->ihd", torch.softmax(sc.masked_fill(late[None], -math.inf), 2), vv))
        x = x + torch.cat(out).reshape(n, -1) @ w["o"].T
        x = x + torch.nn.functional.gelu(ln(x) @ w["up"].T) @ w["down"].T
    return ln(x) @ m.emb.double().T


@pytest.mark.parametrize("keep", [300, 77])
def test_answers_over_the_tokens_that_the_questions_looked_at(example, keep):  # noqa: F811
    case = F.make_case("small")
    steps, temperature, top_p = 6, 0.7, 0.9
    run = example.Answers(case, [5, 1, 18, 33], steps, keep=keep)
    full = run.cache[:, :run.prefix].clone()
    inv = torch.from_numpy(case.inv_freq_target).cuda().double()
    g = torch.Generator(device="cuda").manual_seed(5)
    uniform = torch.rand(steps, 4, generator=g, device="cuda")
    evict = run.cut_documents
    gathered = {}

    def watched():
        gathered["w"] = run.weights.clone()
        evict()

    run.cut_documents = watched
    logits = run.question_pass()
    w = gathered["w"].double()
    rows = sum(run.question_len) * (run.n_q_heads // run.t.n_kv_heads)
    assert float((w.sum(2) / rows - 1).abs().max()) <= 2.0 ** -10
    assert run.prefix_len.tolist() == [keep]
    hkv, d = run.t.n_kv_heads, run.t.head_dim
    cut = run.cache[:, :keep].clone()
    for i, kept in enumerate(run.kept):
        idx = kept[0].long()                                        # [hkv, keep]
        assert bool((idx[:, 1:] > idx[:, :-1]).all()) and bool((idx[:, :4] == torch.arange(4, device="cuda")).all())
        assert bool((idx[:, -32:] == torch.arange(run.prefix - 32, run.prefix, device="cuda")).all())
        for h in range(hkv):
            for plane in (2 * i, 2 * i + 1):
                assert torch.equal(cut[plane, :, h * d:(h + 1) * d], full[plane, idx[h], h * d:(h + 1) * d])
            left = torch.ones(run.prefix, dtype=torch.bool, device="cuda")
            left[idx[h]] = False
            mid = idx[h, 4:-32]
            assert float(w[i, h, mid].min()) >= float(w[i, h, :run.prefix][left].max())
    each = []
    tokens = run.answer(logits, steps, each, uniform=uniform, temperature=temperature, top_p=top_p)
    torch.cuda.synchronize()
    at, worst = 0, 0.0
    for r, n in enumerate(run.question_len):
        ids = torch.cat([run.ids[at:at + n], tokens[r, :-1]])
        want = decoder(run, full, cut, ids, n, inv)
        rms = float(want.square().mean().sqrt())
        worst = max(worst, float((logits[at:at + n].double() - want[:n]).abs().max()) / rms)
        for k in range(steps):
            own = logits[at + n - 1] if k == 0 else each[k - 1][r]
            worst = max(worst, float((own.double() - want[n - 1 + k]).abs().max()) / rms)
            token, _, near = plain(own, uniform[k, r].item(), torch.tensor(temperature).item(), 0, torch.tensor(top_p).item(), 0.0)
            assert int(tokens[r, k]) == token or near < EDGE, (r, k)
        at += n
    print(f"logits over {keep} tokens: worst error {worst:.3e} x RMS")
    assert worst <= 8e-2
    st, word = cr.cr_get_device_status()
    assert st == cr.CR_OK, word
