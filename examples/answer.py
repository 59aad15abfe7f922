"""Answer several questions over one repaired document set.

A request's chunk caches are repaired and written into a paged cache; a batch of
questions then shares those pages as its prefix.  The questions' tokens go
through a small decoder (random weights, synthetic inputs: there is nothing to
download) in one pass, and the answers' tokens one step at a time, captured in a
CUDA graph.  Per layer: LayerNorm and the QKV linear, AnswerSession.append,
AnswerSession.attend, the output linear, LayerNorm and a two-layer MLP.  With --keep the
question pass also gathers the attention weight of the documents' tokens
(AnswerSession.weigh), and the answers go over the heaviest of them alone
(AnswerSession.evict); with --temperature tokens are drawn (AnswerSession.sample) instead
of the best taken.

    python examples/answer.py [--questions N] [--steps K] [--keep M] [--temperature T] [--top-p P]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import fixtures as F  # noqa: E402
from paper_2609_35139_gb300 import (AnswerSession, RepairSession, cr, dims_from,  # noqa: E402
                                    host_to_device, pack_host_weights)

BLOCK = 16


class Decoder:
    """A pre-LN decoder of the target's shape with random weights: the target model's
    stand-in.  Linears and LayerNorms run in the library's kernels."""

    def __init__(self, target, n_q_heads: int, vocab: int, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        d, dh, hkv = target.d_model, target.head_dim, target.n_kv_heads
        w = lambda o, i: (torch.randn(o, i, generator=g, device="cuda") * i ** -0.5).to(torch.bfloat16)
        self.d, self.qw, self.kvw = d, n_q_heads * dh, hkv * dh
        self.layers = [dict(qkv=w(self.qw + 2 * self.kvw, d), o=w(d, self.qw), up=w(4 * d, d), down=w(d, 4 * d))
                       for _ in range(target.n_layers)]
        # tied to the output: entries small beside what the layers add, or the best token would be
        # the input's whatever the attention gives
        self.emb = w(vocab, d) * (0.1 * d ** 0.5)
        self.one, self.zero = torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")

    def run(self, session: AnswerSession, batch, ids, pos, slots, table, kv_len, weights=None, **prefix) -> torch.Tensor:
        """Logits [n, vocab] fp32 of the tokens `ids`, whose K and V join the paged cache; weights
        [n_layers, H_kv, num_slots] gathers the attention weight that they give the cached tokens."""
        n = ids.shape[0]
        buf = lambda cols, dtype=torch.bfloat16: torch.empty(n, cols, dtype=dtype, device="cuda")
        x, u = self.emb[ids].float(), buf(self.d)
        qkv, q, att, up = buf(self.qw + 2 * self.kvw), buf(self.qw), buf(self.qw), buf(4 * self.d)
        lse = None if weights is None else torch.empty(n, session.n_q_heads, device="cuda")
        for i, w in enumerate(self.layers):
            cr.cr_layernorm(x, self.one, self.zero, 1e-5, u)
            cr.cr_linear(u, w["qkv"], None, qkv)
            qn, k, v = qkv.split([self.qw, self.kvw, self.kvw], dim=1)
            session.append(i, qn, k, v, pos, slots, q)
            session.attend(i, batch, q, table, kv_len, att, lse=lse, **prefix)
            if weights is not None:
                session.weigh(i, batch, q, lse, table, kv_len, weights[i], **prefix)
            cr.cr_linear(att, w["o"], None, x, cr.CR_EPI_ADD_F32)
            cr.cr_layernorm(x, self.one, self.zero, 1e-5, u)
            cr.cr_linear(u, w["up"], None, up, cr.CR_EPI_GELU_BF16)
            cr.cr_linear(up, w["down"], None, x, cr.CR_EPI_ADD_F32)
        cr.cr_layernorm(x, self.one, self.zero, 1e-5, u)
        logits = buf(self.emb.shape[0], torch.float32)
        cr.cr_linear(u, self.emb, None, logits, cr.CR_EPI_F32)
        return logits


def repaired_prefix(case, num_blocks: int):
    """Repair the case's request into the first blocks of a paged cache (through its last
    complete block; the rest is left to the question pass).  (cache, tokens in it)"""
    t, r = dims_from(case.target, case.repairer)
    kv, emb = case.pool()
    p = case.plan
    sess = RepairSession(t, r, pack_host_weights(case.weights, case.repairer.n_blocks), max_tokens=p.n_tokens)
    a = sess.assemble(host_to_device(kv), host_to_device(emb), p.chunk_start, p.chunk_len, p.chunk_idx, p.cu_chunks)
    sess.compress(a)
    sess.forward(a)
    n = a.n_tokens // BLOCK * BLOCK
    slots = torch.arange(a.n_tokens, dtype=torch.int64, device="cuda")
    slots[n:] = -1
    cache = torch.zeros(2 * t.n_layers, num_blocks * BLOCK, t.n_kv_heads * t.head_dim, dtype=torch.bfloat16,
                        device="cuda")
    sess.apply_paged(a, slots, cache, num_blocks * BLOCK, case.inv_freq_target, cr.CR_ROPE_GLOBAL)
    return cache, n


class Answers:
    """A batch of questions over one shared prefix: block tables, lengths and slots.  keep: the
    tokens of the prefix that the answers see (None: all)."""

    def __init__(self, case, question_len, steps: int, seed: int = 0, vocab: int = 4096, keep=None):
        self.question_len = list(question_len)
        n_req = len(self.question_len)
        room = [-(-(n + steps) // BLOCK) for n in self.question_len]
        prefix_blocks = case.plan.n_tokens // BLOCK
        self.cache, self.prefix = repaired_prefix(case, prefix_blocks + sum(room))
        self.t, _ = dims_from(case.target, case.repairer)
        self.n_q_heads = self.t.d_model // self.t.head_dim
        self.model = Decoder(self.t, self.n_q_heads, vocab, seed)
        self.session = AnswerSession(self.t, self.n_q_heads, self.cache, block_size=BLOCK,
                                     max_tokens=sum(self.question_len) + n_req, max_requests=n_req,
                                     inv_freq_target=case.inv_freq_target)
        self.prefix_table = torch.arange(prefix_blocks, dtype=torch.int32, device="cuda")[None].contiguous()
        self.prefix_len = torch.tensor([self.prefix], dtype=torch.int32, device="cuda")
        table = np.zeros((n_req, max(room)), np.int32)
        at = prefix_blocks
        for i, b in enumerate(room):
            table[i, :b] = np.arange(at, at + b)
            at += b
        self.table = torch.from_numpy(table).cuda()
        g = torch.Generator(device="cuda").manual_seed(seed + 1)
        self.ids = torch.randint(0, vocab, (sum(self.question_len),), generator=g, device="cuda")
        self.kv_len = torch.zeros(n_req, dtype=torch.int32, device="cuda")
        self.keep = keep
        self.weights = None if keep is None else torch.zeros(self.t.n_layers, self.t.n_kv_heads, self.cache.shape[1],
                                                             device="cuda")

    def _places(self, req, idx):
        """Position (after the prefix) and slot of each request's idx-th own token."""
        slot = self.table.long()[req, idx // BLOCK] * BLOCK + idx % BLOCK
        return (self.prefix + idx).to(torch.int32), slot

    def question_pass(self) -> torch.Tensor:
        """All questions' tokens in one pass; logits of every token."""
        n = torch.tensor(self.question_len, device="cuda")
        req = torch.repeat_interleave(torch.arange(len(n), device="cuda"), n)
        idx = torch.arange(len(req), device="cuda") - (torch.cumsum(n, 0) - n)[req]
        pos, slots = self._places(req, idx)
        self.kv_len.copy_(n)
        cu = np.concatenate([[0], np.cumsum(self.question_len)])
        batch = self.session.batch(cu, [0, len(self.question_len)])
        logits = self.model.run(self.session, batch, self.ids, pos, slots, self.table, self.kv_len,
                                weights=self.weights, prefix_table=self.prefix_table, prefix_len=self.prefix_len)
        self.last = (torch.cumsum(n, 0) - 1)
        if self.keep is not None:
            self.cut_documents()
        return logits

    def cut_documents(self):
        """Of every layer's and KV head's document tokens the first four, the last 32 and the ones that
        the questions looked at most stay, at the front of the prefix's blocks.  Their K keeps the
        rotation of its position, and the tokens behind keep theirs."""
        keep = torch.tensor([self.keep], dtype=torch.int32, device="cuda")
        self.kept = []
        for i in range(self.t.n_layers):
            kept, new_len = self.session.evict(i, self.prefix_table, self.prefix_len, keep, self.weights[i], self.keep,
                                               first=4, last=32)
            self.kept.append(kept)
        self.prefix_len = new_len

    def answer(self, logits: torch.Tensor, steps: int, step_logits=None, uniform=None, **sampling) -> torch.Tensor:
        """`steps` tokens of every request [n_req, steps], one captured step replayed; a list
        step_logits takes each step's logits.  The best tokens, or, with uniform [steps, n_req], tokens
        drawn with AnswerSession.sample's parameters `sampling`."""
        n_req = len(self.question_len)
        u = None if uniform is None else uniform[0].clone()

        def pick(rows):
            return rows.argmax(1) if u is None else self.session.sample(rows, u, **sampling)

        ids = pick(logits[self.last])
        req = torch.arange(n_req, device="cuda")
        batch = self.session.batch(np.arange(n_req + 1), [0, n_req])
        idx = self.kv_len.long()                     # each request's next own token
        pos, slots = self._places(req, idx)
        slots = slots.contiguous()
        out = [ids.clone()]

        def step():
            new = self.model.run(self.session, batch, ids, pos, slots, self.table, self.kv_len,
                                 prefix_table=self.prefix_table, prefix_len=self.prefix_len)
            return new, pick(new)

        graph = None
        for k in range(1, steps):
            if u is not None:
                u.copy_(uniform[k])
            p, s = self._places(req, idx)
            pos.copy_(p)
            slots.copy_(s)
            self.kv_len.copy_(idx + 1)
            if graph is None:
                side = torch.cuda.Stream()
                side.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(side):
                    step()                           # warm-up: it writes the same rows as the replay
                torch.cuda.current_stream().wait_stream(side)
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    new, best = step()
            graph.replay()
            ids.copy_(best)
            if step_logits is not None:
                step_logits.append(new.clone())
            out.append(ids.clone())
            idx = idx + 1
        return torch.stack(out, 1)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--questions", type=int, default=8)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--keep", type=int, default=None, help="document tokens that the answers see (default: all)")
    ap.add_argument("--temperature", type=float, default=0.0, help="0: the best tokens")
    ap.add_argument("--top-p", type=float, default=0.95)
    a = ap.parse_args()
    from paper_2609_35139_gb300 import build
    build.build()
    run = Answers(F.make_case("small"), [11 + 5 * (i % 4) for i in range(a.questions)], a.steps, keep=a.keep)
    draw = {} if a.temperature == 0 else dict(uniform=torch.rand(a.steps, a.questions, device="cuda"),
                                              temperature=a.temperature, top_p=a.top_p)
    logits = run.question_pass()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    tokens = run.answer(logits, a.steps, **draw)
    torch.cuda.synchronize()
    st, word = cr.cr_get_device_status()
    assert st == cr.CR_OK, f"device status {word}"
    print(f"{a.questions} questions over {int(run.prefix_len[0])} of {run.prefix} shared tokens, {a.steps} answer tokens each, "
          f"{(time.perf_counter() - t0) * 1e3:.1f} ms; first answer: {tokens[0].tolist()}")


if __name__ == "__main__":
    main()
