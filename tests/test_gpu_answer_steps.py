"""The answer steps of examples/answer.py by their logits: every captured and replayed step against a
float64 decoder over the same weights and repaired rows, and the same decoder with a mistake
planted, which the tolerance has to tell from it.

Tolerance: 8e-2 of the logits' RMS, derived in test_gpu_answer_path.py."""
import pytest
import torch

import fixtures as F
from test_gpu_answer_path import _plain, example  # noqa: F401

pytestmark = pytest.mark.gpu

TOLERANCE = 8e-2


def test_logits_of_every_answer_step(example):  # noqa: F811
    case = F.make_case("small")
    steps = 7
    run = example.Answers(case, [5, 1, 18, 33], steps)
    rows = run.cache[:, :run.prefix].clone()
    inv = torch.from_numpy(case.inv_freq_target).cuda().double()
    got = []
    tokens = run.answer(run.question_pass(), steps, got)
    torch.cuda.synchronize()
    assert len(got) == steps - 1
    no_values = rows.clone()
    no_values[1::2] = 0.0                                  # the prefix has keys, but gives nothing
    next_layer = rows.roll(-2, 0)                          # each layer reads the next one's planes
    at = 0
    for r, n in enumerate(run.question_len):
        ids = torch.cat([run.ids[at:at + n], tokens[r, :-1]])
        at += n
        want = _plain(run, rows, ids, inv)
        rms = float(want.square().mean().sqrt())
        mine = torch.stack([x[r] for x in got]).double()   # the step of token n + k gives logits n + k
        off = lambda other: float((mine - other[n:]).abs().max()) / rms  # noqa: E731
        assert off(want) <= TOLERANCE, (r, off(want))
        for planted in (no_values, next_layer):
            assert off(_plain(run, planted, ids, inv)) > 2 * TOLERANCE, r
        print(f"request {r}: steps off by {off(want):.2e} x RMS, "
              f"{off(_plain(run, next_layer, ids, inv)):.2f} with the next layer's rows")
