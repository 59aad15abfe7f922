"""cr_sample (AnswerSession.sample) against a plain float64 restatement.

The kernel's weights are good to 2^-28 of themselves, so the sums that a border is compared with are off by
less than 2^-26 of the whole: a token is right if u shifted by that much either way selects it, among the
tokens kept when the top-p cut is shifted as much.  Away from borders that is one token."""
import math

import pytest
import torch

from paper_2609_35139_gb300 import AnswerSession, cr

pytestmark = pytest.mark.gpu
EDGE = 2.0 ** -26


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


@pytest.fixture(scope="module")
def sess():
    cache = torch.zeros(2, 16, 128, dtype=torch.bfloat16, device="cuda")
    return AnswerSession(cr.target_dims(1, 2, 64, 256, "bf16"), 4, cache, max_tokens=1)


def plain(x, u, t, k, p, m):
    """(token, logp, distance of u and of the top-p cut to the nearest border) of one row in float64."""
    x = x.double()
    if bool(torch.isnan(x).any()) or float(x.max()) == math.inf or float(x.max()) == -math.inf or not (0 <= t < math.inf):
        return -1, math.nan, 1.0
    if t == 0:
        return int(torch.nonzero(x == x.max())[0]), 0.0, 1.0
    order = torch.sort(x, descending=True, stable=True).indices
    w = torch.exp((x[order] - x.max()) / t)
    if k > 0:
        w[k:] = 0.0
    near = 1.0
    if p < 1:
        before = torch.cumsum(w, 0) - w
        share = before / w.sum()
        if len(w) > 1:
            near = min(near, float((share[1:] - p).abs().min()) if p > 0 else 1.0)
        keep = share < p
        keep[0] = True
        w = torch.where(keep, w, 0.0)
    if m > 0:
        w = torch.where(w >= min(m, 1.0), w, 0.0)
    y = torch.zeros_like(w).scatter_(0, order, w)
    cum = torch.cumsum(y, 0) / y.sum()
    u = min(max(u, 0.0), 1.0) if u == u else 0.0
    token = int((cum > u).to(torch.int8).argmax()) if u < 1 else int(torch.nonzero(y > 0)[-1])
    inner = cum[y > 0]
    near = min(near, float((inner[:-1] - u).abs().min()) if len(inner) > 1 else 1.0)
    return token, float(torch.log(y[token] / y.sum())), near


def check(sess, x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    n = x.shape[0]
    logp = torch.full((n,), 7.0, device="cuda")
    token = sess.sample(x, u, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, logp=logp)
    row = lambda v, r: (v[r].item() if torch.is_tensor(v) else torch.tensor(v).item())
    for r in range(n):
        par = [row(v, r) for v in (temperature, top_k, top_p, min_p)]
        want, lp, near = plain(x[r], u[r].item(), *par)
        if near < EDGE and int(token[r]) != want:
            t, k, p, m = par
            other = {y[0]: y for y in (plain(x[r], u[r].item() + a, t, k, p + b if 0 < p < 1 else p, m)
                                       for a in (-EDGE, 0, EDGE) for b in (-EDGE, 0, EDGE))}
            assert int(token[r]) in other, (r, int(token[r]), sorted(other))
            want, lp, _ = other[int(token[r])]
        assert int(token[r]) == want, (r, int(token[r]), want)
        if want < 0:
            assert math.isnan(float(logp[r]))
        else:
            # z and its log-sum in fp32: 2^-22 of their size each
            assert abs(float(logp[r]) - lp) <= 2.0 ** -22 * (4 + 2 * abs(lp) + math.log(x.shape[1] + 1)), (float(logp[r]), lp)
    return token


def logits(n, v, dtype=torch.float32, seed=0, std=2.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(n, v, generator=g, device="cuda") * std).to(dtype), torch.rand(n, generator=g, device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", [1, 2, 5, 127, 128, 129, 1000, 4096, 32003])
@pytest.mark.parametrize("kw", [dict(), dict(top_k=7), dict(top_p=0.8), dict(min_p=0.1), dict(top_k=50, top_p=0.9, min_p=0.02),
                                dict(temperature=0.0), dict(temperature=0.3, top_p=0.5), dict(temperature=3.0, top_k=900)])
def test_sizes_and_filters(sess, dtype, v, kw):
    x, u = logits(9, v, dtype, seed=v)
    check(sess, x, u, **kw)


@pytest.mark.parametrize("v", [100003, 131072, 262144, 1048575])
@pytest.mark.parametrize("n", [1, 40])
def test_large_vocabularies(sess, v, n):
    x, u = logits(n, v, seed=n)
    check(sess, x, u, top_p=0.95)
    check(sess, x, u, temperature=0.7, top_k=1000)
    check(sess, x.to(torch.bfloat16), u)


def test_more_rows_than_sms(sess):
    x, u = logits(400, 5000, seed=1)
    check(sess, x, u, top_k=40, top_p=0.9)


@pytest.mark.parametrize("kw", [dict(top_k=5), dict(top_p=0.5), dict(top_k=6, top_p=0.5), dict(min_p=1.0), dict()])
@pytest.mark.parametrize("value", [0.0, -3.5, 1e30])
def test_all_logits_equal(sess, kw, value):
    """Ties rank by index: a cut among equals keeps the first of them, borders exact."""
    for v in (4, 64, 1000):
        x = torch.full((33, v), value, device="cuda")
        u = (torch.arange(33, device="cuda") + 0.37) / 33.0
        check(sess, x, u, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kw", [dict(top_k=30), dict(top_p=0.6), dict(top_k=100, top_p=0.7, min_p=0.2)])
def test_few_values(sess, dtype, kw):
    """Many ties, cuts inside them."""
    x, u = logits(40, 3001, seed=5)
    check(sess, torch.round(x).to(dtype), u, **kw)


@pytest.mark.parametrize("step", [2.0 ** -4, 2.0 ** -7, 2.0 ** -12])
@pytest.mark.parametrize("kw", [dict(top_k=300), dict(top_k=300, top_p=0.9), dict(top_p=0.5), dict(top_p=0.97, min_p=0.01)])
def test_equal_values_at_a_cut_among_many(sess, kw, step):
    """Lists of candidates too long to be compared each with each, with up to some dozen equal ones at the cut."""
    x, u = logits(12, 20011, seed=51)
    check(sess, torch.floor(x / step) * step, u, **kw)


def test_masked_tokens_are_never_drawn(sess):
    x, u = logits(60, 1500, seed=6)
    x[:, 3:] = torch.where(torch.rand(60, 1497, device="cuda") < 0.97, -math.inf, x[:, 3:])
    for kw in (dict(), dict(top_k=200), dict(top_k=1499), dict(top_p=0.9), dict(temperature=5.0, min_p=0.01)):
        token = check(sess, x, u, **kw)
        assert bool(torch.isfinite(x.gather(1, token[:, None])).all())
    one = torch.full((3, 700), -math.inf, device="cuda")
    one[:, 321] = -5.0
    assert sess.sample(one, u[:3], top_k=4, top_p=0.3).tolist() == [321] * 3


def test_rows_without_an_answer(sess):
    x, u = logits(6, 300, seed=7)
    x[0] = -math.inf
    x[1, 17] = math.nan
    x[2, 299] = math.inf
    x[3, 0] = -math.nan
    t = torch.tensor([1.0, 1.0, 1.0, 1.0, -1.0, math.nan], device="cuda")
    assert check(sess, x, u, temperature=t).tolist() == [-1] * 6
    x, u = logits(2, 300, seed=8)
    t = torch.tensor([math.inf, 0.0], device="cuda")
    assert check(sess, x, u, temperature=t)[0] == -1
    x[1, 5] = math.nan
    assert sess.sample(x, u, temperature=0.0)[1] == -1


def test_far_apart_and_extreme_values(sess):
    u = torch.tensor([0.0, 0.5, 0.99999994, 0.3], device="cuda")
    x = torch.tensor([[3e38, -3e38, 3e38, 0.0]] * 4, device="cuda")
    check(sess, x, u)
    check(sess, x, u, top_k=3, top_p=0.6)
    x = torch.tensor([[1e-40, 2e-40, -1e-40, 0.0, -0.0]] * 4, device="cuda")
    check(sess, x, u, top_k=2)
    check(sess, x, u, temperature=1e-38, top_k=4)
    x, u = logits(20, 999, seed=9)
    for t in (1e-30, 1e-6, 1e6, 1e38):
        check(sess, x, u, temperature=t)
        check(sess, x, u, temperature=t, top_k=10, top_p=0.5)


def test_ends_of_u(sess):
    x, _ = logits(6, 777, seed=10)
    u = torch.tensor([0.0, 0.99999994, 1.0, -2.0, math.nan, 3.0], device="cuda")
    token = sess.sample(x, u, top_k=30)
    kept = torch.sort(torch.topk(x, 30).indices, 1).values
    assert token.tolist() == [int(kept[r, 0 if r in (0, 3, 4) else 29]) for r in range(6)]


def test_parameters_row_by_row(sess):
    x, u = logits(50, 2000, seed=11)
    g = torch.Generator().manual_seed(0)
    pick = lambda v, dtype: torch.tensor(v, dtype=dtype)[torch.randint(0, len(v), (50,), generator=g)].cuda()
    t, k = pick([0.0, 0.5, 1.0, 1.7], torch.float32), pick([0, -1, 1, 20, 2000, 5000], torch.int32)
    p, m = pick([0.0, 0.3, 0.95, 1.0, 2.0], torch.float32), pick([0.0, 0.05, 0.5, 1.0, 1.5], torch.float32)
    check(sess, x, u, t, k, p, m)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_alignment(sess, dtype):
    """Rows of any stride and base: loads of one value where four do not line up."""
    x, u = logits(5, 1203, dtype, seed=12)
    want = sess.sample(x.clone(), u, top_p=0.9)
    for pad, off in ((0, 1), (1, 0), (5, 3), (61, 8)):
        wide = torch.zeros(5, 1203 + pad + off, dtype=dtype, device="cuda")
        wide[:, off:off + 1203] = x
        assert torch.equal(sess.sample(wide[:, off:off + 1203], u, top_p=0.9), want)


def test_captured_on_another_stream_and_without_buffers(sess):
    x, u = logits(8, 9000, seed=13)
    want = sess.sample(x, u, top_k=20, top_p=0.9)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = sess.sample(x, u, top_k=20, top_p=0.9, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
    x2, u2 = logits(8, 9000, seed=14)
    k = torch.full((8,), 20, dtype=torch.int32, device="cuda")
    out = torch.empty(8, dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sess.sample(x, u, top_k=k, top_p=0.9, out=out)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    x.copy_(x2)
    u.copy_(u2)
    k.fill_(1)
    g.replay()
    assert torch.equal(out, x2.argmax(1))


def test_shares_follow_the_weights(sess):
    """Over evenly spaced u the tokens come as often as their weights say (a step of u each way)."""
    x, _ = logits(1, 50, seed=15)
    n = 4096
    u = (torch.arange(n, device="cuda") + 0.5) / n
    token = sess.sample(x.expand(n, 50).contiguous(), u, temperature=1.3, top_k=12)
    w = torch.softmax(torch.where(x[0] >= torch.topk(x[0], 12).values[-1], x[0].double() / 1.3, -math.inf), 0)
    assert float((torch.bincount(token, minlength=50).double() / n - w).abs().max()) <= 1.01 / n


@pytest.mark.parametrize("v", [5000, 1048575])
@pytest.mark.parametrize("kw", [dict(top_p=0.999), dict(top_p=0.5), dict(top_k=4000, top_p=0.9), dict(top_p=0.99, temperature=40.0)])
def test_flat_rows(sess, v, kw):
    """Weights near one another: cuts far down, among too many values to gather; sums near 2^64."""
    g = torch.Generator(device="cuda").manual_seed(v)
    x = torch.rand(3, v, generator=g, device="cuda")
    x[1] = torch.round(x[1] * 8) / 8
    x[2] = 1.0
    check(sess, x, torch.tensor([0.2, 0.7, 0.95], device="cuda"), **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_value_far_above_the_others(sess, dtype):
    """A peak and a flat rest: half of the sum in one value, the cut deep in the rest."""
    x, u = logits(12, 30000, dtype, seed=21, std=0.5)
    x[:, 77] = 10.3
    for kw in (dict(top_p=0.6), dict(top_p=0.95), dict(top_k=3000, top_p=0.8), dict(min_p=1e-6)):
        check(sess, x, u, **kw)


def test_equal_calls_give_equal_tokens(sess):
    x, u = logits(64, 70001, seed=22)
    first = sess.sample(x, u, top_p=0.9)
    for _ in range(5):
        assert torch.equal(sess.sample(x, u, top_p=0.9), first)


@pytest.mark.parametrize("temperature", [0.05, 0.3, 30.0])
@pytest.mark.parametrize("v", [34872, 131072, 49153])
@pytest.mark.parametrize("kw", [dict(top_k=45), dict(top_k=45, top_p=0.9), dict(top_k=700, min_p=0.001), dict(top_p=0.95)])
def test_cold_and_hot_rows(sess, temperature, v, kw):
    """Far from the largest in steps of the weight, or all of them near it; and CTAs without a value."""
    x, u = logits(3, v, seed=61)
    check(sess, x, u, temperature=temperature, **kw)
