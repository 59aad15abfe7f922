"""cr_paged_evict (AnswerSession.evict) against a plain restatement: copies and indexes, so equality."""
import numpy as np
import pytest
import torch

from paper_2609_35139_gb300 import AnswerSession, cr

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


class Pages:
    """Requests of the given lengths in shuffled blocks, with weights; max_blocks wider than needed."""

    def __init__(self, lens, hkv=2, d=64, block=16, layers=2, layer=1, kind="spread", seed=0, spare=2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.hkv, self.d, self.block, self.layer = list(lens), hkv, d, block, layer
        need = [-(-n // block) for n in lens]
        blocks = sum(need) + 3
        order = torch.randperm(blocks, generator=g, device="cuda").cpu().numpy()
        self.table = torch.full((len(lens), max(need) + spare), -1, dtype=torch.int32, device="cuda")
        self.slots, at = [], 0
        for r, (n, b) in enumerate(zip(lens, need)):
            mine = order[at:at + b].astype(np.int64)
            at += b
            self.table[r, :b] = torch.from_numpy(mine.astype(np.int32)).cuda()
            self.slots.append(torch.from_numpy((mine[:, None] * block + np.arange(block)).reshape(-1)[:n]).cuda())
        self.cache = torch.randn(2 * layers, blocks * block, hkv * d, generator=g, device="cuda").to(torch.bfloat16)
        w = torch.randn(hkv, blocks * block, generator=g, device="cuda")
        if kind == "spread":
            w = (3 * w).exp()
        elif kind == "ties":
            w = torch.floor(2 * w) + 0.0          # a few values, negative ones and both zeros among them
            w[w == 0] *= -1.0
        elif kind == "equal":
            w = torch.full_like(w, 0.25)
        elif kind == "odd":
            x = torch.rand(w.shape, generator=g, device="cuda")
            w = torch.where(x < 0.1, float("nan"), torch.where(x < 0.2, float("inf"), torch.where(x < 0.3, -float("inf"), w)))
        self.weights = w
        self.len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.session = AnswerSession(cr.target_dims(layers, hkv, d, 4 * hkv * d, "bf16"), 4 * hkv, self.cache, block_size=block,
                                     max_tokens=1)

    def plain(self, keep, max_keep, first, last):
        """(cache, weights, kept, new_len) by sorting."""
        cache, weights = self.cache.clone(), self.weights.clone()
        kept = torch.full((len(self.lens), self.hkv, max_keep), -9, dtype=torch.int32, device="cuda")
        new = []
        for r, n in enumerate(self.lens):
            b = max(0, min(keep[r], max_keep))
            new.append(min(n, b))
            if n <= b:
                kept[r, :, :n] = torch.arange(n, dtype=torch.int32, device="cuda")
                continue
            la = min(last, b)
            fi = min(first, b - la)
            s = self.slots[r]
            for h in range(self.hkv):
                w = self.weights[h, s[fi:n - la]].double().cpu().numpy()
                rank = np.lexsort((np.arange(len(w)), np.where(np.isnan(w), -np.inf, -w), ~np.isnan(w)))
                idx = np.sort(np.concatenate([np.arange(fi), fi + rank[:b - fi - la], np.arange(n - la, n)]))
                i = torch.from_numpy(idx).cuda()
                kept[r, h, :b] = i.to(torch.int32)
                c = slice(h * self.d, (h + 1) * self.d)
                for plane in (2 * self.layer, 2 * self.layer + 1):
                    cache[plane, s[:b], c] = self.cache[plane, s[i], c]
                weights[h, s[:b]] = self.weights[h, s[i]]
        return cache, weights, kept, torch.tensor(new, dtype=torch.int32, device="cuda")

    def run(self, keep, max_keep=None, first=0, last=0, **kw):
        keep = [keep] * len(self.lens) if isinstance(keep, int) else keep
        max_keep = max(1, max(keep)) if max_keep is None else max_keep
        k = torch.tensor(keep, dtype=torch.int32, device="cuda")
        kept = torch.full((len(self.lens), self.hkv, max_keep), -9, dtype=torch.int32, device="cuda")
        _, new = self.session.evict(self.layer, self.table, self.len, k, self.weights, max_keep, first=first, last=last,
                                    kept=kept, **kw)
        return kept, new

    def check(self, keep, max_keep=None, first=0, last=0):
        ks = [keep] * len(self.lens) if isinstance(keep, int) else keep
        want = self.plain(ks, max(1, max(ks)) if max_keep is None else max_keep, first, last)
        kept, new = self.run(keep, max_keep, first, last)
        torch.cuda.synchronize()
        assert torch.equal(kept, want[2]) and torch.equal(new, want[3])
        assert torch.equal(self.cache.view(torch.int16), want[0].view(torch.int16))
        assert torch.equal(self.weights.view(torch.int32), want[1].view(torch.int32))


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "odd"])
@pytest.mark.parametrize("lens,keep", [([1], 1), ([2], 1), ([63, 64, 65], 40), ([200, 17, 0, 1], 64), ([611], 301),
                                       ([5000, 4097], 1000), ([10240], 10239), ([3000], 1)])
def test_the_heaviest_stay(kind, lens, keep):
    Pages(lens, kind=kind, seed=len(lens) + keep).check(keep, first=2, last=9)


@pytest.mark.parametrize("hkv,d", [(8, 128), (4, 128), (2, 64), (1, 64), (3, 128)])
@pytest.mark.parametrize("block", [8, 64, 512])
def test_heads_and_blocks(hkv, d, block):
    Pages([700, 64, 1500], hkv, d, block, seed=block).check([333, 70, 1200])


@pytest.mark.parametrize("first,last", [(0, 0), (4, 0), (0, 64), (50, 50), (99, 99), (200, 30), (30, 200), (100, 0), (0, 100)])
def test_first_and_last(first, last):
    """More first and last ones than the budget: the last come first, then the first."""
    Pages([400, 100, 101], kind="ties", seed=first).check(100, first=first, last=last)


def test_budgets_by_request():
    """Whole, one less, nothing, more than the list has room for, negative (recorded)."""
    Pages([300, 300, 300, 300], seed=3).check([300, 299, 0, 300], max_keep=300)
    Pages([300, 200], seed=4).check([1000, 1000], max_keep=250)
    p = Pages([300, 20], seed=5)
    want = p.plain([-3, 20], 20, 0, 0)
    kept, new = p.run([-3, 20], 20)
    st, word = cr.cr_get_device_status()
    cr.cr_clear_device_status()
    assert st == cr.CR_ERR_DEVICE_INDEX, word
    assert new.tolist() == [0, 20] and torch.equal(kept, want[2]) and torch.equal(p.cache, want[0])


@pytest.mark.parametrize("n,keep", [(70001, 30000), (131072, 131000)])
def test_long(n, keep):
    Pages([n, 500], hkv=2, d=64, block=64, kind="ties", seed=n).check(keep, first=4, last=256)


def test_more_requests_than_sms():
    Pages([40 + 3 * i for i in range(120)], hkv=2, seed=8).check(100, last=16)


def test_a_wide_table_of_short_requests():
    """Room for a million tokens a request in the table, a few hundred there."""
    Pages([300, 1000], block=16, spare=65536, seed=9).check(200, first=1)


def test_twice_in_a_row():
    """What was kept is cut again."""
    p = Pages([900, 350], seed=10)
    p.check(400)
    p.lens = [400, 350]
    p.len = torch.tensor(p.lens, dtype=torch.int32, device="cuda")
    p.slots = [s[:n] for s, n in zip(p.slots, p.lens)]
    p.check(123, first=1, last=3)


def test_captured_and_replayed():
    """The same graph over changing lengths, budgets and weights."""
    p = Pages([500, 800], hkv=8, d=128, seed=11)
    keep = torch.tensor([10, 20], dtype=torch.int32, device="cuda")
    kept = torch.full((2, 8, 400), -9, dtype=torch.int32, device="cuda")
    new = torch.empty(2, dtype=torch.int32, device="cuda")
    warm = p.cache.clone(), p.weights.clone()
    p.session.evict(1, p.table, p.len, keep, p.weights, 400, kept=kept, new_len=new)
    p.cache.copy_(warm[0])
    p.weights.copy_(warm[1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        p.session.evict(1, p.table, p.len, keep, p.weights, 400, last=7, kept=kept, new_len=new)
    full = p.slots
    for lens, budget in (([500, 800], [400, 300]), ([399, 555], [100, 400]), ([100, 0], [60, 5])):
        p.lens, p.slots = lens, [s[:n] for s, n in zip(full, lens)]
        p.len.copy_(torch.tensor(lens, dtype=torch.int32))
        keep.copy_(torch.tensor(budget, dtype=torch.int32))
        kept.fill_(-9)
        want = p.plain(budget, 400, 0, 7)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(kept, want[2]) and torch.equal(new, want[3])
        assert torch.equal(p.cache, want[0]) and torch.equal(p.weights, want[1])


def test_streams_and_two_calls_at_once():
    ps = [Pages([5000, 3000], hkv=8, d=128, seed=s) for s in (1, 2)]
    wants = [p.plain([2000, 2500], 2500, 4, 64) for p in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    got = []
    for p, s in zip(ps, streams):
        s.wait_stream(torch.cuda.current_stream())
        keep = torch.tensor([2000, 2500], dtype=torch.int32, device="cuda")
        s.wait_stream(torch.cuda.current_stream())
        got.append(p.session.evict(1, p.table, p.len, keep, p.weights, 2500, first=4, last=64, stream=s) + (keep,))
    torch.cuda.synchronize()
    for p, want, (kept, new, _) in zip(ps, wants, got):
        assert torch.equal(new, want[3]) and torch.equal(p.cache, want[0]) and torch.equal(p.weights, want[1])
        for r, n in enumerate(new.tolist()):
            assert torch.equal(kept[r, :, :n], want[2][r, :, :n])


def test_bad_blocks_and_lengths_are_reported():
    p = Pages([100, 60], seed=12)
    before = p.cache.clone()
    p.table[0, 2], p.table[1, 0] = 10 ** 6, -2
    kept, new = p.run(50)
    torch.cuda.synchronize()
    st, word = cr.cr_get_device_status()
    cr.cr_clear_device_status()
    assert st == cr.CR_ERR_DEVICE_INDEX, word
    assert new.tolist() == [50, 50]
    # tokens of the bad blocks are the lightest
    assert not bool(((kept[0] >= 32) & (kept[0] < 48)).any())
    assert bool(((kept[1] < 16).sum(1) == 50 - 44).all())
    # what no request owns is as it was
    owned = torch.zeros(p.cache.shape[1], dtype=torch.bool, device="cuda")
    for s in p.slots:
        owned[s] = True
    assert torch.equal(p.cache[:, ~owned], before[:, ~owned])
    for bad in ([-1, 60], [100, 10 ** 8]):
        p = Pages([100, 60], seed=13)
        p.len = torch.tensor(bad, dtype=torch.int32, device="cuda")
        p.run(50)
        st, word = cr.cr_get_device_status()
        cr.cr_clear_device_status()
        assert st == cr.CR_ERR_DEVICE_INDEX, word
