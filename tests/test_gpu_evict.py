"""Choice and move of the positions that stay (optr_evict_select, optr_kv_compact)
against plain statements; both move and compare only, so every output is compared
exactly."""
import math
import random

import pytest
import torch

from paper_2608_02691_gb300 import optr, synth
from test_gpu_chunk import PAPER, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


def params(h_kv=2, **opts):
    R_k, R_v = synth.rotations(h_kv, 0)
    return optr.optr_params_create(R_k, R_v, torch.zeros(h_kv, 128), 4 * h_kv, **opts)


# ------------------------------------------------------------------ choice

def plain_select(score, lens, keep, first, last, n_most):
    B, h, _ = score.shape
    kept, counts = torch.full((B, h, n_most), 77, dtype=torch.int32), []
    s = score.cpu()
    for b, n in enumerate(lens):
        m = min(n, max(keep[b], 0, min(n, first + last)))
        counts.append(m)
        for j in range(h):
            ends = set(range(min(n, first))) | set(range(max(0, n - last), n))
            x = s[b, j, :n].tolist()
            val = lambda i: math.inf if math.isnan(x[i]) else x[i]
            nan = lambda i: not math.isnan(x[i])
            rest = sorted((i for i in range(n) if i not in ends), key=lambda i: (nan(i), -val(i), i))
            kept[b, j, :m] = torch.tensor(sorted(list(ends) + rest[:m - len(ends)]), dtype=torch.int32)
    return kept.tolist(), counts


def select(p, score, lens, keep, first, last, n_most):
    B, h, _ = score.shape
    kept = torch.full((B, h, n_most), 77, dtype=torch.int32, device="cuda")
    n_kept = torch.full((B,), 77, dtype=torch.int32, device="cuda")
    optr.optr_evict_select(p, score, i32(lens), i32(keep), first, last, kept, n_kept)
    return kept.tolist(), n_kept.tolist()


KINDS = {
    "plain": lambda x: x.abs(),
    "signed": lambda x: x,
    "many zeros": lambda x: torch.where(x < 0.5, 0.0, x),
    "few values": lambda x: (x * 2).round(),
    "all equal": lambda x: torch.zeros_like(x),
    "both zeros": lambda x: torch.where(x < 0, -0.0, 0.0),
    "near": lambda x: 1 + (x * 4).round() * 2.0 ** -23,
    "infinities and NaN": lambda x: torch.where(x > 1, math.inf, torch.where(x < -1, math.nan, torch.where(x.abs() < 0.3, -math.inf, x))),
    "subnormal": lambda x: x * 1e-41,
}


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,k", [(1, 1), (40, 7), (2049, 1024), (9001, 100), (40000, 30000)])
def test_choice(kind, n, k):
    p = params()
    g = torch.Generator(device="cuda").manual_seed(n)
    lens = [n, max(1, n // 3)]
    score = KINDS[kind](torch.randn(2, 2, n, device="cuda", generator=g))
    for first, last in ((0, 0), (4, 30)):
        m = min(n, max(k, first + last))
        assert select(p, score, lens, [k, k], first, last, m) == plain_select(score, lens, [k, k], first, last, m)
    assert optr.optr_device_error(p) == 0


@pytest.mark.parametrize("lens,keep,first,last", [
    ([0, 1, 5], [3, 3, 3], 0, 0), ([0, 1, 5], [0, 0, 0], 0, 0), ([100, 100, 100], [0, -5, 99], 0, 0),
    ([100, 100, 100], [100, 101, 1000], 4, 4), ([100, 60, 10], [1, 1, 1], 64, 0), ([100, 60, 10], [1, 1, 1], 0, 64),
    ([100, 60, 10], [5, 50, 9], 30, 40), ([100, 60, 10], [50, 50, 50], 1 << 30, 1 << 30),
])
def test_lengths_and_ends(lens, keep, first, last):
    p = params(3)
    g = torch.Generator(device="cuda").manual_seed(1)
    score = torch.randn(3, 3, 101, device="cuda", generator=g)
    assert select(p, score, lens, keep, first, last, 100) == plain_select(score, lens, keep, first, last, 100)
    assert optr.optr_device_error(p) == 0


@pytest.mark.parametrize("n,h", [(131072, 1), (400001, 1), (131071, 8)])
def test_long_rows(n, h):
    """Past what eight CTAs hold in shared memory too."""
    p = params(h)
    g = torch.Generator(device="cuda").manual_seed(2)
    score = torch.randn(1, h, n, device="cuda", generator=g).abs()
    score[score < 0.2] = 0
    kept, counts = select(p, score, [n], [n // 3], 64, 256, n // 3)
    key = score[0].double()
    key[:, :64] = key[:, n - 256:] = 1e9
    want = key.sort(dim=1, descending=True, stable=True).indices[:, :n // 3].sort(1).values
    assert counts == [n // 3] and torch.equal(torch.tensor(kept[0]), want.int().cpu())
    # and where the threshold is a zero
    kept, counts = select(p, score, [n], [n - n // 20], 0, 0, n)
    want = score[0].sort(dim=1, descending=True, stable=True).indices[:, :n - n // 20].sort(1).values
    assert torch.equal(torch.tensor(kept[0])[:, :n - n // 20], want.int().cpu())


def test_many_rows():
    p = params(8)
    g = torch.Generator(device="cuda").manual_seed(3)
    r = random.Random(3)
    lens = [r.randint(0, 700) for _ in range(64)]
    keep = [r.randint(0, 400) for _ in range(64)]
    score = torch.randn(64, 8, 700, device="cuda", generator=g).abs()
    assert select(p, score, lens, keep, 4, 16, 400) == plain_select(score, lens, keep, 4, 16, 400)


def test_choice_out_of_range_is_flagged():
    p = params()
    score = torch.rand(3, 2, 50, device="cuda")
    kept, counts = select(p, score, [51, 20, -1], [10, 10, 10], 0, 0, 10)
    assert counts == [-1, 10, -1] and kept[0] == [[77] * 10] * 2 == kept[2]
    assert kept[1] == plain_select(score, [0, 20, 0], [10] * 3, 0, 0, 10)[0][1]
    assert optr.optr_device_error(p) == optr.OPTR_DEVERR_SEQ_LEN
    kept, counts = select(p, score, [50, 50, 50], [11, 10, 10], 0, 0, 10)   # more than the list holds
    assert counts == [-1, 10, 10] and kept[0] == [[77] * 10] * 2
    assert optr.optr_device_error(p) == optr.OPTR_DEVERR_SEQ_LEN


def test_choice_refusals():
    p = params()
    score = torch.rand(1, 2, 50, device="cuda")
    for bad in (dict(score=score.double()), dict(score=score[:, :1]), dict(score=score.transpose(1, 2)),
                dict(first=-1), dict(last=-1), dict(keep=i32([1, 2]))):
        a = dict(score=score, keep=i32([5]), first=0, last=0)
        a.update(bad)
        with pytest.raises((ValueError, optr.OptrError)):
            optr.optr_evict_select(p, a["score"], i32([50]), a["keep"], a["first"], a["last"],
                                   torch.zeros(1, 2, 9, dtype=torch.int32, device="cuda"), i32([0]))


# -------------------------------------------------------------------- move

class Cache:
    """Random records and windows; `lens` tokens of each sequence."""

    def __init__(self, lens, h_kv=2, seed=0, spare=2, **opts):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.p = params(h_kv, **opts)
        self.lens, self.h, self.B = lens, h_kv, len(lens)
        self.sink, self.recent = opts.get("sink", 0), opts.get("recent", 0)
        self.meta = 4 if opts.get("group", 32) == 128 else 16
        pages = max(1, max(-(-n // 16) for n in lens)) + spare
        num = self.B * pages + 3
        rec = 1152 if self.meta == 4 else 1536
        self.pool = torch.randint(0, 256, (num, h_kv, rec), device="cuda", generator=g, dtype=torch.uint8)
        self.bt = torch.randperm(num, generator=g, device="cuda")[:self.B * pages].view(self.B, pages).int()
        self.n_score = 16 * pages + 5
        self.score = torch.rand(self.B, h_kv, self.n_score, device="cuda", generator=g)
        self.win = self.slots = None
        if self.sink + self.recent:
            shape = (self.B + 2, h_kv, 2, self.sink + self.recent, 128)
            self.win = torch.randint(-32768, 32768, shape, device="cuda", generator=g, dtype=torch.int32).short() \
                .view(torch.bfloat16)
            self.slots = torch.randperm(self.B + 2, generator=g, device="cuda")[:self.B].int()
        self.g = g

    def lists(self, counts):
        """A random rising list of counts[b] positions for each head, the windows' among them."""
        kept = torch.full((self.B, self.h, max(1, max(counts))), 99999999, dtype=torch.int32, device="cuda")
        for b, (n, m) in enumerate(zip(self.lens, counts)):
            x = torch.rand(self.h, max(n, 1), device="cuda", generator=self.g)
            x[:, :self.sink] = 2
            if self.recent:
                x[:, max(0, n - self.recent):n] = 2
            kept[b, :, :m] = x[:, :n].topk(m, 1).indices.sort(1).values.int()
        return kept

    def run(self, kept, counts, score=True, **over):
        a = dict(lens=i32(self.lens), bt=self.bt, slots=self.slots)
        a.update(over)
        args = (self.p, kept, i32(counts), a["lens"], a["bt"], self.pool)
        s = self.score if score else None
        if self.win is None:
            optr.optr_kv_compact(*args, s)
        else:
            optr.optr_kv_compact_win(*args, self.win, a["slots"], s)

    def plain(self, kept, counts, skip=()):
        """Pool, score and windows after the move, record by record; (b, h, i) in skip stay, and whole
        (b, h)."""
        pool, score = self.pool.clone(), self.score.clone()
        win = None if self.win is None else self.win.view(torch.int16).clone()
        page, slot = lambda b, i: self.bt[b].long()[i // 16], lambda i: i % 16
        at = torch.cat([base + size * torch.arange(16)[:, None] + torch.arange(size) for base, size in
                        ((0, 32), (512, 32), (1024, self.meta), (1024 + 16 * self.meta, self.meta))], 1).cuda()
        for b, (n, m) in enumerate(zip(self.lens, counts)):
            for h in range(self.h):
                if (b, h) in skip:
                    continue
                i = torch.tensor([x for x in range(m) if (b, h, x) not in skip], device="cuda", dtype=torch.long)
                src = kept[b, h].long()[i]
                pool[page(b, i)[:, None], h, at[slot(i)]] = self.pool[page(b, src)[:, None], h, at[slot(src)]]
                score[b, h, m:n] = 0
                score[b, h, i] = self.score[b, h, src]
                if win is not None and self.recent and m < n:
                    row = lambda s: self.sink + (s - self.sink) % self.recent
                    pos = torch.arange(n - self.recent, n, device="cuda")
                    sl = int(self.slots[b])
                    win[sl, h, :, row(pos - (n - m))] = self.win.view(torch.int16)[sl, h, :, row(pos)]
        return pool, score, win

    def check(self, want, score=True):
        pool, s, win = want
        assert torch.equal(self.pool, pool)
        if score:
            assert torch.equal(self.score, s)
        if win is not None:
            assert torch.equal(self.win.view(torch.int16), win)


CONFIGS = [dict(), dict(group=128), dict(sink=16, recent=100), dict(sink=0, recent=33), dict(sink=48, recent=0), PAPER]


@pytest.mark.parametrize("opts", CONFIGS)
@pytest.mark.parametrize("lens,counts", [
    ([500], [400]), ([1000, 777, 500], [400, 777, 499]), ([3000], [1700]), ([20000], [9001]), ([5000] * 20, [2048] * 20),
])
def test_move(lens, counts, opts):
    c = Cache(lens, **opts)
    kept = c.lists(counts)
    want = c.plain(kept, counts)
    c.run(kept, counts)
    c.check(want)
    assert optr.optr_device_error(c.p) == 0


@pytest.mark.parametrize("opts", CONFIGS[:2])
@pytest.mark.parametrize("lens,counts", [
    ([0], [0]), ([1], [0]), ([1], [1]), ([2, 33, 0], [1, 0, 0]), ([17], [16]), ([600], [1]), ([40000], [33000]),
    ([1030, 1], [1025, 1]),
])
def test_small_and_whole_lists(lens, counts, opts):
    c = Cache(lens, seed=1, **opts)
    kept = c.lists(counts)
    want = c.plain(kept, counts)
    c.run(kept, counts)
    c.check(want)
    assert optr.optr_device_error(c.p) == 0


@pytest.mark.parametrize("kind", ["the last", "the first", "one gap", "every second"])
@pytest.mark.parametrize("group", [32, 128])
def test_shapes_of_lists(kind, group):
    """Sources far behind their destinations, on them, one behind, and twice as far."""
    n, m = 9000, 4500
    c = Cache([n], h_kv=1, seed=2, group=group)
    x = {"the last": range(n - m, n), "the first": range(m), "one gap": [i + (i >= 5) for i in range(m)],
         "every second": range(1, 2 * m, 2)}[kind]
    kept = i32(x).view(1, 1, m)
    want = c.plain(kept, [m])
    c.run(kept, [m])
    c.check(want)


def test_without_scores():
    c = Cache([700], seed=3)
    kept = c.lists([300])
    pool, _, _ = c.plain(kept, [300])
    before = c.score.clone()
    c.run(kept, [300], score=False)
    assert torch.equal(c.pool, pool) and torch.equal(c.score, before)


def test_the_longest_ring():
    c = Cache([5000], h_kv=1, seed=4, sink=1024, recent=1024)
    kept = c.lists([3001])
    want = c.plain(kept, [3001])
    c.run(kept, [3001])
    c.check(want)


def test_lists_out_of_order_are_flagged_entry_by_entry():
    c = Cache([2000], seed=5)
    m = 1500
    kept = c.lists([m])
    kept[0, 0, 700] = 2000            # behind the end
    kept[0, 1, 40] = 39               # before its destination
    kept[0, 1, 900] = kept[0, 1, 899]  # twice
    skip = {(0, 0, 700), (0, 1, 40), (0, 1, 900)}
    # the entry behind 2000 does not rise either
    skip.add((0, 0, 701))
    want = c.plain(kept, [m], skip)
    score = want[1]
    c.run(kept, [m])
    assert torch.equal(c.pool, want[0])
    assert torch.equal(c.score, score)
    assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_KEPT


def test_pages_out_of_range_are_flagged_and_left():
    c = Cache([100], h_kv=1, seed=6)
    kept = i32(range(20, 100)).view(1, 1, 80)
    bt = c.bt.clone()
    bt[0, 2], bt[0, 4] = -1, c.pool.shape[0]   # positions 32 .. 47 and 64 .. 79, as sources and destinations
    skip = {(0, 0, i) for i in range(80) if i // 16 in (2, 4) or (i + 20) // 16 in (2, 4)}
    want = c.plain(kept, [80], skip)
    c.run(kept, [80], bt=bt)
    assert torch.equal(c.pool, want[0])
    assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_PAGE_ID


def test_counts_out_of_range_leave_the_sequence():
    c = Cache([100, 100, 100, 100], seed=7)
    counts = [50, 101, -1, 50]
    kept = c.lists([50, 100, 50, 50])
    pages = c.bt.shape[1]
    lens = i32([100, 100, 100, 16 * pages + 1])
    want = c.plain(kept, counts, skip={(b, h) for b in (1, 2, 3) for h in (0, 1)})
    c.run(kept, counts, lens=lens)
    c.check(want)
    assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_SEQ_LEN


def test_windows_that_are_not_kept_leave_the_head():
    c = Cache([900, 900, 900], seed=8, **PAPER)
    counts = [600, 600, 319]           # fewer than the windows' 320
    kept = c.lists([600, 600, 600])
    kept[0, 0, 63] = 64 if int(kept[0, 0, 64]) > 64 else 63
    kept[0, 0, :64] = torch.arange(1, 65).int()
    kept[1, 1, 600 - 256] -= 1
    skip = {(0, 0), (1, 1), (2, 0), (2, 1)}
    want = c.plain(kept, counts, skip)
    c.run(kept, counts)
    c.check(want)
    assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_KEPT
    c = Cache([900, 900], seed=9, **PAPER)
    kept = c.lists([600, 600])
    want = c.plain(kept, [600, 600], skip={(1, 0), (1, 1)})
    slots = c.slots.clone()
    slots[1] = 4
    c.run(kept, [600, 600], slots=slots)
    c.check(want)
    assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_WIN_SLOT


def test_move_refusals():
    c = Cache([100], seed=10)
    kept = c.lists([50])
    for bad in (lambda: c.run(kept.long(), [50]), lambda: c.run(kept[:, :1], [50]), lambda: c.run(kept, [50, 50]),
                lambda: optr.optr_kv_compact(c.p, kept, i32([50]), i32([100]), c.bt, c.pool, c.score.half())):
        with pytest.raises(ValueError):
            bad()
    w = Cache([400], seed=10, **PAPER)
    with pytest.raises(optr.OptrError):   # windows need the _win call
        optr.optr_kv_compact(w.p, w.lists([350]), i32([350]), i32([400]), w.bt, w.pool)
    with pytest.raises(optr.OptrError):
        optr.optr_kv_compact_win(w.p, w.lists([350]), i32([350]), i32([400]), w.bt, w.pool, None, None)


def test_choice_and_move_in_a_graph():
    """Replayed on another cache's bytes: the lists and counts of the replay's time."""
    c = Cache([3000, 900], seed=11, **PAPER)
    keep, lens = i32([1000, 800]), i32([3000, 900])
    kept = torch.full((2, 2, 1000), -1, dtype=torch.int32, device="cuda")
    n_kept = torch.zeros(2, dtype=torch.int32, device="cuda")

    def call():
        optr.optr_evict_select(c.p, c.score, lens, keep, 64, 256, kept, n_kept)
        optr.optr_kv_compact_win(c.p, kept, n_kept, lens, c.bt, c.pool, c.win, c.slots, c.score)

    saved = [x.clone() for x in (c.pool, c.score, c.win)]
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for seed in (1, 2):
        for x, y in zip((c.pool, c.score, c.win), saved):
            x.copy_(y)
        c.score.mul_(torch.rand(c.score.shape, device="cuda", generator=c.g))
        lists = torch.tensor(plain_select(c.score, [3000, 900], [1000, 800], 64, 256, 1000)[0], device="cuda").int()
        want = c.plain(lists, [1000, 800])
        g.replay()
        c.check(want)
    assert optr.optr_device_error(c.p) == 0


@pytest.mark.parametrize("n,counts,opts", [(20000, 9001, dict()), (9000, 8700, dict(group=128)), (33000, 32000, PAPER)])
def test_long_lists_of_one_sequence(n, counts, opts):
    """More chunks than one, in clusters of every width (16 CTAs from 8193 places on)."""
    c = Cache([n], seed=n % 7, **opts)
    kept = c.lists([counts])
    want = c.plain(kept, [counts])
    c.run(kept, [counts])
    c.check(want)
    assert optr.optr_device_error(c.p) == 0


@pytest.mark.parametrize("B,n,h", [(16, 4097, 8), (19, 8192, 8), (5, 70000, 4), (4, 131072, 4)])
def test_choice_in_every_split(B, n, h):
    """Rows that one CTA takes, and clusters of 2, 4 and 8 with up to 64 scores a thread."""
    g = torch.Generator(device="cuda").manual_seed(n)
    p = params(h)
    score = torch.rand(B, h, n, device="cuda", generator=g)
    score[:, :, ::3] = 0.0
    k = n // 3 + 7
    kept = torch.full((B, h, k), -1, dtype=torch.int32, device="cuda")
    count = i32([0] * B)
    optr.optr_evict_select(p, score, i32([n] * B), i32([k] * B), 4, 64, kept, count)
    key = score.clone()
    key[:, :, :4] = 2.0
    key[:, :, -64:] = 2.0
    order = key.sort(dim=2, descending=True, stable=True).indices[:, :, :k]
    assert torch.equal(kept.long(), order.sort(dim=2).values) and count.tolist() == [k] * B
