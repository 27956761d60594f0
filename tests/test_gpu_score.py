"""Attention weights summed by position (optr_kv_score) against the formula in 64 bits.

Tolerance.  Queries (over a power of two by row) and keys (by key) enter in fp16 hi + lo
parts, each within 2^-22 of its largest, products and sums in float32: of 128 products
q_i k_i each is off by some 2^-22 |q_i k_i| at random, and the rotation's float32 sums add
as much, so a logit l (of size |q||k| / sqrt(128), in units of e) by some 4 * 2^-22 of
sqrt(sum (q_i k_i)^2) / sqrt(128), which is below |q||k| / 128: at |q| = 1.5 sqrt(128) and |k| =
sqrt(128) by 1.5e-6, at 10 times the largest |k| and a queries' scale s by 1e-6 s with room.  A weight
moves by that factor, and a sum of weights by no more than its largest; exp2's
approximation, the sums' and the normaliser's roundings add a few 2^-22.  So each position's sum is held to 8e-6
(1 + scale) of itself plus 2^-24 of what was there before, twelve deviations and more, and the norm to a fifth."""
import math
import random

import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_chunk import PAPER, Case, cu_of, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


class Score(Case):
    """test_gpu_chunk's cache of past + new tokens, whose last ones are the new ones."""

    def __init__(self, new, past, scale=1.5, spare=0, **kw):
        super().__init__([0] * len(new), [a + b for a, b in zip(past, new)], scale=scale, spare=spare, **kw)
        self.new, self.past = new, past
        self.n = [a + b for a, b in zip(past, new)]
        g = torch.Generator(device="cuda").manual_seed(99 + len(new))
        t = sum(new)
        self.q = (torch.randn(t, 4 * self.h, 128, device="cuda", generator=g) * scale).bfloat16()
        self.cu, self.pos0 = cu_of(new), i32(past)
        self.max_new = max(1, max(new))
        self.n_score = 16 * self.bt.shape[1] + 3
        self.score = torch.rand(self.B, self.h, self.n_score, device="cuda", generator=g)
        self.scale = scale

    def run(self, **over):
        a = dict(q=self.q, cu=self.cu, pos0=self.pos0, max_new=self.max_new, bt=self.bt, slots=self.slots,
                 score=self.score)
        a.update(over)
        ws = optr.new_score_workspace(self.p, a["q"].shape[0], self.B, a["max_new"], self.bt.shape[1])
        ws.fill_(0xA5)
        args = (self.p, a["q"], a["cu"], a["pos0"], a["max_new"], a["bt"], self.pool)
        out = a["score"].clone()
        if self.win is None:
            optr.optr_kv_score(*args, out, ws)
        else:
            optr.optr_kv_score_win(*args, self.win, a["slots"], out, ws)
        return out

    def added(self, drop=(), windows=True):
        """What is added, in 64 bits; positions (b, s) of `drop` are left out."""
        out = torch.zeros(self.B, self.h, self.n_score, dtype=torch.float64, device="cuda")
        cu = self.cu.tolist()
        for b, n in enumerate(self.n):
            r0, r1 = cu[b], cu[b + 1]
            if r1 == r0:
                continue
            pos = torch.arange(n, device="cuda")
            exact = (pos < self.sink) | (pos >= n - self.recent)
            gone = torch.zeros(n, dtype=torch.bool, device="cuda")
            for bb, s in drop:
                if bb == b:
                    gone[s] = True
            i = torch.arange(r1 - r0, device="cuda")[:, None]
            for h in range(self.h):
                k = self.rows(b, h, 0, n, 0) @ self.R_k[h].T
                if self.win is not None:
                    s = pos[exact]
                    row = torch.where(s < self.sink, s, self.sink + (s - self.sink) % max(1, self.recent))
                    if windows:
                        k[exact] = self.win[int(self.slots[b]), h][0, row].double() - self.mu[h]
                    else:
                        gone[s] = True
                for j in range(4):
                    l = self.q[r0:r1, 4 * h + j].double() @ k.T / 128 ** 0.5
                    l = l.masked_fill((pos > self.past[b] + i) | gone, -math.inf)
                    out[b, h, :n] += torch.softmax(l, 1).nan_to_num(0.0).sum(0)
        return out

    def check(self, got, want=None, before=None):
        before = self.score if before is None else before
        add = self.added() if want is None else want
        want = before.double() + add
        assert torch.isfinite(got).all()
        err = (got.double() - want).abs()
        tol = 8e-6 * (1 + self.scale)
        # one rounding of the sum that is there for each 64 tokens
        allowed = tol * add + 2.0 ** -24 * want * (1 + max(self.new) // 64) * 1.01
        worst = (err - allowed).max().item()
        assert worst <= 0, (worst, (err / (add + 1e-30)).max().item())
        assert torch.equal(got[add == 0], before[add == 0])
        assert err.norm() <= tol / 5 * add.norm() + 2.0 ** -24 * want.norm()


SHAPES = [
    ([1], [0]), ([1], [1]), ([1], [15]), ([1], [16]), ([1], [127]), ([1], [128]), ([1], [1023]), ([2], [0]),
    ([4], [300]), ([5], [2049]), ([8], [120]), ([9], [400]), ([31], [300]), ([32], [300]), ([33], [300]), ([63], [1]),
    ([64], [0]), ([64], [5000]), ([65], [0]), ([129], [7]), ([200], [4000]),
    ([2, 0, 5, 1], [100, 50, 0, 3000]), ([0, 0, 3], [0, 9, 500]), ([70, 1, 130], [40, 5000, 0]),
    ([1] * 40, list(range(0, 1200, 30))), ([3, 1, 4, 2] * 10, list(range(0, 1200, 30))), ([300], [1000]),
]
CONFIGS = [dict(), dict(group=128), dict(sink=16, recent=100), dict(sink=0, recent=33),
           dict(sink=48, recent=0), PAPER, dict(PAPER, fold=True), dict(h_kv=1), dict(h_kv=8)]


@pytest.mark.parametrize("new,past", SHAPES)
@pytest.mark.parametrize("opts", CONFIGS[:1] + CONFIGS[2:3] + CONFIGS[5:6])
def test_matches_the_formula(new, past, opts):
    c = Score(new, past, **opts)
    c.check(c.run())
    assert optr.optr_device_error(c.p) == 0


@pytest.mark.parametrize("opts", CONFIGS)
@pytest.mark.parametrize("new,past", [([1, 1, 1], [1000, 333, 70]), ([3, 40], [1000, 333]), ([150], [700])])
def test_configurations(new, past, opts):
    c = Score(new, past, seed=1, **opts)
    c.check(c.run())
    assert optr.optr_device_error(c.p) == 0


@pytest.mark.parametrize("new", [[1], [7], [64]])
def test_long_context_is_split_and_joined(new):
    c = Score(new, [60000], h_kv=1, seed=2)
    c.check(c.run())


def test_each_token_gives_its_weight_of_one():
    """Every head of every token gives weights that sum to 1: 4 m a KV head, to 1e-5 of it."""
    c = Score([1, 40, 100], [3000, 77, 0], seed=3, sink=16, recent=100)
    got = c.run(score=torch.zeros_like(c.score)).double().sum(2)
    want = torch.tensor([4.0, 160.0, 400.0], device="cuda", dtype=torch.float64)[:, None].expand_as(got)
    assert ((got - want).abs() <= 1e-5 * want).all(), got


@pytest.mark.parametrize("new", [[2], [40]])
@pytest.mark.parametrize("scale", [1e-20, 12.0, 60.0, 2e4])
@pytest.mark.parametrize("opts", [dict(), PAPER])
def test_small_and_large_queries(new, scale, opts):
    """Uniform weights at one end; at the other a logit of thousands, far past the range of a float's
    exponent from one tile to the next: the largest keys alone count.  Two near maxima may then share
    otherwise than in 64 bits, so above 60 only the weights' sum and their place are held.  A logit of L (in
    units of log2) is a float32 sum of 24 products a step, each step rounded to 2^-24 L: 5 of these at random,
    and as many as two more by the reference and the normaliser of that size.  So a weight, computed once for
    the normaliser and once for the sum, moves by a factor of 2^(8 * 2^-24 L) at most, and so does their sum."""
    c = Score(new, [900], scale=scale, seed=4, **opts)
    got = c.run()
    assert torch.isfinite(got).all()
    if scale < 100:
        c.check(got)
    add = (got.double() - c.score.double())
    q, k = c.q.double().norm(dim=2).max(), max((c.rows(0, h, 0, c.n[0], 0).norm(dim=1).max() for h in range(c.h)))
    if c.win is not None:
        k = max(k, (c.win[int(c.slots[0])][:, 0].double() - c.mu[:, None]).norm(dim=2).nan_to_num(0).max())
    L = float(q * k) / 128 ** 0.5 / math.log(2)
    tol = 1e-4 + math.expm1(math.log(2) * 8 * L * 2.0 ** -24)
    assert ((add.sum(2) - 4 * new[0]).abs() <= tol * 4 * new[0]).all()
    assert add.min() >= -1e-6 and torch.equal(got[:, :, c.n[0]:], c.score[:, :, c.n[0]:])


def test_a_needle_far_above_the_first_keys():
    """One cached key of 40 times the size, behind many tiles: its logits pass those of the tiles before
    by more than a float's exponent range, for some rows upwards, for others downwards."""
    for at in (5, 3000, 5990):
        c = Score([8], [6000], h_kv=1, seed=5, scale=6.0)
        k = c.q[0, 0].double() * 8
        mu = c.mu.float()
        k = (k.float() + mu[0]).bfloat16().view(1, 1, 128)
        optr.optr_kv_append(c.p, k, k, cu_of([1]), i32([at]), c.bt, c.pool)
        got = c.run()
        c.check(got)


def test_equal_calls_give_equal_bits():
    for new, past in (([40, 3, 64], [3000, 9000, 64]), ([1, 1, 1], [3000, 9000, 64])):
        c = Score(new, past, seed=6)
        first = c.run()
        for _ in range(3):
            assert torch.equal(c.run(), first)


def test_sequences_do_not_touch_each_other():
    c = Score([3, 40, 1], [500, 90, 2000], seed=7)
    both = c.run()
    for b in range(3):
        cu, new = c.cu.tolist(), [0, 0, 0]
        new[b] = c.new[b]
        # n - new before: the others get no token
        got = c.run(q=c.q[cu[b]:cu[b + 1]].contiguous(), cu=cu_of(new))
        assert torch.equal(got[b], both[b])
        others = [x for x in range(3) if x != b]
        assert torch.equal(got[others], c.score[others])


@pytest.mark.parametrize("new", [[3, 2], [70, 9]])
def test_pages_out_of_range_are_left_out(new):
    c = Score(new, [300, 600], seed=8)
    bt = c.bt.clone()
    bt[0, 3], bt[1, 20] = -1, c.pool.shape[0]
    drop = [(0, s) for s in range(48, 64)] + [(1, s) for s in range(320, 336)]
    c.check(c.run(bt=bt), c.added(drop))
    assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_PAGE_ID


@pytest.mark.parametrize("new", [[3, 2], [70, 9]])
def test_window_slots_out_of_range_are_left_out(new):
    c = Score(new, [700, 600], seed=9, **PAPER)
    slots = c.slots.clone()
    slots[0] = 4
    want = c.added()
    want[0] = c.added(windows=False)[0]
    c.check(c.run(slots=slots), want)
    assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_WIN_SLOT


@pytest.mark.parametrize("new", [[3, 2], [70, 9]])
def test_sequences_out_of_range_add_nothing(new):
    c = Score(new, [300, 600], seed=10)
    want = c.added()
    pages = c.bt.shape[1]
    for bad in (-1, 16 * pages - new[0] + 1):
        want[0] = 0
        c.check(c.run(pos0=i32([bad, 600])), want)
        assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_SEQ_LEN
    c.check(c.run(max_new=new[0] - 1), want)
    assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_CU_NEW
    short = c.score[:, :, :300].contiguous()     # fewer sums than positions
    got = c.run(score=short)
    assert torch.equal(got, short)
    assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_SEQ_LEN


def test_refusals():
    c = Score([3], [300], seed=11)
    ws = optr.new_score_workspace(c.p, 3, 1, 3, c.bt.shape[1])
    args = (c.p, c.q, c.cu, c.pos0, 3, c.bt, c.pool)
    with pytest.raises(optr.OptrError) as e:
        optr.optr_kv_score(*args, c.score, ws[:-256])
    assert e.value.status == -4
    with pytest.raises(optr.OptrError):
        optr.optr_kv_score(*args, c.score, ws[1:])
    with pytest.raises(ValueError):
        optr.optr_kv_score(*args, c.score.half(), ws)
    with pytest.raises(ValueError):
        optr.optr_kv_score(*args, c.score[:, :1], ws)
    with pytest.raises(ValueError):
        optr.optr_kv_score(c.p, c.q.float(), *args[2:], c.score, ws)
    with pytest.raises(ValueError):
        optr.optr_kv_score(c.p, c.q.cpu(), *args[2:], c.score, ws)
    with pytest.raises(optr.OptrError):
        optr.optr_kv_score(*args[:4], 0, *args[5:], c.score, ws)
    w = Score([3], [300], seed=11, **PAPER)
    with pytest.raises(optr.OptrError):
        optr.optr_kv_score(w.p, w.q, w.cu, w.pos0, 3, w.bt, w.pool, w.score, ws)


@pytest.mark.parametrize("new", [[2, 1], [40, 70]])
def test_another_stream_and_a_captured_graph(new):
    c = Score(new, [500, 90], seed=12, **PAPER)
    want = c.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = c.run()
    s.synchronize()
    assert torch.equal(got, want)
    m = max(new)
    ws = optr.new_score_workspace(c.p, sum(new), 2, m, c.bt.shape[1])
    out = c.score.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        optr.optr_kv_score_win(c.p, c.q, c.cu, c.pos0, m, c.bt, c.pool, c.win, c.slots, out, ws)
    for r in range(2):
        c.q.copy_(torch.randn_like(c.q.float()) * 1.5)
        out.copy_(c.score)
        g.replay()
        c.check(out)


def test_many_sequences():
    r = random.Random(13)
    new = [r.choice([0, 1, 1, 2, 3, 9]) for _ in range(100)]
    past = [r.randint(0, 400) for _ in range(100)]
    c = Score(new, past, h_kv=2, seed=13, sink=16, recent=20)
    c.check(c.run())
