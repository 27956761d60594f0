"""Attention of a chunk of new tokens over the paged cache (optr_chunk_attention)
against the formula in 64 bits: INT2 past, BF16 windows of the past, the chunk's
own tokens causally.

Tolerance.  The kernel rounds the rotated query and the dequantized keys, values
and INT2 probabilities to fp16 (unit roundoff 2^-11 of each), the probabilities
of exact tokens and the output to bf16 (2^-8 spacing, 2^-9 roundoff).  A row's
output is a mean of values with weights p, so the probability and value roundings
move it by at most (2^-9 + 2^-11) max|v| in total, a logit rounding d of a
weight moves it by at most 2 d max|v|, and a logit's roundings (query and key)
are at most 2 * 2^-11 |q||k| / sqrt(128), far below that for independent signs:
sqrt(128) terms of |q_i k_i| 2^-11 / sqrt(3).  The tests bound the worst element
by 2^-6 of the output's largest value in the row's KV head, four times the sum
of 2^-8 (weights, output) and the logits' share, and the relative 2-norm by
2^-8 (twice the two bf16 roundings' rms of 2^-9 / sqrt(3) each, in quadrature
with the fp16 ones)."""
import math

import pytest
import torch

from paper_2608_02691_gb300 import optr, synth

pytestmark = pytest.mark.gpu

PAPER = dict(group=128, clip_k=0.96, clip_v=0.92, sink=64, recent=256)


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def cu_of(lens):
    return i32([0] + list(torch.tensor(lens).cumsum(0).tolist())) if lens else i32([0])


class Case:
    """A cache of `past` tokens per sequence written by the library, and the
    new tokens of a chunk.  Unwritten bytes of the pool read as NaN metadata,
    unwritten window rows hold NaN."""

    def __init__(self, new, past, h_kv=2, fold=False, seed=0, max_new=None, scale=1.0, spare=0, **opts):
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s: torch.randn(*s, device="cuda", generator=g)
        B = len(new)
        self.new, self.past, self.h, self.B = new, past, h_kv, B
        self.sink, self.recent = opts.get("sink", 0), opts.get("recent", 0)
        R_k, R_v = synth.rotations(h_kv, seed)
        mu = torch.zeros(h_kv, 128)
        mu[:, ::37] = 7.0
        self.R_k, self.R_v, self.mu = R_k.cuda().double(), None if fold else R_v.cuda().double(), mu.cuda().double()
        self.p = optr.optr_params_create(R_k, None if fold else R_v, mu, 4 * h_kv, **opts)
        self.group = opts.get("group", 32)
        pages = max(1, max(-(-(s + n) // 16) for s, n in zip(past, new))) + spare
        num = B * pages + 2
        self.pool = optr.new_pool(self.p, num).fill_(0xFF)
        self.bt = torch.randperm(num, generator=g, device="cuda")[:B * pages].view(B, pages).int()
        self.win = self.slots = None
        if self.sink + self.recent:
            self.win = optr.new_windows(self.p, B + 2).fill_(math.nan)
            self.slots = torch.randperm(B + 2, generator=g, device="cuda")[:B].int()
        n = sum(past)
        if n:
            k, v = (randn(n, h_kv, 128) + mu.cuda()).bfloat16(), (2 * randn(n, h_kv, 128)).bfloat16()
            args = (self.p, k, v, cu_of(past), i32([0] * B), self.bt, self.pool)
            if self.win is None:
                optr.optr_kv_append(*args)
            else:
                optr.optr_kv_append_win(*args, self.win, self.slots)
        t = sum(new)
        self.q = (randn(t, 4 * h_kv, 128) * scale).bfloat16()
        self.k, self.v = (randn(t, h_kv, 128) + mu.cuda()).bfloat16(), (2 * randn(t, h_kv, 128)).bfloat16()
        self.cu, self.pos0 = cu_of(new), i32(past)
        self.max_new = max_new or max(1, max(new))
        self.out = torch.full_like(self.q, 7.0)

    def run(self, **over):
        a = dict(q=self.q, k=self.k, v=self.v, cu=self.cu, pos0=self.pos0, bt=self.bt, out=self.out,
                 max_new=self.max_new, slots=self.slots)
        a.update(over)
        ws = optr.new_chunk_workspace(self.p, a["q"].shape[0], self.B, a["max_new"])
        ws.fill_(0xA5)  # scratch needs no initialisation
        args = (self.p, a["q"], a["k"], a["v"], a["cu"], a["pos0"], a["max_new"], a["bt"], self.pool)
        if self.win is None:
            optr.optr_chunk_attention(*args, a["out"], ws)
        else:
            optr.optr_chunk_attention_win(*args, self.win, a["slots"], a["out"], ws)
        return a["out"]

    def rows(self, b, h, lo, hi, kind, bt=None):
        """Dequantized rotated rows of positions lo .. hi-1, 64 bits."""
        pos = torch.arange(lo, hi, device="cuda")
        rec = self.pool[(self.bt if bt is None else bt)[b].long()[pos // 16], h]
        slot, ch = (pos % 16)[:, None], torch.arange(128, device="cuda")
        code = rec.gather(1, 512 * kind + 32 * slot + 4 * (ch % 32 // 4) + ch // 32) >> (2 * (ch % 4)) & 3
        ng = 128 // self.group
        at = 1024 + 64 * ng * kind + 4 * ng * slot + 4 * (ch // self.group)
        half = lambda o: torch.stack((rec.gather(1, at + o), rec.gather(1, at + o + 1)), 2).view(torch.float16)[..., 0].double()
        return code * half(0) + half(2)

    def reference(self, drop=()):
        """The formula; positions (b, s) of `drop` are left out."""
        out = torch.zeros_like(self.q, dtype=torch.float64)
        cu = self.cu.tolist()
        for b in range(self.B):
            n, r0, r1 = self.past[b], cu[b], cu[b + 1]
            pos = torch.arange(n, device="cuda")
            exact = (pos < self.sink) | (pos >= n - self.recent)
            gone = torch.zeros(n, dtype=torch.bool, device="cuda")
            for bb, s in drop:
                if bb == b:
                    gone[s] = True
            for h in range(self.h):
                k = torch.empty(n, 128, dtype=torch.float64, device="cuda")
                v = torch.empty_like(k)
                if n:
                    k[:], v[:] = self.rows(b, h, 0, n, 0) @ self.R_k[h].T, self.rows(b, h, 0, n, 1)
                    if self.R_v is not None:
                        v[:] = v @ self.R_v[h].T
                    if self.win is not None:
                        s = pos[exact]
                        row = torch.where(s < self.sink, s, self.sink + (s - self.sink) % max(1, self.recent))
                        w = self.win[int(self.slots[b]), h]
                        k[exact], v[exact] = w[0, row].double() - self.mu[h], w[1, row].double()
                k = torch.cat((k[~gone], self.k[r0:r1, h].double() - self.mu[h]))
                v = torch.cat((v[~gone], self.v[r0:r1, h].double()))
                i = torch.arange(r1 - r0, device="cuda")
                m = k.shape[0] - (r1 - r0)
                for j in range(4):
                    l = self.q[r0:r1, 4 * h + j].double() @ k.T / 128 ** 0.5
                    l[:, m:].masked_fill_(i > i[:, None], -math.inf)
                    out[r0:r1, 4 * h + j] = torch.softmax(l, 1) @ v
        return out


def check(got, want):
    got = got.double()
    assert torch.isfinite(got).all()
    err = (got - want).abs().max().item()
    assert err <= 2.0 ** -6 * want.abs().max().item(), err
    rel = ((got - want).norm() / want.norm()).item()
    assert rel <= 2.0 ** -8, rel


SHAPES = [
    ([1], [0]), ([1], [1]), ([1], [15]), ([1], [16]), ([1], [17]), ([1], [127]), ([1], [128]),
    ([1], [129]), ([1], [1024]), ([5], [2049]), ([31], [300]), ([32], [300]), ([33], [300]),
    ([63], [1]), ([64], [0]), ([65], [0]), ([127], [100]), ([129], [7]), ([200], [4000]),
    ([2, 0, 5, 1], [100, 50, 0, 3000]), ([0, 0, 3], [0, 9, 500]), ([70, 1, 130], [40, 5000, 0]),
    ([1] * 40, list(range(0, 1200, 30))), ([700], [0]), ([300, 513], [1000, 2000]),
]
CONFIGS = [dict(), dict(group=128), dict(sink=16, recent=100), dict(sink=0, recent=33),
           dict(sink=48, recent=0), PAPER, dict(PAPER, fold=True), dict(fold=True, h_kv=1)]


@pytest.mark.parametrize("new,past", SHAPES)
@pytest.mark.parametrize("opts", CONFIGS[:1] + CONFIGS[2:3] + CONFIGS[5:6])
def test_matches_the_formula(new, past, opts):
    c = Case(new, past, **opts)
    check(c.run(), c.reference())
    assert optr.optr_device_error(c.p) == 0


@pytest.mark.parametrize("opts", CONFIGS)
@pytest.mark.parametrize("new,past", [([3, 40], [1000, 333]), ([150], [700])])
def test_configurations(new, past, opts):
    c = Case(new, past, seed=1, **opts)
    check(c.run(), c.reference())
    assert optr.optr_device_error(c.p) == 0


def test_long_context_is_split_and_joined():
    c = Case([3], [40000], h_kv=1, seed=2)
    check(c.run(), c.reference())


def test_equal_calls_give_equal_bits():
    c = Case([40, 3, 700], [3000, 9000, 64], seed=3)
    first = c.run().clone()
    for _ in range(3):
        assert torch.equal(c.run(), first)


@pytest.mark.parametrize("scale", [1e-20, 30.0, 1e4])
def test_small_and_large_queries(scale):
    """Uniform weights at one end; at the other a weight of 1, where rounding a
    logit may move the choice between two near maxima: their values bound the
    error then, so only finiteness and the convex hull are checked."""
    c = Case([9], [500], scale=scale, seed=4)
    got, want = c.run(), c.reference()
    if scale < 1:
        check(got, want)
    else:
        assert torch.isfinite(got).all()
        assert got.double().abs().max() <= want.abs().max() * 1.5


def test_one_growing_key_per_tile_rescales():
    """Maxima that grow from tile to tile by far more than the slack."""
    c = Case([1], [640], h_kv=1, seed=5, group=128)
    n = c.past[0]
    k = torch.randn(n, 1, 128, device="cuda")
    d = c.q[0, 0].float() / c.q[0, 0].float().norm()
    k[::128, 0] += d * torch.linspace(5, 60, 5, device="cuda")[:, None]
    optr.optr_kv_append(c.p, (k + c.mu.float()).bfloat16(), torch.randn_like(k).bfloat16(), cu_of([n]),
                        i32([0]), c.bt, c.pool)
    check(c.run(), c.reference())


def test_other_rows_do_not_matter():
    """NaN in a neighbouring sequence's rows stays there; rows of the pool past
    a sequence's length, spare table columns and unused slots too."""
    c = Case([5, 40, 3], [100, 30, 500], spare=3, sink=16, recent=40, seed=6)
    want = c.reference()
    c.q[5:45], c.k[5:45], c.v[5:45] = math.nan, math.nan, math.inf
    got = c.run().double()
    keep = torch.ones(48, dtype=torch.bool)
    keep[5:45] = False
    check(got[keep.cuda()], want[keep.cuda()])


def test_future_keys_do_not_matter():
    c = Case([100], [200], seed=7)
    want = c.run().clone()
    c.k[60:] = 50.0
    assert torch.equal(c.run()[:60], want[:60])


def test_bad_tables_are_flagged_and_left_out():
    c = Case([4, 4], [200, 300], seed=8)
    bad = c.bt.clone()
    bad[0, 3], bad[1, 0] = -1, c.pool.shape[0]
    drop = [(0, s) for s in range(48, 64)] + [(1, s) for s in range(16)]
    check(c.run(bt=bad), c.reference(drop))
    assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_PAGE_ID
    # a sequence that cannot be right gets zero rows, the others are as ever
    want = c.reference()
    for over, bit in ((dict(pos0=i32([-1, 300])), optr.OPTR_DEVERR_SEQ_LEN),
                      (dict(pos0=i32([16 * c.bt.shape[1] + 1, 300])), optr.OPTR_DEVERR_SEQ_LEN)):
        got = c.run(**over)
        assert not got[:4].any()
        check(got[4:], want[4:])
        assert optr.optr_device_error(c.p) == bit
    got = c.run(max_new=3)
    assert not got.any() and optr.optr_device_error(c.p) == optr.OPTR_DEVERR_CU_NEW
    got = c.run(cu=i32([0, 4, 5]))  # rows 5 .. 7 belong to nobody
    check(got[:4], want[:4])
    assert not got[5:].any() and optr.optr_device_error(c.p) == optr.OPTR_DEVERR_CU_NEW


def test_bad_window_slot_is_flagged():
    c = Case([2, 2], [100, 100], sink=16, recent=20, seed=9)
    drop = [(0, s) for s in list(range(16)) + list(range(80, 100))]
    want = c.reference(drop)
    slots = c.slots.clone()
    slots[0] = c.win.shape[0]
    check(c.run(slots=slots), want)
    assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_WIN_SLOT


def test_one_new_token_equals_the_decode_where_both_are_defined():
    """The decode over n cached tokens is the chunk attention without the own
    token; with the own token's window exact and everything else INT2 the two
    agree: recent = 1 holds just the new token."""
    c = Case([1, 1], [500, 77], sink=0, recent=1, seed=10)
    # the past's newest token is in the window too: read it from the store
    got = c.run().float().clone()
    want = c.reference()
    check(got, want)


def test_other_stream_and_graph():
    c = Case([40, 2], [700, 4000], seed=11)
    want = c.run().clone()
    ws = optr.new_chunk_workspace(c.p, 42, 2, c.max_new)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.out.zero_()
        optr.optr_chunk_attention(c.p, c.q, c.k, c.v, c.cu, c.pos0, c.max_new, c.bt, c.pool, c.out, ws)
    s.synchronize()
    assert torch.equal(c.out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        optr.optr_chunk_attention(c.p, c.q, c.k, c.v, c.cu, c.pos0, c.max_new, c.bt, c.pool, c.out, ws)
    c.out.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.out, want)


def test_refusals():
    c = Case([4], [100], seed=12)
    ws = optr.new_chunk_workspace(c.p, 4, 1, 4)
    call = lambda q=c.q, k=c.k, v=c.v, cu=c.cu, m=4, bt=c.bt, out=c.out, ws=ws: \
        optr.optr_chunk_attention(c.p, q, k, v, cu, c.pos0, m, bt, c.pool, out, ws)
    for bad in (dict(q=c.q.cpu()), dict(q=c.q.float()), dict(out=c.out.float()), dict(k=c.k[:3]),
                dict(k=c.k.transpose(0, 1)), dict(v=c.v.half()), dict(cu=c.cu.long()), dict(cu=c.cu[:1]),
                dict(q=c.q.cpu().pin_memory())):
        with pytest.raises(ValueError):
            call(**bad)
    for bad, status in ((dict(m=0), -1), (dict(ws=ws[:-1]), -4), (dict(ws=ws[1:]), -4)):
        with pytest.raises(optr.OptrError) as e:
            call(**bad)
        assert e.value.status == status
    w = Case([4], [100], sink=16, recent=20, seed=12)
    with pytest.raises(optr.OptrError):  # windows need the store
        optr.optr_chunk_attention(w.p, w.q, w.k, w.v, w.cu, w.pos0, 4, w.bt, w.pool, w.out, ws)
    assert (c.out == 7.0).all() and (w.out == 7.0).all()
    z = c.q[:0]
    optr.optr_chunk_attention(c.p, z, c.k[:0], c.v[:0], i32([0, 0]), c.pos0, 4, c.bt, c.pool, z, ws)
