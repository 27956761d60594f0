"""Verification of drafted tokens (optr_verify_drafts) against a plain statement.

Acceptance and the candidates are single float32 operations (a product, a
difference, a quotient, each rounded to nearest), so the plain form computes
the same numbers and every output is compared exactly; a test in 64 bits checks
that the choice is the true maximum up to those roundings, 3 * 2^-24 of it, and
one draws many times: the token's frequencies are the target's, within 5
standard deviations."""
import pytest
import torch

from paper_2608_02691_gb300 import optr, synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def p():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)
    R_k, R_v = synth.rotations(1, 0)
    return optr.optr_params_create(R_k, R_v, torch.zeros(1, 128), 4)


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


class Case:
    def __init__(self, lens, vocab, dtype=torch.float32, probs=True, seed=0, sharp=3.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        B, n = len(lens), sum(lens)
        rows = lambda m: torch.softmax(sharp * torch.randn(m, vocab, device="cuda", generator=g), 1)
        self.lens, self.vocab = lens, vocab
        self.cu = i32([0] + list(torch.tensor(lens).cumsum(0).tolist()))
        self.tp = rows(n + B).to(dtype)
        # drafts near the target: the row after the same prefix, mixed
        at = torch.cat([torch.arange(m) + sum(lens[:b]) + b for b, m in enumerate(lens)]).cuda()
        q = 0.5 * self.tp[at].float() + 0.5 * rows(n)
        self.dp = q.to(dtype) if probs else None
        self.x = torch.multinomial(q, 1, generator=g)[:, 0].int() if n else i32([])
        self.u = torch.rand(n, device="cuda", generator=g)
        self.e = torch.empty(B, vocab, device="cuda").exponential_(generator=g)

    def run(self, p, **over):
        a = dict(tp=self.tp, dp=self.dp, x=self.x, u=self.u, e=self.e, cu=self.cu)
        a.update(over)
        B = self.cu.numel() - 1
        acc, tok = torch.full((B,), 99, dtype=torch.int32, device="cuda"), \
            torch.full((self.x.numel() + B,), 99, dtype=torch.int32, device="cuda")
        optr.optr_verify_drafts(p, a["tp"], a["dp"], a["x"], a["u"], a["e"], a["cu"], acc, tok)
        return acc.tolist(), tok.tolist()

    def plain(self):
        acc, tok, r0 = [], [], 0
        for b, n in enumerate(self.lens):
            a = 0
            while a < n:
                x, t = int(self.x[r0 + a]), r0 + b + a
                if not 0 <= x < self.vocab:
                    break
                q = self.dp[r0 + a, x].float() if self.dp is not None else torch.ones((), device="cuda")
                if not bool(self.u[r0 + a] * q < self.tp[t, x].float()):
                    break
                a += 1
            row = self.tp[r0 + b + a].float()
            r = row.clone()
            if a < n:
                if self.dp is not None:
                    r = (row - self.dp[r0 + a].float()).clamp(min=0)
                elif 0 <= int(self.x[r0 + a]) < self.vocab:
                    r[int(self.x[r0 + a])] = 0
                if not r.any():
                    r = row
            c = r / self.e[b]
            t = int((c == c.max()).nonzero()[0, 0])  # the first of equals
            acc.append(a)
            tok += self.x[r0:r0 + a].tolist() + [t] + [-1] * (n - a)
            r0 += n
        return acc, tok


LENS = [[0], [1], [4], [0, 3, 0, 8, 1], [33, 64, 65, 0], [100], [2] * 300]


@pytest.mark.parametrize("lens", LENS, ids=lambda l: f"{len(l)}x{max(l)}")
@pytest.mark.parametrize("vocab", [1, 2, 5, 100, 1001, 4096, 50257])
@pytest.mark.parametrize("dtype,probs", [(torch.float32, True), (torch.bfloat16, True), (torch.float32, False),
                                         (torch.bfloat16, False)])
def test_plain(p, lens, vocab, dtype, probs):
    if sum(lens) * vocab > 2 ** 25:
        vocab = 1024 + vocab % 64
    c = Case(lens, vocab, dtype, probs, seed=vocab + len(lens))
    assert c.run(p) == c.plain()
    assert optr.optr_device_error(p) == 0


def test_every_count_of_accepted_drafts(p):
    lens = [5] * 6 + [40] * 3
    c = Case(lens, 777, seed=1)
    c.u.zero_()
    stop = [0, 1, 2, 3, 4, 5, 31, 32, 40]
    r0 = 0
    for b, (n, s) in enumerate(zip(lens, stop)):
        if s < n:  # a token the target never gives
            c.tp[r0 + b + s, c.x[r0 + s].long()] = 0
        r0 += n
    got = c.run(p)
    assert got[0] == stop and got == c.plain()


def test_64_bits(p):
    c = Case([6] * 50, 3001, seed=2)
    acc, tok = c.run(p)
    for b in range(50):
        t = 7 * b + acc[b]
        r = c.tp[t].double()
        if acc[b] < 6:
            r = (r - c.dp[6 * b + acc[b]].double()).clamp(min=0)
        w = r / c.e[b].double()
        assert w[tok[t]] >= w.max() * (1 - 3 * 2.0 ** -24)


def test_residual_zero_everywhere_draws_from_the_target(p):
    for probs in (True, False):
        c = Case([2, 2], 600, probs=probs, seed=3)
        c.u.fill_(0.9999)
        if probs:
            c.dp = c.tp[[0, 1, 3, 4]].clone() * 2  # q above p throughout: rejected, no residual
        else:
            c.tp[[0, 3]] = 0
            c.tp[0, c.x[0].long()] = c.tp[3, c.x[2].long()] = 0.5  # p is all on the rejected draft
        acc, tok = c.run(p)
        assert acc == [0, 0] and (acc, tok) == c.plain()
        if not probs:
            assert tok[0] == int(c.x[0]) and tok[3] == int(c.x[2])


@pytest.mark.parametrize("vocab", [4096, 40001])
def test_the_lowest_of_equal_candidates_wins(p, vocab):
    c = Case([0, 0], vocab, seed=4)
    c.tp.fill_(0.25)
    c.e.fill_(1.0)
    assert c.run(p) == ([0, 0], [0, 0])
    first = (vocab // 2, vocab - 1)
    for b, f in enumerate(first):
        c.e[b, :f] = 2.0
    assert c.run(p)[1] == list(first)
    c.tp.fill_(-0.0)  # no mass at all, of either sign: the first token
    c.tp[:, 0] = 0.0
    assert c.run(p)[1] == [0, 0]


def test_frequencies_are_the_targets(p):
    n, vocab = 40000, 4
    c = Case([1] * n, vocab, seed=5)
    target = torch.tensor([0.4, 0.3, 0.2, 0.1], device="cuda")
    draft = torch.tensor([0.1, 0.2, 0.3, 0.4], device="cuda")
    c.tp[:] = target
    c.dp[:] = draft
    g = torch.Generator(device="cuda").manual_seed(6)
    c.x = torch.multinomial(draft.expand(n, 4), 1, generator=g)[:, 0].int()
    tok = torch.tensor(c.run(p)[1])[::2]  # the first token of each, accepted or drawn
    f = torch.bincount(tok, minlength=4).double() / n
    t = target.double().cpu()
    assert ((f - t).abs() <= 5 * (t * (1 - t) / n).sqrt()).all(), f


def test_unaligned_rows(p):
    c = Case([3, 1], 4096, seed=7)
    want = c.run(p)
    shift = lambda x: torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view_as(x).copy_(x)
    assert c.run(p, tp=shift(c.tp), dp=shift(c.dp), e=shift(c.e)) == want
    assert c.run(p, dp=shift(c.dp)) == want


def test_bad_tokens_are_rejected(p):
    for bad in (-1, 500, 2 ** 31 - 1, -2 ** 31):
        for probs in (True, False):
            c = Case([3, 3], 500, probs=probs, seed=8)
            c.u.zero_()
            c.x[1] = bad
            got = c.run(p)
            assert got == c.plain() and got[0] == [1, 3]
            assert optr.optr_device_error(p) == optr.OPTR_DEVERR_TOKEN


def test_bad_offsets_leave_other_sequences(p):
    c = Case([3, 3, 3], 500, seed=9)
    acc, tok = c.run(p)
    got = c.run(p, cu=i32([0, 3, 20, 9]))
    assert got[0] == [acc[0], -1, -1] and got[1][:4] == tok[:4] and got[1][4:] == [99] * 8
    assert optr.optr_device_error(p) == optr.OPTR_DEVERR_CU_NEW
    got = c.run(p, cu=i32([-1, 3, 6, 9]))
    assert got[0] == [-1] + acc[1:] and got[1][4:] == tok[4:]
    assert optr.optr_device_error(p) == optr.OPTR_DEVERR_CU_NEW


def test_other_stream_and_graph(p):
    c = Case([4, 2], 2048, seed=10)
    want = c.plain()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        assert c.run(p) == want
    acc, tok = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        optr.optr_verify_drafts(p, c.tp, c.dp, c.x, c.u, c.e, c.cu, acc, tok)
    for k in range(2):
        g.replay()
        assert (acc.tolist(), tok.tolist()) == c.plain()
        c.e.copy_(c.e.flip(1))
        c.u.copy_(1 - c.u)


def test_refusals(p):
    c = Case([2, 1], 50, seed=11)
    for bad in (dict(tp=c.tp.half()), dict(tp=c.tp.cpu()), dict(tp=c.tp[:4]), dict(dp=c.dp.bfloat16()),
                dict(dp=c.dp[:, :49]), dict(x=c.x.long()), dict(u=c.u[:2]), dict(e=c.e.double()),
                dict(e=c.e[:1]), dict(cu=c.cu.long()), dict(tp=c.tp[:, ::2])):
        with pytest.raises(ValueError):
            c.run(p, **bad)
