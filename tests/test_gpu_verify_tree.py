"""Verification of trees of drafts (optr_verify_tree) against a plain statement.

Acceptance, residuals and quotients are single float32 operations, so the plain form
computes the same numbers from the same masses S; a mass is a sum, which the plain form
takes in 64 bits and rounds to float32.  The kernel's own sum is within (r + 2) 2^-24 of
it, r terms a thread (131072 / 4096 and below): cases are drawn, and checked, so that
no decision lies within 2^-17 of its border.  Frequencies of many draws are the
target's, within 5 standard deviations."""
import random

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


def some(n, r):
    return [-1] + [r.randint((i - 1) // 3, i - 1) for i in range(1, n)]


def star(n, r):
    return [-1] + [0] * (n - 1)


def chain(n, r):
    return list(range(-1, n - 1))


class Case:
    def __init__(self, lens, vocab, dtype=torch.float32, probs=True, seed=0, shape=some, near=0.5, sharp=3.0,
                 repeat=True):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = random.Random(seed)
        B, n = len(lens), sum(lens)
        z = sharp * torch.randn(n, vocab, device="cuda", generator=g)
        self.lens, self.vocab, self.probs = lens, vocab, probs
        self.trees = [shape(m, r) if m else [] for m in lens]
        self.cu = i32([0] + list(torch.tensor(lens).cumsum(0).tolist()))
        self.tp = torch.softmax(z, 1).to(dtype)
        q = torch.softmax(z + near * torch.randn(n, vocab, device="cuda", generator=g), 1).to(dtype)
        self.dp = q if probs else None
        self.parent = i32(sum(self.trees, []))
        up = torch.tensor([c + max(x, 0) for c, t in zip(self.cu.tolist(), self.trees) for x in t], device="cuda")
        self.x = torch.multinomial(q[up].float(), 1, generator=g)[:, 0].int()
        if not probs and not repeat:
            self.x = (torch.arange(n, device="cuda") % vocab).int()
        self.u = torch.rand(n, device="cuda", generator=g)
        self.e = torch.empty(B, vocab, device="cuda").exponential_(generator=g).clamp_min(1e-20)

    def run(self, p, **over):
        a = dict(tp=self.tp, dp=self.dp, x=self.x, parent=self.parent, u=self.u, e=self.e, cu=self.cu)
        a.update(over)
        B, n = a["cu"].numel() - 1, a["x"].numel()
        acc = torch.full((B,), 99, dtype=torch.int32, device="cuda")
        path, nxt = (torch.full((n,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
        optr.optr_verify_tree(p, a["tp"], a["dp"], a["x"], a["parent"], a["u"], a["e"], a["cu"], acc, path, nxt)
        return acc.tolist(), path.tolist(), nxt.tolist()

    def plain(self):
        """The outputs, and how near the nearest decision was to its border (relative)."""
        acc, path, nxt, margin = [], [], [], 1.0
        cu, x, u = self.cu.tolist(), self.x.tolist(), self.u.cpu()
        tp, dp, e = self.tp.float().cpu(), None if self.dp is None else self.dp.float().cpu(), self.e.cpu()
        for b, m in enumerate(self.lens):
            if m == 0:
                acc.append(-1)
                continue
            c0, way = cu[b], [0]
            while True:
                r = way[-1]
                w, S, step = tp[c0 + r].clone(), torch.tensor(1.0), None
                for c in range(m):
                    if self.trees[b][c] != r:
                        continue
                    t = x[c0 + c]
                    if not 0 <= t < self.vocab:
                        continue
                    q = dp[c0 + r] if dp is not None else None
                    left = (u[c0 + c] * (q[t] if dp is not None else 1.0)) * S
                    if S is not None and (left != 0 or w[t] != 0):
                        # the mass alone is not exact, so the margin counts where there is one
                        exact = dp is None or float(S) == 1.0
                        if not exact:
                            margin = min(margin, abs(float(left - w[t])) / max(float(left), float(w[t])))
                    if left < w[t]:
                        step = c
                        break
                    if dp is not None:
                        w = (w - S * q).clamp_min(0)
                        S = w.double().sum().float()
                    else:
                        S = S - w[t]
                        w[t] = 0
                if step is None:
                    break
                way.append(step)
            ratio = w / e[b]
            if not bool((ratio > 0).any()):
                ratio = tp[c0 + r] / e[b]
            top = torch.cat((ratio, torch.zeros(1))).topk(2).values
            if dp is not None:
                margin = min(margin, float((top[0] - top[1]) / top[0]) if float(top[0]) else 1.0)
            a = len(way) - 1
            acc.append(a)
            path += [c0 + c for c in way] + [-1] * (m - 1 - a)
            nxt += [x[c0 + c] for c in way[1:]] + [int(ratio.argmax())] + [-1] * (m - 1 - a)
        return (acc, path, nxt), margin


CASES = [
    ([1], 1000, some), ([2], 7, some), ([8], 32000, some), ([24, 1, 5], 4001, some), ([64], 1003, some),
    ([33] * 20, 517, some), ([40], 2000, star), ([12, 12], 5000, chain), ([1024], 64, some), ([200], 50, star),
    ([24] * 16, 131072, some), ([7, 0, 3, 0], 130, some), ([5] * 300, 333, some), ([3], 1, some), ([9], 3, star),
]


@pytest.mark.parametrize("dtype,probs", [(torch.float32, True), (torch.float32, False), (torch.bfloat16, True),
                                         (torch.bfloat16, False)])
@pytest.mark.parametrize("lens,vocab,shape", CASES)
def test_matches_the_plain_form(p, lens, vocab, shape, dtype, probs):
    if vocab > 50000 and (dtype is torch.bfloat16 or not probs):
        pytest.skip("one of the large ones is enough")
    for seed in range(3):
        c = Case(lens, vocab, dtype, probs, seed, shape)
        want, margin = c.plain()
        if margin < 2.0 ** -17:
            continue  # (a decision within the sums' rounding; drawn, not chosen by outcome)
        assert c.run(p) == want
        assert optr.optr_device_error(p) == 0


@pytest.mark.parametrize("probs", [True, False])
def test_unaligned_rows_and_equal_calls(p, probs):
    c = Case([24, 9], 4004, probs=probs, seed=3)
    want = c.run(p)
    assert all(c.run(p) == want for _ in range(3))
    shift = lambda x: torch.empty(x.numel() + 1, device="cuda", dtype=x.dtype)[1:].view_as(x).copy_(x)
    assert c.run(p, tp=shift(c.tp)) == want and c.run(p, e=shift(c.e)) == want
    if probs:
        assert c.run(p, dp=shift(c.dp)) == want


def test_a_chain_accepts_what_the_drafts_verification_accepts(p):
    """Row r's only child is tried against the target alone, as optr_verify_drafts does; the target row
    after the last draft and the residual's draw are the same too."""
    for seed in range(20):
        c = Case([9], 400, seed=seed, shape=chain)
        acc, path, nxt = c.run(p)
        a2 = torch.zeros(1, dtype=torch.int32, device="cuda")
        t2 = torch.zeros(9, dtype=torch.int32, device="cuda")
        optr.optr_verify_drafts(p, c.tp, c.dp[:8].contiguous(), c.x[1:].contiguous(), c.u[1:].contiguous(), c.e,
                                i32([0, 8]), a2, t2)
        assert (acc, nxt) == (a2.tolist(), t2.tolist())


@pytest.mark.parametrize("probs", [True, False])
def test_the_text_has_the_targets_distribution(p, probs):
    """The token after the root of many small trees, drafts drawn anew: its frequencies."""
    V, B, kids = 6, 40000, 3
    g = torch.Generator(device="cuda").manual_seed(5)
    t = torch.softmax(torch.randn(V, device="cuda", generator=g), 0)
    q = torch.softmax(torch.randn(V, device="cuda", generator=g), 0)
    n = kids + 1
    tp = t.expand(B * n, V).contiguous()
    if probs:
        x = torch.multinomial(q.expand(B * n, V), 1, generator=g)[:, 0].int()
        dp = q.expand(B * n, V).contiguous()
    else:
        x, dp = torch.arange(n, device="cuda").repeat(B).int(), None
    parent = i32([-1] + [0] * kids).repeat(B)
    u = torch.rand(B * n, device="cuda", generator=g)
    e = torch.empty(B, V, device="cuda").exponential_(generator=g).clamp_min(1e-20)
    acc = torch.empty(B, dtype=torch.int32, device="cuda")
    path, nxt = (torch.empty(B * n, dtype=torch.int32, device="cuda") for _ in range(2))
    optr.optr_verify_tree(p, tp, dp, x, parent, u, e, (torch.arange(B + 1, device="cuda") * n).int(), acc, path, nxt)
    seen = torch.bincount(nxt.view(B, n)[:, 0].long(), minlength=V).double() / B
    assert ((seen - t).abs() <= 5 * (t * (1 - t) / B).sqrt()).all(), (seen, t)
    assert (acc > 0).double().mean() > 0.3


def test_many_children_wear_the_residual_out(p):
    """Equal target and draft: a first child of u < 1 is accepted; with u = 1 (out of the range that is
    asked for, but of any float's) all are rejected, the residual is zero and the target's row decides."""
    V, n = 100, 20
    g = torch.Generator(device="cuda").manual_seed(6)
    t = torch.softmax(torch.randn(1, V, device="cuda", generator=g), 1).expand(n, V).contiguous()
    x = torch.randint(0, V, (n,), device="cuda", generator=g).int()
    e = torch.empty(1, V, device="cuda").exponential_(generator=g).clamp_min(1e-20)
    c = Case([n], V, shape=star)
    acc, path, nxt = c.run(p, tp=t, dp=t, x=x, u=torch.full((n,), 0.999, device="cuda"), e=e)
    assert acc == [1] and path[:2] == [0, 1]
    acc, path, nxt = c.run(p, tp=t, dp=t, x=x, u=torch.ones(n, device="cuda"), e=e)
    assert acc == [0] and nxt[0] == int((t[0] / e[0]).argmax())


def test_tokens_and_parents_out_of_range(p):
    c = Case([6, 4], 50, seed=7, shape=lambda n, r: [-1, 0, 0, 1, 1, 2][:n])
    c.u.zero_()  # the first child in range is accepted
    c.tp.clamp_(min=1e-6)
    bad = c.x.clone()
    bad[1], bad[7] = 50, -1
    acc, path, nxt = c.run(p, x=bad)
    assert path[:2] == [0, 2] and path[6:8] == [6, 8]
    assert optr.optr_device_error(p) == optr.OPTR_DEVERR_TOKEN
    par = c.parent.clone()
    par[1], par[8], par[9] = 1, 77, -1
    acc, path, nxt = c.run(p, parent=par)
    assert path[:2] == [0, 2] and path[6:8] == [6, 7] and acc == [2, 1]
    assert optr.optr_device_error(p) == optr.OPTR_DEVERR_TREE


def test_offsets_out_of_range(p):
    c = Case([6, 4], 50, seed=8)
    whole = c.run(p)
    for cu in ([0, 6, 11], [0, -1, 10], [0, 11, 10]):
        acc, path, nxt = c.run(p, cu=i32(cu))
        assert -1 in acc
        assert optr.optr_device_error(p) == optr.OPTR_DEVERR_CU_NEW
    acc, path, nxt = c.run(p, cu=i32([0, 6, 6]))     # rows of no sequence: flagged, not written
    assert acc[0] == whole[0][0] and acc[1] == -1 and path[6:] == [99] * 4 and nxt[:6] == whole[2][:6]
    assert optr.optr_device_error(p) == optr.OPTR_DEVERR_CU_NEW
    n = optr.TREE_MAX_ROWS + 1
    big = Case([n], 3, seed=9)
    acc, path, nxt = big.run(p)
    assert acc == [-1] and path == [99] * n
    assert optr.optr_device_error(p) == optr.OPTR_DEVERR_CU_NEW


def test_refusals(p):
    c = Case([6], 50, seed=10)
    with pytest.raises(ValueError):
        c.run(p, tp=c.tp.half())
    with pytest.raises(ValueError):
        c.run(p, dp=c.dp[:5])
    with pytest.raises(ValueError):
        c.run(p, u=c.u[:5])
    with pytest.raises(ValueError):
        c.run(p, parent=c.parent.long())
    with pytest.raises(ValueError):
        c.run(p, e=c.e.expand(2, 50))


def test_a_captured_graph_takes_new_numbers(p):
    c = Case([24, 9], 4001, seed=11)
    acc = torch.empty(2, dtype=torch.int32, device="cuda")
    path, nxt = (torch.empty(33, dtype=torch.int32, device="cuda") for _ in range(2))
    call = lambda: optr.optr_verify_tree(p, c.tp, c.dp, c.x, c.parent, c.u, c.e, c.cu, acc, path, nxt)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for seed in (12, 13):
        d = Case([24, 9], 4001, seed=seed)
        c.u.copy_(d.u)
        c.e.copy_(d.e)
        g.replay()
        got = acc.tolist(), path.tolist(), nxt.tolist()
        assert got == c.run(p)
