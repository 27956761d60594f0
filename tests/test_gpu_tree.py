"""Attention of trees of drafted tokens (optr_tree_attention) against the formula in
64 bits, with test_gpu_chunk's cases and its tolerance (the arithmetic is the same, the
rows see fewer of each other); a chain against the chunk attention, bit for bit."""
import math
import random

import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_chunk import PAPER, Case, check, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


def chain(n):
    return list(range(-1, n - 1))


def star(n):
    return [-1] + [0] * (n - 1)


def alone(n):
    return [-1] * n


def some(n, seed=0):
    r = random.Random(seed)
    return [-1] + [r.randint(max(0, (i - 1) // 3), i - 1) for i in range(1, n)]


def forest(n):
    r = random.Random(n)
    return [-1 if r.random() < 0.2 else r.randrange(i) if i else -1 for i in range(n)]


class Tree(Case):
    def __init__(self, new, past, shape=some, **kw):
        super().__init__(new, past, **kw)
        self.trees = [shape(n)[:n] for n in new]
        self.parent = i32(sum(self.trees, []))

    def run(self, parent=None, **over):
        a = dict(q=self.q, k=self.k, v=self.v, cu=self.cu, pos0=self.pos0, bt=self.bt, out=self.out,
                 max_new=self.max_new, slots=self.slots)
        a.update(over)
        ws = optr.new_chunk_workspace(self.p, a["q"].shape[0], self.B, a["max_new"])
        ws.fill_(0xA5)
        args = (self.p, a["q"], a["k"], a["v"], self.parent if parent is None else parent, a["cu"], a["pos0"],
                a["max_new"], a["bt"], self.pool)
        if self.win is None:
            optr.optr_tree_attention(*args, a["out"], ws)
        else:
            optr.optr_tree_attention_win(*args, self.win, a["slots"], a["out"], ws)
        return a["out"]

    def reference(self, drop=()):
        """Row by row with what it sees: test_gpu_chunk's formula over a chunk of the row's ancestors and
        itself, whose last row it is."""
        out = torch.zeros_like(self.q, dtype=torch.float64)
        cu = self.cu.tolist()
        for b in range(self.B):
            n, r0, r1 = self.past[b], cu[b], cu[b + 1]
            if r1 == r0:
                continue
            seen = torch.zeros(r1 - r0, r1 - r0, dtype=torch.bool, device="cuda")
            for i, up in enumerate(self.trees[b]):
                if up >= 0:
                    seen[i] = seen[up]
                seen[i, i] = True
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
                m = k.shape[0] - (r1 - r0)
                for j in range(4):
                    l = self.q[r0:r1, 4 * h + j].double() @ k.T / 128 ** 0.5
                    l[:, m:].masked_fill_(~seen, -math.inf)
                    out[r0:r1, 4 * h + j] = torch.softmax(l, 1) @ v
        return out


SHAPES = [
    ([1], [0]), ([1], [1000]), ([2], [0]), ([8], [1024]), ([31], [300]), ([33], [300]), ([64], [0]),
    ([65], [0]), ([127], [100]), ([129], [7]), ([200], [4000]), ([2, 0, 5, 1], [100, 50, 0, 3000]),
    ([70, 1, 130], [40, 5000, 0]), ([5] * 40, list(range(0, 1200, 30))), ([300, 513], [1000, 2000]),
    ([1024], [50]),
]


@pytest.mark.parametrize("new,past", SHAPES)
@pytest.mark.parametrize("opts", [dict(), dict(sink=16, recent=100), PAPER])
def test_matches_the_formula(new, past, opts):
    c = Tree(new, past, **opts)
    check(c.run(), c.reference())
    assert optr.optr_device_error(c.p) == 0


@pytest.mark.parametrize("shape", [star, alone, forest, chain])
@pytest.mark.parametrize("opts", [dict(group=128), dict(sink=48, recent=0), dict(PAPER, fold=True)])
def test_shapes_of_trees(shape, opts):
    c = Tree([3, 40, 150, 1], [1000, 333, 0, 64], shape=shape, seed=1, **opts)
    check(c.run(), c.reference())
    assert optr.optr_device_error(c.p) == 0


@pytest.mark.parametrize("new,past", [([5, 200, 1], [100, 3000, 0]), ([1000], [0])])
@pytest.mark.parametrize("opts", [dict(), PAPER])
def test_a_chain_is_the_chunk_attention(new, past, opts):
    c = Tree(new, past, shape=chain, seed=2, **opts)
    want = Case.run(c).clone()
    assert torch.equal(c.run(out=torch.full_like(want, 7.0)), want)


def test_long_context_is_split_and_joined():
    c = Tree([9], [40000], h_kv=1, seed=3)
    check(c.run(), c.reference())


def test_siblings_do_not_see_each_other():
    """Another branch's keys and values change nothing, NaN included in what no row sees as a key
    (its value is 0 times a weight of 0 and has to be finite)."""
    c = Tree([6], [200], shape=lambda n: [-1, 0, 0, 1, 2, 4], seed=4)
    first = c.run().clone()
    k, v = c.k.clone(), c.v.clone()
    k[3], v[3] = 30.0, -5.0     # a leaf: row 3 alone sees it
    got = c.run(k=k, v=v)
    same = [0, 1, 2, 4, 5]
    assert torch.equal(got[same], first[same])
    assert not torch.equal(got[3], first[3])


def test_equal_calls_give_equal_bits():
    c = Tree([40, 3, 700], [3000, 9000, 64], seed=5)
    first = c.run().clone()
    for _ in range(3):
        assert torch.equal(c.run(), first)


def test_parents_out_of_range_are_flagged_and_count_as_none():
    c = Tree([4, 3], [100, 20], seed=6)
    bad = c.parent.clone()
    bad[1], bad[3], bad[6] = 1, -2, 1000000
    c.trees = [[-1, -1, c.trees[0][2], -1], [-1, c.trees[1][1], -1]]
    check(c.run(parent=bad), c.reference())
    assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_TREE
    assert optr.optr_device_error(c.p) == 0


def test_refusals():
    c = Tree([4], [100], seed=7)
    with pytest.raises(optr.OptrError) as e:
        c.run(max_new=optr.TREE_MAX_ROWS + 1)
    assert e.value.status == -3
    with pytest.raises(ValueError):
        c.run(parent=c.parent[:3])
    with pytest.raises(ValueError):
        c.run(parent=c.parent.long())
    with pytest.raises(optr.OptrError):  # windows need the _win call
        w = Tree([4], [100], seed=7, **PAPER)
        ws = optr.new_chunk_workspace(w.p, 4, 1, 4)
        optr.optr_tree_attention(w.p, w.q, w.k, w.v, w.parent, w.cu, w.pos0, 4, w.bt, w.pool, w.out, ws)
    # more rows than max_new: zero rows and a flag, as for a chunk
    assert (c.run(max_new=3) == 0).all()
    assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_CU_NEW


def test_another_stream_and_a_captured_graph():
    c = Tree([7, 40], [500, 90], seed=8)
    want = c.run().clone()
    out = torch.zeros_like(want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.run(out=out)
    s.synchronize()
    assert torch.equal(out, want)
    ws = optr.new_chunk_workspace(c.p, 47, 2, 40)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        optr.optr_tree_attention(c.p, c.q, c.k, c.v, c.parent, c.cu, c.pos0, 40, c.bt, c.pool, out, ws)
    for shape in (star, chain, some):  # the replay takes the parents of its time
        c.trees = [shape(7), shape(40)]
        c.parent.copy_(i32(sum(c.trees, [])))
        out.zero_()
        g.replay()
        check(out, c.reference())
