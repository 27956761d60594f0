"""The operators as a server uses them, one after another.

Trees: a step's tree attends (optr_tree_attention), is verified (optr_verify_tree), and the
accepted rows are written (optr_kv_append).  The accepted way is a chunk of its own: the
chunk attention over it gives the tree's rows, to both kernels' tolerance (test_gpu_chunk's),
and after the write a decode at the last accepted row is the formula's over the cache.

Eviction: decode steps add their weights up (optr_kv_score), the choice (optr_evict_select)
follows the sums, the move (optr_kv_compact) keeps the records' bits, and decodes over what
stays, and over tokens written behind it, are the formula's in 64 bits over the kept positions."""
import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_chunk import PAPER, Case, check, cu_of, i32
from test_gpu_tree import Tree, some

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


def append(c, k, v, lens, pos0):
    args = (c.p, k, v, cu_of(lens), i32(pos0), c.bt, c.pool)
    if c.win is None:
        optr.optr_kv_append(*args)
    else:
        optr.optr_kv_append_win(*args, c.win, c.slots)


def decode(c, q, lens):
    out = torch.empty(c.B, 4 * c.h, 128, device="cuda")
    ws = optr.new_workspace(c.p, c.B, c.bt.shape[1])
    args = (c.p, q, c.bt, i32(lens), c.pool)
    if c.win is None:
        optr.optr_decode_attention(*args, out, ws)
    else:
        optr.optr_decode_attention_win(*args, c.win, c.slots, out, ws)
    return out


@pytest.mark.parametrize("opts", [dict(), dict(sink=16, recent=100), PAPER])
def test_a_step_of_drafted_trees(opts):
    past = [700, 33, 1500]
    c = Tree([24, 9, 40], past, shape=some, spare=3, seed=21, **opts)
    tree = c.run().clone()
    g = torch.Generator(device="cuda").manual_seed(22)
    n, V, cu = c.q.shape[0], 501, c.cu.tolist()
    z = 2 * torch.randn(n, V, device="cuda", generator=g)
    tp, dp = torch.softmax(z, 1), torch.softmax(z + 0.3 * torch.randn(n, V, device="cuda", generator=g), 1)
    up = torch.tensor([cu[b] + max(x, 0) for b, t in enumerate(c.trees) for x in t], device="cuda")
    tokens = torch.multinomial(dp[up], 1, generator=g)[:, 0].int()
    u = torch.rand(n, device="cuda", generator=g)
    e = torch.empty(c.B, V, device="cuda").exponential_(generator=g)
    acc = torch.empty(c.B, dtype=torch.int32, device="cuda")
    path, nxt = (torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(2))
    optr.optr_verify_tree(c.p, tp, dp, tokens, c.parent, u, e, c.cu, acc, path, nxt)
    acc, path = acc.tolist(), path.tolist()
    ways = [path[cu[b]:cu[b] + acc[b] + 1] for b in range(c.B)]
    assert sum(acc) > 3  # (drafts agree with the target often enough)
    for b, way in enumerate(ways):  # a way goes from the root down
        assert way[0] == cu[b] and path[cu[b] + acc[b] + 1:cu[b + 1]] == [-1] * (cu[b + 1] - cu[b] - acc[b] - 1)
        for x, y in zip(way, way[1:]):
            assert cu[b] + c.trees[b][y - cu[b]] == x
    lens, rows = [len(w) for w in ways], torch.tensor(sum(ways, []), device="cuda")
    q, k, v = (x[rows].contiguous() for x in (c.q, c.k, c.v))
    chunk = Case.run(c, q=q, k=k, v=v, cu=cu_of(lens), max_new=max(lens), out=torch.empty_like(q))
    check(chunk, tree[rows].double())
    append(c, k, v, lens, past)
    last = torch.tensor(lens, device="cuda").cumsum(0) - 1
    now = [a + b for a, b in zip(past, lens)]
    out = decode(c, q[last].contiguous(), now)
    check(out, Chat.attend(c, q[last], now)[0])
    assert optr.optr_device_error(c.p) == 0


class Chat(Case):
    """A cache of `past` tokens with room for more, and what a plain account of it holds: the kept
    positions' keys (centered, model basis) and values in 64 bits."""

    def held(self, b, h, n):
        k, v = self.rows(b, h, 0, n, 0) @ self.R_k[h].T, self.rows(b, h, 0, n, 1) @ self.R_v[h].T
        if self.win is not None:
            s = torch.arange(n, device="cuda")
            s = s[(s < self.sink) | (s >= n - self.recent)]
            row = torch.where(s < self.sink, s, self.sink + (s - self.sink) % max(1, self.recent))
            w = self.win[int(self.slots[b]), h]
            k[s], v[s] = w[0, row].double() - self.mu[h], w[1, row].double()
        return k, v

    def attend(self, q, lens):
        """The formula for one query a sequence: outputs, and weights by KV head and position."""
        out = torch.empty(self.B, 4 * self.h, 128, dtype=torch.float64, device="cuda")
        weights = torch.zeros(self.B, self.h, max(lens), dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            for h in range(self.h):
                k, v = Chat.held(self, b, h, n)
                p = torch.softmax(q[b, 4 * h:4 * h + 4].double() @ k.T / 128 ** 0.5, 1)
                out[b, 4 * h:4 * h + 4] = p @ v
                weights[b, h, :n] = p.sum(0)
        return out, weights


@pytest.mark.parametrize("opts", [dict(), dict(group=128), dict(sink=16, recent=100), PAPER])
def test_a_chat_over_its_budget(opts):
    past, steps, keep = [900, 1300, 420], 3, [500, 400, 600]
    c = Chat([0] * 3, past, spare=2, seed=31, **opts)
    g = torch.Generator(device="cuda").manual_seed(32)
    score = torch.zeros(c.B, c.h, 16 * c.bt.shape[1], device="cuda")
    total = torch.zeros_like(score, dtype=torch.float64)
    one = cu_of([1] * c.B)
    ws = optr.new_score_workspace(c.p, c.B, c.B, 1, c.bt.shape[1])
    lens = list(past)

    def step():
        q = (1.5 * torch.randn(c.B, 4 * c.h, 128, device="cuda", generator=g)).bfloat16()
        k = (torch.randn(c.B, c.h, 128, device="cuda", generator=g) + c.mu.float()).bfloat16()
        v = torch.randn(c.B, c.h, 128, device="cuda", generator=g).bfloat16()
        append(c, k, v, [1] * c.B, lens)
        args = (c.p, q, one, i32(lens), 1, c.bt, c.pool)
        if c.win is None:
            optr.optr_kv_score(*args, score, ws)
        else:
            optr.optr_kv_score_win(*args, c.win, c.slots, score, ws)
        lens[:] = [n + 1 for n in lens]
        want, weights = c.attend(q, lens)
        check(decode(c, q, lens), want)
        return weights

    for _ in range(steps):
        w = step()
        total[:, :, :w.shape[2]] += w
    # a weight to 8e-6 (1 + 1.5) of it (test_gpu_score's bound), a rounding of the sum a step
    assert ((score.double() - total).abs() <= (2e-5 + steps * 2.0 ** -24) * total).all()
    first, last = max(4, c.sink), max(8, c.recent)
    most = max(min(n, max(k, min(n, first + last))) for n, k in zip(lens, keep))
    kept = torch.full((c.B, c.h, most), -1, dtype=torch.int32, device="cuda")
    counts = torch.empty(c.B, dtype=torch.int32, device="cuda")
    optr.optr_evict_select(c.p, score, i32(lens), i32(keep), first, last, kept, counts)
    m = counts.tolist()
    assert m == [min(n, max(k, first + last)) for n, k in zip(lens, keep)]
    before, sums, old = {}, score.clone(), list(lens)
    for b in range(c.B):
        for h in range(c.h):
            before[b, h] = [c.rows(b, h, 0, old[b], kind) for kind in (0, 1)]
            chosen = kept[b, h, :m[b]].long()
            others = torch.ones(old[b], dtype=torch.bool, device="cuda")
            others[chosen] = False
            middle = chosen[(chosen >= first) & (chosen < old[b] - last)]
            if others.any() and middle.numel():  # no position that goes has more than one that stays
                assert sums[b, h, :old[b]][others].max() <= sums[b, h][middle].min()
    if c.win is None:
        optr.optr_kv_compact(c.p, kept, counts, i32(lens), c.bt, c.pool, score)
    else:
        optr.optr_kv_compact_win(c.p, kept, counts, i32(lens), c.bt, c.pool, c.win, c.slots, score)
    lens[:] = m
    for b in range(c.B):
        for h in range(c.h):
            chosen = kept[b, h, :m[b]].long()
            for kind in (0, 1):
                assert torch.equal(c.rows(b, h, 0, m[b], kind), before[b, h][kind][chosen])
            assert torch.equal(score[b, h, :m[b]], sums[b, h][chosen])
            assert not score[b, h, m[b]:old[b]].any()
    total = score.double()
    for _ in range(steps):  # the chat goes on behind what stayed
        w = step()
        total[:, :, :w.shape[2]] += w
    assert ((score.double() - total).abs() <= (2e-5 + (steps + 1) * 2.0 ** -24) * total).all()
    assert optr.optr_device_error(c.p) == 0


def test_a_decode_step_with_its_account_in_a_graph():
    """A decode step, its weights and the choice, captured once and replayed on new queries: what the
    calls give one by one."""
    c = Chat([0] * 2, [300, 1000], spare=2, seed=41, **PAPER)
    lens = [300, 1000]
    q = torch.randn(2, 8, 128, device="cuda").bfloat16()
    n_lens, pos0, keep = i32(lens), i32([n - 1 for n in lens]), i32([330, 400])
    out, score = torch.empty(2, 8, 128, device="cuda"), torch.zeros(2, 2, 16 * c.bt.shape[1], device="cuda")
    kept, counts = torch.full((2, 2, 400), -1, dtype=torch.int32, device="cuda"), i32([0, 0])
    ws = optr.new_workspace(c.p, 2, c.bt.shape[1])
    sws = optr.new_score_workspace(c.p, 2, 2, 1, c.bt.shape[1])
    cu = cu_of([1, 1])

    def step():
        optr.optr_decode_attention_win(c.p, q, c.bt, n_lens, c.pool, c.win, c.slots, out, ws)
        optr.optr_kv_score_win(c.p, q, cu, pos0, 1, c.bt, c.pool, c.win, c.slots, score, sws)
        optr.optr_evict_select(c.p, score, n_lens, keep, 64, 256, kept, counts)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        q.copy_(torch.randn(q.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)))
        start = score.clone()
        graph.replay()
        got = [x.clone() for x in (out, score, kept, counts)]
        score.copy_(start)
        kept.fill_(-1)
        step()
        for x, y in zip(got, (out, score, kept, counts)):
            assert torch.equal(x, y)
    assert counts.tolist() == [300, 400]
