"""Attention weights (optr_kv_score) in each form that its work takes, against the formula in 64 bits with
test_gpu_score's cases and tolerance: a cluster a (sequence, KV head) with its logits in shared memory or in
the workspace, one even line of pages, and tiles on the tensor core; blocks whose queries differ in size."""
import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_chunk import PAPER, i32
from test_gpu_score import Score

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("h,new,past", [
    (1, [1], [5000]),                                   # clusters of 8
    (2, [1] * 10, list(range(0, 2000, 200))),           # 20: of 4
    (8, [1] * 9, [3, 900, 17, 0, 2500, 1, 15, 16, 33]),  # 72: of 2
    (8, [1] * 12, [100 * i for i in range(12)]),        # 96: none
    (8, [1, 0] * 10, [40 * i for i in range(20)]),      # 160: two rounds, half of it empty
    (4, [4, 1, 3, 2], [1500, 0, 31, 700]),
])
@pytest.mark.parametrize("opts", [dict(), dict(group=128), PAPER])
def test_logits_in_shared_memory(h, new, past, opts):
    c = Score(new, past, h_kv=h, seed=51, **opts)
    c.check(c.run())
    assert optr.optr_device_error(c.p) == 0


@pytest.mark.parametrize("h,new,past", [
    (8, [4, 1, 3, 2], [9100, 20, 0, 8200]),             # clusters of 4
    (8, [4] + [1] * 13, [2600] + [300] * 13),           # none
])
@pytest.mark.parametrize("opts", [dict(), dict(group=128), dict(sink=16, recent=100)])
def test_logits_in_the_workspace(h, new, past, opts):
    c = Score(new, past, h_kv=h, seed=52, **opts)
    c.check(c.run())
    assert optr.optr_device_error(c.p) == 0


@pytest.mark.parametrize("new,past", [([4], [30000]), ([2, 4, 0, 1], [25001, 7, 60, 333])])
@pytest.mark.parametrize("opts", [dict(), PAPER])
def test_an_even_line_of_pages(new, past, opts):
    c = Score(new, past, seed=53, **opts)
    c.check(c.run())
    assert optr.optr_device_error(c.p) == 0


@pytest.mark.parametrize("new", [[5], [8], [9], [31, 1], [32], [33], [64, 63], [65], [128, 3]])
@pytest.mark.parametrize("opts", [dict(group=128), dict(PAPER, fold=True), dict(sink=0, recent=33)])
def test_tiles(new, opts):
    c = Score(new, [700, 129][:len(new)], seed=54, **opts)
    c.check(c.run())
    assert optr.optr_device_error(c.p) == 0


@pytest.mark.parametrize("new", [[4], [60]])
@pytest.mark.parametrize("opts", [dict(), dict(group=128), PAPER])
def test_queries_of_very_different_sizes(new, opts):
    """The tensor core's form has one power of two for a block's queries.  An element is known to 2^-38 of
    the block's largest, so a logit of any row to 2^-38 |k| / sqrt(128) times 128 of those: under 2^-23 here."""
    c = Score(new, [600], seed=55, **opts)
    size = torch.tensor([1.0, 1e-3, 0.0, 1e-6, 0.3], device="cuda")[torch.arange(new[0], device="cuda") % 5]
    c.q.mul_(size[:, None, None])
    c.check(c.run())


@pytest.mark.parametrize("new", [[2, 3], [40, 12]])
def test_equal_keys_give_equal_weights(new):
    """Constant keys (scale 0 in the record): every weight is 1 / n."""
    c = Score(new, [500, 80], seed=56, group=128)
    k = torch.zeros(sum(c.n), c.h, 128, dtype=torch.bfloat16, device="cuda")
    optr.optr_kv_append(c.p, k, k, i32([0, c.n[0], sum(c.n)]), i32([0, 0]), c.bt, c.pool)
    c.check(c.run())


def test_the_workspace_holds_every_form():
    """Bytes behind what the size says stay as they are, in each form."""
    for h, new, past, opts in ((2, [1], [500], dict()), (8, [4, 1, 3, 2], [9100, 20, 0, 8200], dict()),
                               (2, [4], [30000], dict()), (2, [70], [300], PAPER)):
        c = Score(new, past, h_kv=h, seed=57, **opts)
        n = optr.optr_kv_score_workspace_size(c.p, sum(new), c.B, c.max_new, c.bt.shape[1])
        ws = torch.full((n + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
        args = (c.p, c.q, c.cu, c.pos0, c.max_new, c.bt, c.pool)
        out = c.score.clone()
        if c.win is None:
            optr.optr_kv_score(*args, out, ws[:n])
        else:
            optr.optr_kv_score_win(*args, c.win, c.slots, out, ws[:n])
        c.check(out)
        assert (ws[n:] == 0x5A).all()


@pytest.mark.parametrize("new", [[4], [6], [40]])
@pytest.mark.parametrize("size", [-6.4, 6.4, -40.0, 40.0])
@pytest.mark.parametrize("opts", [dict(), dict(group=128), dict(sink=16, recent=100)])
def test_all_logits_alike_and_far_from_zero(new, size, opts):
    """Every key the same row of +-1 in the rotated basis, every query `size` times it: log2 logits of 16.3
    size, 105 at 6.4 and 653 at 40, above and below zero, as large as sums of magnitudes allow.  All weights
    are 1 / n: keys of equal bits have equal logits, so only the normaliser's sum counts; window keys are
    bf16 of the same row, whose logit differs by 2^-8 of the rest, so only their sums are compared there.
    A logit and a normaliser of 653 are rounded to 2^-15 each, a weight by ln 2 of their sum: 4.3e-5; its
    sums and exponentials add less than 1e-5 to that, and 1e-4 is allowed."""
    c = Score(new, [3000], h_kv=1, seed=58, **opts)
    g = torch.Generator(device="cuda").manual_seed(59)
    row = torch.randn(128, device="cuda", generator=g).sign().double()
    n = c.n[0]
    k = (c.R_k[0] @ row + c.mu[0]).bfloat16().view(1, 1, 128).expand(n, 1, 128).contiguous()
    args = (c.p, k, k, i32([0, n]), i32([0]), c.bt, c.pool)
    if c.win is None:
        optr.optr_kv_append(*args)
    else:
        optr.optr_kv_append_win(*args, c.win, c.slots)
    c.q.copy_((size * (c.R_k[0] @ row)).bfloat16().expand_as(c.q))
    c.score.zero_()
    got = c.run().double()[0, 0, :n]
    if c.win is None:
        want = torch.zeros(n, dtype=torch.float64, device="cuda")
        for i in range(new[0]):
            seen = c.past[0] + i + 1
            want[:seen] += 4 / seen
        assert ((got - want).abs() <= 1e-4 * want).all()
    assert abs(float(got.sum()) - 4 * new[0]) <= 1e-4 * 4 * new[0] and torch.isfinite(got).all()
