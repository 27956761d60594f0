"""Inputs of draft verification that it has to report, or to take as exactly as
any other; exact comparisons, as in test_gpu_verify."""
import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_verify import Case, i32, p  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("probs", [True, False])
@pytest.mark.parametrize("bad", [-1, 500, 2 ** 31 - 1, -2 ** 31])
@pytest.mark.parametrize("first,at", [(0, 1), (0, 32), (2, 39), (31, 64), (40, 45)])
def test_bad_tokens_after_a_rejection_are_flagged(p, first, at, bad, probs):  # noqa: F811
    """Whatever the random numbers leave of the sequence."""
    c = Case([3, 70, 2], 500, probs=probs, seed=20)
    c.u.zero_()
    c.tp[4 + first, c.x[3 + first].long()] = 0  # draft `first` of sequence 1 is rejected
    want = c.run(p)
    assert want[0][1] == first and optr.optr_device_error(p) == 0
    c.x[3 + at] = bad
    assert c.run(p) == want
    assert optr.optr_device_error(p) == optr.OPTR_DEVERR_TOKEN


@pytest.mark.parametrize("cu,rows", [([2, 5, 9], (2, 11)), ([0, 5, 7], (0, 9)), ([1, 1, 1], (1, 3))])
def test_offsets_that_leave_drafts_out_are_flagged(p, cu, rows):  # noqa: F811
    """Offsets that do not begin at 0 or end at n_draft: each sequence has its
    drafts all the same, rows of none stay as they were."""
    c = Case([5, 4], 700, seed=21)
    c.u.zero_()
    acc, tok = c.run(p, cu=i32(cu))
    assert optr.optr_device_error(p) == optr.OPTR_DEVERR_CU_NEW
    lo, hi = rows
    assert tok[:lo] == [99] * lo and tok[hi:] == [99] * (11 - hi)
    assert all(0 <= t < 700 or t == -1 for t in tok[lo:hi])
    c.lens = [b - a for a, b in zip(cu, cu[1:])]
    c.tp, c.dp, c.x, c.u = c.tp[lo:hi], c.dp[cu[0]:cu[-1]], c.x[cu[0]:cu[-1]], c.u[cu[0]:cu[-1]]
    assert (acc, tok[lo:hi]) == c.plain()


@pytest.mark.parametrize("vocab", [4096, 4001])
def test_a_subnormal_noise_value_hides_no_larger_quotient(p, vocab):  # noqa: F811
    c = Case([0], vocab, seed=22)
    c.tp.fill_(1e-6)
    c.e.fill_(1.0)
    c.tp[0, 40], c.e[0, 40] = 1e-10, 1e-39  # 1e29, where 1 / 1e-39 is past float32
    c.tp[0, 41], c.e[0, 41] = 0.5, 1e-30    # 5e29
    assert c.run(p) == c.plain() == ([0], [41])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [5, 128, 1000, 4096, 50257])
@pytest.mark.parametrize("low", [-40.0, -37.0, 20.0])
def test_noise_over_the_whole_range(p, vocab, low, dtype):  # noqa: F811
    c = Case([2, 0, 3], vocab, dtype, seed=23)
    g = torch.Generator(device="cuda").manual_seed(24)
    draw = lambda *s: torch.rand(*s, device="cuda", generator=g)
    c.tp = (c.tp.float() * 10 ** (-30 * draw(8, vocab))).to(dtype)
    for seed in range(4):
        c.e = (10 ** (low + (38.4 - low) * draw(3, vocab).double())).float().clamp(1e-40, 3e38)
        c.u = draw(5)
        assert c.run(p) == c.plain()
