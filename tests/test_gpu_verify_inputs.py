"""Inputs of draft verification that it has to report, or to take as exactly as
any other; exact comparisons, as in test_gpu_verify."""
import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_verify import Case, p  # noqa: F401

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
