"""Attention weights (optr_kv_score) under a bound on a sequence's new tokens far above what any has: a server that
knows no better passes the largest, and pays for the tokens that there are."""
import time

import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_chunk import PAPER
from test_gpu_score import Score

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("most", [1 << 20, (1 << 29) + 1, 1 << 30, (1 << 30) + 4, (1 << 31) - 1])
@pytest.mark.parametrize("new", [[1], [30, 2], [70, 0, 9]])
@pytest.mark.parametrize("opts", [dict(), PAPER])
def test_large_bounds(most, new, opts):
    c = Score(new, [300, 90, 5][:len(new)], seed=81, **opts)
    begin = time.monotonic()
    got = c.run(max_new=most)
    torch.cuda.synchronize()
    assert time.monotonic() - begin < 5.0
    c.check(got)
    # (more than 64 tokens' columns make no difference to a block)
    assert torch.equal(got, c.run(max_new=sum(new) + 64))
    assert optr.optr_device_error(c.p) == 0
