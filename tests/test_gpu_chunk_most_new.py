"""Chunk attention (optr_chunk_attention) under a bound on a sequence's new tokens far above what any has."""
import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_chunk import PAPER, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("most", [1 << 20, 1 << 29, (1 << 29) + 1, 1 << 30, (1 << 30) + 1, (1 << 31) - 1])
@pytest.mark.parametrize("opts", [dict(), PAPER])
def test_large_bounds(most, opts):
    c = Case([64, 3, 100], [9000, 70, 0], seed=82, **opts)
    want = c.run().clone()
    got = c.run(max_new=most, out=torch.full_like(want, 7.0))
    assert torch.equal(got, want)
    assert optr.optr_device_error(c.p) == 0
