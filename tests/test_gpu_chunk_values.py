"""Chunk attention over caches whose values are small or large; tolerances as in
test_gpu_chunk."""
import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_chunk import Case, check, cu_of, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("size", [1e-5, 1e-3, 4096.0])
@pytest.mark.parametrize("new", [3, 70])
def test_value_sizes(new, size):
    """Over thousands of keys the output is far smaller than the values."""
    c = Case([new], [4000], seed=30)
    n = c.past[0]
    k, v = torch.randn(n, c.h, 128, device="cuda"), torch.randn(n, c.h, 128, device="cuda") * size
    optr.optr_kv_append(c.p, (k + c.mu.float()).bfloat16(), v.bfloat16(), cu_of([n]), i32([0]), c.bt, c.pool)
    c.v = (c.v.float() * (size / 64)).bfloat16()  # the chunk's own do not outweigh them
    check(c.run(), c.reference())
    assert optr.optr_device_error(c.p) == 0
