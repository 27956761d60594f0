"""Chunk attention with offsets that fall: the sequences that are in order keep
their rows, rows of no sequence are zero; tolerances as in test_gpu_chunk."""
import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_chunk import Case, check, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("past", [40, 3000])
@pytest.mark.parametrize("size", [1, 30])
@pytest.mark.parametrize("cu,good", [
    ([0, 20, 3, 9], [2]),     # past the end, back, then 3 .. 8
    ([0, 9, 4, 4], [0]),      # back to 4 at the end
    ([0, 5, 2, 12], [0]),     # 2 .. 11 would be too many
    ([0, 3, -7, 9], [0]),
    ([4, 9, 0, 4], [0, 2]),   # in another order
])
def test_falling_offsets(cu, good, size, past):
    n = 9 * size
    cu = [x * size for x in cu]
    lens = [b - a for a, b in zip(cu, cu[1:])]
    c = Case([3 * size] * 3, [past, past + 7, past // 2], seed=60)
    got = c.run(cu=i32(cu), max_new=9 * size).clone()
    assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_CU_NEW
    owned = torch.zeros(n, dtype=torch.bool, device="cuda")
    for b in good:
        one = Case([3 * size] * 3, [past, past + 7, past // 2], seed=60)
        r0, r1 = cu[b], cu[b + 1]
        one.cu, one.new = i32([r0 if x <= b else r1 for x in range(4)]), [lens[b] if x == b else 0 for x in range(3)]
        check(got[r0:r1], one.reference()[r0:r1])
        owned[r0:r1] = True
    assert not got[~owned].any()
