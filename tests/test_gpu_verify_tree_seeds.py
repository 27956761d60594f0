"""Tree verification (optr_verify_tree) against test_gpu_verify_tree's plain form: as many drawn cases of each
shape as are to be compared, whatever the seeds of those whose nearest decision lies within the sums' rounding."""
import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_verify_tree import Case, chain, p, some, star  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lens,vocab,shape", [
    ([40], 2000, star), ([200], 50, star), ([1024], 64, some), ([64], 1003, some), ([33] * 20, 517, some),
    ([9], 3, star), ([12, 12], 5000, chain), ([24, 1, 5], 4001, some)])
def test_three_cases_of_each(p, lens, vocab, shape, dtype):  # noqa: F811
    compared = 0
    for seed in range(100, 160):
        c = Case(lens, vocab, dtype, True, seed, shape)
        want, margin = c.plain()
        if margin < 2.0 ** -17:
            continue
        assert c.run(p) == want
        compared += 1
        if compared == 3:
            break
    assert compared == 3
    assert optr.optr_device_error(p) == 0
