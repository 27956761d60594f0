"""Cached groups whose values leave fp16's range: chunk attention and read-back
compute with fp16 rows, so they report such a value where they meet one."""
import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_chunk import Case, check
from test_gpu_kv_read import check as check_rows, read

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


def set_group(c, pos, kind, group, scale, least):
    """{scale, min} of a group of sequence 0's record of pos, head 0."""
    ng = 128 // c.group
    at = 1024 + 64 * ng * kind + 4 * ng * (pos % 16) + 4 * group
    rec = c.pool[int(c.bt[0, pos // 16]), 0]
    rec[at:at + 4] = torch.tensor([scale, least], dtype=torch.float16, device="cuda").view(torch.uint8)


INSIDE = [(20000.0, 5504.0), (40000.0, -65504.0), (0.0, 65504.0)]
PAST = [(30000.0, 20000.0), (21856.0, 0.0), (float("inf"), 0.0), (0.0, float("inf")), (1.0, float("-inf")),
        (float("nan"), 0.0)]


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("group,at", [(32, 0), (32, 3), (128, 0)])
def test_read_back(group, at, kind):
    c = Case([1], [200], group=group, seed=31)
    for scale, least in INSIDE:
        set_group(c, 77, kind, at, scale, least)
        check_rows(c, (0,), (200,), *read(c, (0,), (200,)))
        assert optr.optr_device_error(c.p) == 0
    for scale, least in PAST:
        set_group(c, 77, kind, at, scale, least)
        read(c, (0,), (200,))
        assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_FP16_RANGE
        for first, n in ((0, 77), (78, 122)):  # read without it
            check_rows(c, (first,), (n,), *read(c, (first,), (n,)))
            assert optr.optr_device_error(c.p) == 0


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("group,at", [(32, 1), (32, 2), (128, 0)])
@pytest.mark.parametrize("new", [2, 50])
def test_chunk_attention(new, group, at, kind):
    c = Case([new], [200], group=group, sink=16, recent=100, seed=32)
    want = c.reference()
    for scale, least in PAST:
        set_group(c, 120, kind, at, scale, least)  # a window position: its record is not read
        check(c.run(), want)
        assert optr.optr_device_error(c.p) == 0
    for scale, least in INSIDE + PAST:
        set_group(c, 40, kind, at, scale, least)
        got = c.run()
        past = (scale, least) in PAST
        assert optr.optr_device_error(c.p) == (optr.OPTR_DEVERR_FP16_RANGE if past else 0)
        if not past:
            assert torch.isfinite(got).all()
