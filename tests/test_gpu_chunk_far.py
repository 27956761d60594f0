"""Chunk attention over a pool whose pages lie past 32-bit offsets, and over
windows there; tolerances as in test_gpu_chunk."""
import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_chunk import Case, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("new,past", [((3, 1), (700, 1)), ((200, 70), (300, 1000))])
def test_far_pages_and_slots(new, past):
    c = Case(list(new), list(past), h_kv=8, group=128, sink=64, recent=256, seed=21)
    want = c.reference()
    far, slot = 500000, 3300
    pool = torch.empty(far + c.pool.shape[0], *c.pool.shape[1:], dtype=torch.uint8, device="cuda")
    win = torch.empty(slot + c.win.shape[0], *c.win.shape[1:], dtype=torch.bfloat16, device="cuda")
    assert pool.numel() > 2 ** 32 and win.numel() > 2 ** 31
    pool[far:], win[slot:] = c.pool, c.win
    c.pool, c.win = pool, win
    check(c.run(bt=c.bt + far, slots=c.slots + slot), want)
    assert optr.optr_device_error(c.p) == 0
