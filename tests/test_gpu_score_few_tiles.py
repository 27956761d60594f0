"""Attention weights (optr_kv_score) of one to four tokens whose tables are too wide for their logits to be kept (256
MB): tiles on the tensor core, as of more tokens; test_gpu_score's cases and tolerance."""
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


@pytest.mark.parametrize("new,past", [([1], [0]), ([1], [1000]), ([2], [300]), ([3, 1], [129, 0]), ([4, 0, 2], [500, 9, 15])])
@pytest.mark.parametrize("opts", [dict(), dict(group=128), PAPER])
def test_wide_tables(new, past, opts):
    h, B, most = 8, len(new), max(new)
    pages = -(-max(a + b for a, b in zip(past, new)) // 16)
    widest = (256 << 20) // (B * h * 256 * most)    # 16 positions of 16 bytes a token
    got = []
    # either side of the border, with the same cache
    for spare in (widest - pages, widest + 1 - pages):
        c = Score(new, past, h_kv=h, seed=91, spare=spare, **opts)
        c.score.zero_()
        got.append(c.run()[:, :, :max(c.n)])
        c.score = c.score[:, :, :max(c.n)].contiguous()
        c.n_score = max(c.n)
        c.check(got[-1])
        assert optr.optr_device_error(c.p) == 0
        del c
        torch.cuda.empty_cache()
