"""Attention weights (optr_kv_score): one workspace for all steps of a server, sized by the largest."""
import itertools

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


@pytest.mark.parametrize("h", [1, 8])
@pytest.mark.parametrize("opts", [dict(), PAPER])
def test_the_size_grows_with_each_argument(h, opts):
    p = Score([1], [16], h_kv=h, seed=71, **opts).p
    batches = [1, 2, 8, 15, 16, 17, 40, 64, 65, 300, 1000, 8000]
    news = [1, 2, 3, 4, 5, 16, 63, 64, 65, 8192]
    pages = [1, 2, 16, 17, 64, 513, 2048, 8192, 131072, 1 << 20]
    size = {x: optr.optr_kv_score_workspace_size(p, x[0] * x[1], *x) for x in itertools.product(batches, news, pages)}
    assert all(v > 0 for v in size.values())
    for b, m, n in size:
        for larger in [(y, m, n) for y in batches if y > b] + [(b, y, n) for y in news if y > m] + \
                [(b, m, y) for y in pages if y > n]:
            assert size[b, m, n] <= size[larger], ((b, m, n), larger)


@pytest.mark.parametrize("sized,calls", [
    ((64, 64, 2048), [([1], [9000], 0), ([1] * 16, [40 * i for i in range(16)], 0), ([3], [16500], 0),
                      ([4] * 4, [8200, 30, 0, 700], 0), ([5] * 4, [300] * 4, 0), ([64, 1, 9], [500, 1000, 0], 0)]),
    # tables of 4096 pages: the largest step's logits would take 512 MB, a smaller step's are kept
    ((64, 1, 4096), [([1], [700], 4051), ([1] * 9, [100 * i for i in range(9)], 4044), ([1] * 3, [900] * 3, 2000)]),
    ((1, 5, 2048), [([4], [30000], 100), ([2], [32000], 0), ([5], [77], 9), ([1], [0], 0)])])
@pytest.mark.parametrize("opts", [dict(), dict(group=128), PAPER])
def test_one_workspace_serves_every_smaller_call(sized, calls, opts):
    """sized: sequences, new tokens of one and pages of a table at most; calls: new, past and a table's spare pages."""
    ws = None
    for new, past, spare in calls:
        c = Score(new, past, h_kv=8, seed=72, spare=spare, **opts)
        if ws is None:
            ws = optr.new_score_workspace(c.p, sized[0] * sized[1], *sized)
        assert c.B <= sized[0] and c.max_new <= sized[1] and c.bt.shape[1] <= sized[2]
        out = c.score.clone()
        args = (c.p, c.q, c.cu, c.pos0, c.max_new, c.bt, c.pool)
        if c.win is None:
            optr.optr_kv_score(*args, out, ws)
        else:
            optr.optr_kv_score_win(*args, c.win, c.slots, out, ws)
        c.check(out)
        assert optr.optr_device_error(c.p) == 0
