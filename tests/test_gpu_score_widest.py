"""Attention weights (optr_kv_score): tables wider than any cache that the library writes are refused on the host."""
import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_chunk import PAPER
from test_gpu_score import Score

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [[1], [6]])
@pytest.mark.parametrize("opts", [dict(), PAPER])
def test_widest_tables(new, opts):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    c = Score(new, [74], h_kv=1, seed=95, **opts)

    def call(pages):
        table = torch.full((1, pages), -1, dtype=torch.int32, device="cuda")
        table[0, :c.bt.shape[1]] = c.bt[0]
        ws = optr.new_score_workspace(c.p, sum(new), 1, max(new), pages)
        out = c.score.clone()
        args = (c.p, c.q, c.cu, c.pos0, max(new), table, c.pool)
        if c.win is None:
            optr.optr_kv_score(*args, out, ws)
        else:
            optr.optr_kv_score_win(*args, c.win, c.slots, out, ws)
        return out

    c.check(call(1 << 26))
    with pytest.raises(optr.OptrError) as e:
        call((1 << 26) + 1)
    assert e.value.status == -3
    assert optr.optr_device_error(c.p) == 0
    torch.cuda.empty_cache()
