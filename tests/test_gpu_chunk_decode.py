"""Where chunk attention of one new token and the decode after that token's cache
write take the same keys, they agree: every key but the own one from its INT2
record, or every key exact.  The decode is good to 2e-5 (test_gpu_parity), so the
bounds are those of chunk attention's own roundings, as in test_gpu_chunk."""
import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_chunk import PAPER, Case, check, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


def decode(c):
    """The new tokens written, then one decode of their queries."""
    lens = i32([n + 1 for n in c.past])
    optr.optr_kv_append_win(c.p, c.k, c.v, c.cu, c.pos0, c.bt, c.pool, c.win, c.slots)
    out = torch.empty(c.q.shape, device="cuda")
    ws = optr.new_workspace(c.p, c.B, c.bt.shape[1])
    optr.optr_decode_attention_win(c.p, c.q, c.bt, lens, c.pool, c.win, c.slots, out, ws)
    assert optr.optr_device_error(c.p) == 0
    return out.double()


@pytest.mark.parametrize("group,clips,fold", [(32, 1.0, False), (128, 0.94, False), (32, 1.0, True)])
@pytest.mark.parametrize("past", [[500, 77], [1, 16, 17, 4000], [8192]])
def test_int2_past_and_the_own_token(past, group, clips, fold):
    """recent = 1: the decode's window is the new token; chunk attention reads
    the past without windows from the same records."""
    opts = dict(group=group, clip_k=clips, clip_v=clips)
    c = Case([1] * len(past), past, fold=fold, seed=40, sink=0, recent=1, **opts)
    p = optr.optr_params_create(c.R_k.cpu().float(), None if fold else c.R_v.cpu().float(), c.mu.cpu().float(),
                                4 * c.h, **opts)
    got = torch.empty_like(c.q)
    optr.optr_chunk_attention(p, c.q, c.k, c.v, c.cu, c.pos0, 1, c.bt, c.pool, got,
                              optr.new_chunk_workspace(p, c.B, c.B, 1))
    assert optr.optr_device_error(p) == 0
    check(got, decode(c))


@pytest.mark.parametrize("past", [[0, 1], [63, 64, 65], [128, 319, 200]])
def test_windows_that_hold_everything(past):
    """Up to sink + recent tokens with the own one."""
    c = Case([1] * len(past), past, seed=41, **PAPER)
    got = c.run().clone()
    check(got, decode(c))
