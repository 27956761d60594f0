"""Attention weights (optr_kv_score) where the first keys' logits lie far from the other keys', and both far
from zero: no tile's share of a normaliser may leave a float's exponent range unseen.

Tolerance.  A logit is good to 2^-20 of |q||k| / sqrt(128) (include/optr.h): at log2 logits of 131, 91 in units
of e and no less than |q||k| / sqrt(128) here (keys and queries are parallel), to 8.7e-5.  A weight has its own
logit's error and the normaliser's, 1.8e-4 in all; exponentials and sums add less than 1e-5: 2e-4 of each
position's sum is allowed."""
import math

import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_chunk import i32
from test_gpu_score import Score

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


# log2 logits of the 128 keys and of the others
PAIRS = [(-117.4, -126.1), (-126.1, -117.4), (-115.5, -126.2), (-114.0, -127.0), (-110.0, -125.0), (-103.0, -128.5),
         (-126.2, -115.5), (-100.0, -107.0), (-96.0, -127.0), (-60.0, -130.0), (-58.0, -63.0), (100.0, 130.0),
         (112.0, 131.0), (60.0, 128.0), (117.0, 108.0), (127.5, 116.3), (128.0, 101.0)]


@pytest.mark.parametrize("few,rest", PAIRS)
@pytest.mark.parametrize("new,past,at", [([6], 3000, 0), ([40], 3000, 0), ([6], 60000, 0), ([40], 60000, 0),
                                         ([40], 3000, 1408), ([16], 60000, 30080), ([3], 3000, 0), ([2], 60000, 0)])
@pytest.mark.parametrize("opts", [dict(), dict(group=128), dict(sink=16, recent=100)])
def test_keys_of_two_sizes(few, rest, new, past, at, opts):
    """128 keys from position `at` on, and all others, are one row of +-1 in the rotated basis times a size of
    theirs; the queries are another multiple of that row."""
    c = Score(new, [past], h_kv=1, seed=61, **opts)
    g = torch.Generator(device="cuda").manual_seed(62)
    row = torch.randn(128, device="cuda", generator=g).sign().double()
    line = c.R_k[0] @ row
    n = c.n[0]
    z = math.copysign(7.0, rest)
    size = torch.full((n,), rest, dtype=torch.float64, device="cuda")
    size[at:at + 128] = few
    size *= math.log(2) / (128 ** 0.5 * z)     # 128 z size / sqrt(128) / ln 2 is the log2 logit
    k = (size[:, None] * line + c.mu[0]).bfloat16()[:, None].contiguous()
    args = (c.p, k, k, i32([0, n]), i32([0]), c.bt, c.pool)
    if c.win is None:
        optr.optr_kv_append(*args)
    else:
        optr.optr_kv_append_win(*args, c.win, c.slots)
    c.q.copy_((z * line).bfloat16().expand_as(c.q))
    c.score.zero_()
    got, want = c.run().double(), c.added()
    assert torch.isfinite(got).all()
    off = ((got - want).abs() / want.clamp_min(2.0 ** -100)).max().item()
    assert off <= 2e-4, off
    assert optr.optr_device_error(c.p) == 0
