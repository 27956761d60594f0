"""Chunk attention: output rows that are 16-byte but not 32-byte aligned, and
queries so large that a few keys decide."""
import math

import pytest
import torch

from test_gpu_chunk import PAPER, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("new,past", [([5, 1], [100, 40]), ([70, 130], [40, 0]), ([3], [40000]), ([200], [4000])])
def test_output_aligned_to_16_bytes(new, past):
    """Whole and joined segments: the same bits, and nothing beside the rows."""
    c = Case(new, past, seed=50)
    want = c.run().clone()
    n = c.out.numel()
    buf = torch.full((n + 24,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf[8:8 + n].view_as(c.out)
    assert out.data_ptr() % 32 == 16
    assert torch.equal(c.run(out=out), want)
    assert (buf[:8] == 7.0).all() and (buf[8 + n:] == 7.0).all()


@pytest.mark.parametrize("scale", [8.0, 30.0])
@pytest.mark.parametrize("opts", [dict(), dict(PAPER, h_kv=1)])
def test_large_queries(scale, opts):
    """Rounding the rotated query and a key to fp16 moves a logit l = sum q_i k_i /
    sqrt(128) by independent terms, each at most 2^-11 |q_i k_i| for either, of rms
    1 / sqrt(3) of that: an rms s of at most sqrt(2 / 3) 2^-11 |q * k| / sqrt(128),
    |q * k| the norm of the products, about scale sqrt(128) for keys of unit size
    (those of the cache are smaller than their mean, which is not in them; largest
    of a head's below 1.5 times that).  No logit of the few thousand that count here
    moves by more than 6 s.  Weights that each move by a factor e^(+-6 s) move a mean
    of values within max|v| by at most 2 (e^(6 s) - 1) max|v|; weights, values and
    output in 16 bits add 2^-6 of it as in test_gpu_chunk.  A logit scaled by a wrong
    power of two, or an offset of the wrong keys, moves it by all of max|v|."""
    c = Case([9, 40], [500, 800], scale=scale, seed=51, **opts)
    got, want = c.run().double(), c.reference()
    s = math.sqrt(2 / 3) * 2.0 ** -11 * 1.5 * scale
    bound = (2 * math.expm1(6 * s) + 2.0 ** -6) * 2 * 4.5  # |v|: 2 randn, 4.5 deviations at least seen
    assert bound < want.abs().max() * 1.5
    err = (got - want).abs()
    assert err.max() <= bound, err.max().item()
    # in the mean the logits' rms moves the weights, not six times it
    assert (got - want).norm() <= (2 * s + 2.0 ** -8) * want.norm()
