"""The example's cache read back is what was written, to its INT2 groups' steps."""
import pytest
import torch

from test_gpu_speculative import ex  # noqa: F401

pytestmark = pytest.mark.gpu


def test_rows_read_back(ex):  # noqa: F811
    """A group's range over 128 near-normal channels is 5.2 deviations in the mean
    (below 6), its step a third of that, the error uniform within half a step: an rms
    of 6 / 3 / sqrt(12) = 0.58 of the values' at most, and what clipping at 0.92
    adds to few channels stays within 0.1.  All zeros would be off by 1."""
    model, cache = ex.Model(1), ex.Cache(2, 1200, seed=2)
    lens = [1200, 700]
    g = torch.Generator(device="cuda").manual_seed(3)
    _, k, v = model.qkv(model.emb[torch.randint(ex.VOCAB, (sum(lens),), device="cuda", generator=g)])
    cache.write(k, v, lens)
    r0 = 0
    for n in lens:
        sink, recent = ex.CONFIG["sink"], ex.CONFIG["recent"]
        for got, want in zip(cache.rows(), (k, v)):
            got, want = got[r0:r0 + n].float(), want[r0:r0 + n].float()
            exact = torch.arange(n, device="cuda")
            exact = (exact < sink) | (exact >= n - recent)
            assert torch.equal(got[exact], want[exact])
            rel = ((got - want)[~exact].norm() / want[~exact].norm()).item()
            assert 0.2 <= rel <= 0.68, rel  # (two bits cannot do better than 0.2)
        r0 += n
    ex.check(cache)
