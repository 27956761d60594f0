"""The operators together, as examples/speculative.py runs them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)
    path = os.path.join(os.path.dirname(__file__), "..", "examples", "speculative.py")
    spec = importlib.util.spec_from_file_location("speculative", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_example(ex):
    text, cache, counts = ex.main(["--steps", "6", "--batch", "3", "--prompt", "300"])
    # every token but the last of each text is cached
    assert [len(t) - 1 for t in text] == cache.len
    assert all(0 <= x < ex.VOCAB for t in text for x in t)
    assert all(1 <= c <= 5 for c in counts)
    # the cache read back is the texts' keys and values, to INT2: exactly in
    # the windows of what was written to this cache, closely (its rotated
    # groups hold 4 levels each) elsewhere
    k, v = cache.rows()
    model = ex.Model(1)
    _, wk, wv = model.qkv(model.emb[torch.tensor(sum((t[:-1] for t in text), []), device="cuda")])
    r0 = 0
    for n in cache.len:
        last = slice(r0 + n - 6, r0 + n)  # written by the last steps
        for got, want in ((k, wk), (v, wv)):
            rel = (got[last].float() - want[last].float()).norm() / want[last].float().norm()
            assert rel <= 2.0 ** -6  # the same products in another batch, two bf16 roundings
            rel = (got[r0:r0 + n].float() - want[r0:r0 + n].float()).norm() / want[r0:r0 + n].float().norm()
            assert rel < 1.0
        r0 += n


def test_certain_drafts_are_all_accepted(ex):
    """A target equal to the draft accepts everything: its attention is zero."""
    g = torch.Generator(device="cuda").manual_seed(0)
    model = ex.Model(1)
    model.wo.zero_()
    cache = ex.Cache(2, 200, seed=2)
    last = torch.tensor([3, 4], device="cuda")
    new = ex.step(model, cache, last, 4, g)
    # equal up to the products' rounding in batches of another size
    assert [len(n) for n in new] == [5, 5] and cache.len == [5, 5]
