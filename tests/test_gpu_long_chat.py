"""Trees and eviction together, as examples/long_chat.py runs them."""
import importlib.util
import os
import sys

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
    path = os.path.join(os.path.dirname(__file__), "..", "examples", "long_chat.py")
    spec = importlib.util.spec_from_file_location("long_chat", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    sys.path.remove(os.path.dirname(os.path.abspath(path)))
    return m


def test_example(ex):
    text, chat, made, shrunk = ex.main(["--steps", "20", "--prompt", "400", "--budget", "360"])
    assert 20 * 3 <= made <= 3 * 20 * 3 and shrunk >= 2
    assert all(0 <= x < ex.VOCAB for t in text for x in t)
    assert all(n <= 360 + 32 for n in chat.len)
    # the weights of every token counted are 1 a query head: what stays is part of them
    assert torch.isfinite(chat.score).all() and (chat.score >= 0).all()
    for b, n in enumerate(chat.len):
        assert (chat.score[b, :, :n].sum(1) > 4).all() and not chat.score[b, :, n:].any()


def test_certain_drafts_are_all_accepted(ex):
    """A target equal to the draft accepts a child on each level: its attention is zero."""
    g = torch.Generator(device="cuda").manual_seed(0)
    model = ex.Model(1)
    model.wo.zero_()
    chat = ex.Chat(2, 200, seed=2)
    new = ex.step(model, chat, torch.tensor([3, 4], device="cuda"), 3, g)
    # equal up to the products' rounding in batches of another size
    assert [len(n) for n in new] == [3, 3] and chat.len == [3, 3]
    assert abs(float(chat.score.sum()) - 2 * ex.H * 4 * 3) < 1e-3
