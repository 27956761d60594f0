"""Tree verification (optr_verify_tree): the mass of what a rejected child leaves, over a large vocabulary and many
sequences, where a thread has thousands of its terms.

Tolerance.  S is summed in float32 over 256 probabilities at most (2^-16 of it with every rounding to the same
side), and those sums in 64 bits; the mass and the two products that it meets add 2^-22.  So a decision 2^-15 from
its border is certain."""
import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_verify_tree import i32, p  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [1 << 21, (1 << 21) - 3])
@pytest.mark.parametrize("side", [-1, 1])
def test_terms_that_vanish_beside_the_sum_so_far(p, V, side):  # noqa: F811
    """A residual whose first 2048 tokens weigh 2^-13 each and all others so little that each of them alone is
    lost beside four of those in float32 (but not together: they are 2^-13 of the whole)."""
    B, few, x1, x2 = 160, 2048, 5, 9
    t = torch.full((3, V), 0.99 * 2.0 ** -35, device="cuda")
    t[:, :few] = 2.0 ** -13
    t[:, x1], t[:, x2] = 0.0, 0.6
    q = torch.zeros(3, V, device="cuda")
    q[:, x1] = q[:, x2] = 0.5
    w = (t[0] - q[0]).clamp_min(0).double()
    border = float(w[x2]) / (0.5 * float(w.sum()))
    u = torch.tensor([0.0, 0.9, border * (1 + side * 2.0 ** -15)], device="cuda")
    # the tree is the first sequence's, the others have no rows (but share the SMs)
    cu = i32([0] + [3] * B)
    acc = torch.full((B,), 99, dtype=torch.int32, device="cuda")
    path, nxt = (torch.full((3,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
    noise = torch.ones(B, V, device="cuda")
    optr.optr_verify_tree(p, t, q, i32([0, x1, x2]), i32([-1, 0, 0]), u, noise, cu, acc, path, nxt)
    assert acc.tolist() == [1 if side < 0 else 0] + [-1] * (B - 1)
    assert path.tolist() == ([0, 2, -1] if side < 0 else [0, -1, -1])
    assert optr.optr_device_error(p) == 0
