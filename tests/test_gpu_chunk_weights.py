"""Chunk attention where one key outweighs thousands that still count together."""
import pytest
import torch

from paper_2608_02691_gb300 import optr

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("first", [True, False])
def test_many_small_weights_under_one_large(new, first):
    """Keys are 0 but one, whose weight is 2^25.5 times each other's; the others'
    values are 1 and its own is 0 (constant groups: the records are exact), the
    new tokens' values are 0.  The output is n w / (1 + (n + own) w), w = 2^-25.5.

    In a weight 2^-18.5 of fp16's subnormals (that of the largest key is at least
    2^7) rounding is at most 2^-25, 2^-6.5 of it, and as much of the normalised
    output of 4.3e-5, 2^-10.5 of it; bf16 adds 2^-8.  Where the large key comes last
    only its own tile's weights are that small when they are rounded, 127 of 2047."""
    B, n = 160, 2048
    eye = torch.eye(128)[None]
    p = optr.optr_params_create(eye, None, torch.zeros(1, 128), 4)
    a = 1.5625  # 128 a / sqrt(128) = 17.68 = 25.5 log(2)
    k, v = torch.zeros(B, n, 1, 128, device="cuda"), torch.ones(B, n, 1, 128, device="cuda")
    at = 0 if first else n - 1
    k[:, at], v[:, at] = 1.0, 0.0
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    pages = n // 16
    pool = optr.new_pool(p, B * pages)
    bt = torch.arange(B * pages, device="cuda").view(B, pages).int()
    optr.optr_kv_append(p, k.view(-1, 1, 128).bfloat16(), v.view(-1, 1, 128).bfloat16(),
                        i32([n * b for b in range(B + 1)]), i32([0] * B), bt, pool)
    q = torch.full((B * new, 4, 128), a, dtype=torch.bfloat16, device="cuda")
    kn = torch.zeros(B * new, 1, 128, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    optr.optr_chunk_attention(p, q, kn, kn, i32([new * b for b in range(B + 1)]), i32([n] * B), new, bt,
                              pool, out, optr.new_chunk_workspace(p, B * new, B, new))
    w = torch.exp(torch.tensor(-128 * a / 128 ** 0.5, dtype=torch.float64))
    own = torch.arange(1, new + 1, dtype=torch.float64)
    want = ((n - 1) * w / (1 + (n - 1 + own) * w)).repeat(B)[:, None, None].cuda()
    rel = ((out.double() - want).abs() / want).max().item()
    assert rel <= 2.0 ** -6.4 + 2.0 ** -8, rel
    assert optr.optr_device_error(p) == 0
