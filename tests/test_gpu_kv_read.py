"""Cached rows back in the model's basis (optr_kv_read) against
k = khat R_k^T + mu, v = vhat R_v^T in 64 bits, from the pool's own bytes.

Tolerance.  The dequantized value is rounded to fp16: by Cauchy-Schwarz and
since R's rows have norm 1 that moves an element by at most 2^-11 |khat|, and
|khat| = |y - mu|.  R's two fp16 parts keep it to 2^-21, the 256 float32
accumulations to 256 * 2^-24: 2^-16 |khat| together and to spare.  The result
is rounded once to bf16: 8 bits, so 2^-8 of it at most (of 1 + 2^-8, 1 and
1 + 2^-7 are the nearest)."""

import pytest
import torch

from paper_2608_02691_gb300 import optr
from test_gpu_chunk import Case, cu_of, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _setup():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02691_gb300 import build
    build.build()
    torch.cuda.set_device(0)


def read(c, first, lens, cu=None, bt=None, pool=None, n=None, stream=None):
    """k, v of lens[b] rows from position first[b]; rows past them stay 7."""
    n = sum(lens) if n is None else n
    k = torch.full((n + 130, c.h, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    v = torch.full_like(k, 7.0)
    optr.optr_kv_read(c.p, cu_of(lens) if cu is None else cu, i32(first), c.bt if bt is None else bt,
                      c.pool if pool is None else pool, k[:n], v[:n], stream=stream)
    torch.cuda.synchronize()
    assert (k[n:] == 7.0).all() and (v[n:] == 7.0).all()
    return k[:n], v[:n]


def check(c, first, lens, k, v, skip=()):
    """Every row outside skip against the formula."""
    r0 = 0
    for b, (s, m) in enumerate(zip(first, lens)):
        for h in range(c.h):
            for got, kind, R, add in ((k, 0, c.R_k, c.mu[h]), (v, 1, c.R_v, 0.0)):
                z = c.rows(b, h, s, s + m, kind)
                want = (z @ R[h].T if R is not None else z) + add
                err = (got[r0:r0 + m, h].double() - want).abs()
                bound = (2.0 ** -8 * (1 + 2.0 ** -6)) * want.abs() \
                    + (2.0 ** -11 + 2.0 ** -16) * z.norm(dim=1, keepdim=True)
                ok = err <= bound
                for t in skip:
                    if r0 <= t < r0 + m:
                        ok[t - r0] = True
                assert ok.all(), (b, h, kind, (err / bound).max().item())
        r0 += m


SETS = [((0,), (1,)), ((0, 5, 0), (0, 3, 0)), ((0, 1, 3), (127, 128, 129)), ((17,), (1000,)),
        ((9, 0, 250, 31), (256, 0, 1, 640)), ((15, 16, 17), (1, 1, 1))]


@pytest.mark.parametrize("first,lens", SETS)
@pytest.mark.parametrize("group,h,fold", [(32, 2, False), (128, 2, False), (32, 1, True), (128, 8, False)])
def test_formula(first, lens, group, h, fold):
    c = Case([1] * len(lens), [s + m for s, m in zip(first, lens)], h_kv=h, fold=fold, group=group,
             clip_k=0.96, clip_v=0.92, seed=len(lens) + sum(lens))
    check(c, first, lens, *read(c, first, lens))
    assert optr.optr_device_error(c.p) == 0


def test_many_tiles_of_a_cta():
    c = Case([1, 1], [16000, 24001], h_kv=8, group=128, seed=3)
    first, lens = (3, 0), (15997, 24001)
    check(c, first, lens, *read(c, first, lens))


def test_more_sequences_than_are_held_on_chip():
    lens = [(i * 7) % 4 for i in range(700)]
    first = [i % 5 for i in range(700)]
    c = Case([1] * 700, [s + m for s, m in zip(first, lens)], seed=5)
    check(c, first, lens, *read(c, first, lens))
    assert optr.optr_device_error(c.p) == 0


def test_window_positions_come_from_their_records():
    c = Case([1], [700], group=128, clip_k=0.96, clip_v=0.92, sink=64, recent=256, seed=6)
    check(c, (0,), (700,), *read(c, (0,), (700,)))


def test_pages_past_32_bit_offsets():
    c = Case([1, 1], [100, 333], h_kv=8, seed=7)
    far = 400000  # 12 KB a page
    pool = torch.empty(far + c.pool.shape[0], *c.pool.shape[1:], dtype=torch.uint8, device="cuda")
    assert pool.numel() > 2 ** 32
    pool[far:] = c.pool
    check(c, (0, 1), (100, 332), *read(c, (0, 1), (100, 332), bt=c.bt + far, pool=pool))


@pytest.mark.parametrize("group", [32, 128])
def test_bad_entries_read_as_zero_records(group):
    first, lens = (5, 0), (200, 140)
    c = Case([1, 1], [205, 140], group=group, seed=8)
    mu = c.mu.bfloat16()
    zero = lambda k, v, rows: (k[rows] == mu).all() and not v[rows].any()
    for bad in (-1, c.pool.shape[0], 2 ** 31 - 1, -2 ** 31):
        bt = c.bt.clone()
        bt[0, 3] = bad  # positions 48 .. 63: rows 43 .. 58
        k, v = read(c, first, lens, bt=bt)
        assert zero(k, v, slice(43, 59))
        check(c, first, lens, k, v, skip=range(43, 59))
        assert optr.optr_device_error(c.p) == optr.OPTR_DEVERR_PAGE_ID
    end = c.bt.shape[1] * 16
    for pos, gone in ((-3, slice(0, 3)), (end - 150, slice(150, 200)), (2 ** 31 - 10, slice(0, 200))):
        k, v = read(c, (pos, 0), lens)
        assert zero(k, v, gone)
        assert optr.optr_device_error(c.p) & optr.OPTR_DEVERR_POSITION
        for h in range(2):  # the other sequence is untouched by it
            check(c, (205 - 1, 0), (0, 140), k[200:], v[200:])
        optr.optr_device_error(c.p)
    for cu, gone in (([2, 200, 340], slice(0, 2)), ([0, 200, 330], slice(330, 340)),
                     ([0, -5, 340], slice(0, 0)), ([340, 0, 0], slice(0, 340))):
        k, v = read(c, first, lens, cu=i32(cu))
        assert zero(k, v, gone)
        flags = optr.optr_device_error(c.p)
        assert not gone.stop or flags & optr.OPTR_DEVERR_CU_NEW
    k, v = read(c, first, lens)
    check(c, first, lens, k, v)
    assert optr.optr_device_error(c.p) == 0


def test_other_stream_and_graph():
    c = Case([1], [500], seed=9)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        k, v = read(c, (0,), (500,))
    check(c, (0,), (500,), k, v)
    cu, pos = cu_of([300]), i32([100])
    k, v = torch.zeros(300, 2, 128, dtype=torch.bfloat16, device="cuda"), \
        torch.zeros(300, 2, 128, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        optr.optr_kv_read(c.p, cu, pos, c.bt, c.pool, k, v)
    g.replay()
    check(c, (100,), (300,), k, v)
    pos.fill_(7)  # read where it is used
    c.pool[:, :, :1024] ^= 0x5A
    g.replay()
    check(c, (7,), (300,), k, v)


def test_refusals():
    c = Case([1], [40], seed=10)
    k = torch.full((40, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    v = k.clone()
    call = lambda cu=cu_of([40]), pos=i32([0]), bt=c.bt, k=k, v=v: \
        optr.optr_kv_read(c.p, cu, pos, bt, c.pool, k, v)
    for bad in (dict(k=k.cpu()), dict(k=k.cpu().pin_memory()), dict(v=v.float()), dict(v=v[:39]),
                dict(k=k[:, :1], v=v[:, :1]), dict(k=k.transpose(0, 1), v=v.transpose(0, 1)),
                dict(cu=cu_of([40]).long()), dict(pos=i32([0, 0])), dict(cu=cu_of([20, 20]))):
        with pytest.raises(ValueError):
            call(**bad)
    odd = torch.empty(40 * 256 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(40, 2, 128)
    with pytest.raises(optr.OptrError) as e:
        call(k=odd)
    assert e.value.status == -1
    assert (k == 7.0).all() and (v == 7.0).all()
    call(cu=i32([0, 0]), k=k[:0], v=v[:0])
