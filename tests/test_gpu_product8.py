"""Products of matrices in 8 bits against 64 bits."""
import math

import pytest
import torch

import paper_1806_08054_b200 as ecq
from act8_util import E4M3, E5M2, check_pair, check_plain, expand, pair, random, scale_bytes, scale_places, stored, strided, values

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
# few tokens (both sides of 16, 32, 64), tiles of 128 with K in parts, pairs of CTAs, odd sizes, short and long K
SIZES = [(1, 1, 1), (1, 128, 128), (1, 1000, 300), (3, 130, 2050), (16, 256, 512), (17, 100, 1000), (32, 512, 129), (33, 64, 4096),
         (64, 300, 640), (65, 128, 128), (100, 1, 100), (128, 128, 1024), (129, 257, 385), (300, 300, 3000), (512, 640, 64),
         (2048, 1536, 256), (1793, 1666, 500), (2500, 2300, 1030), (2304, 2048, 31), (3000, 1800, 130)]


def whole_numbers(rows, cols, seed, dtype):
    """Small whole numbers times powers of two that differ from block to block: every sum is exact in 32 bits."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    q = torch.randint(-3, 4, (rows, cols), generator=gen, device="cuda").float()
    e = torch.randint(-1, 2, (rows, -(-cols // 128)), generator=gen, device="cuda")
    p = pair(rows, cols, dtype, extra=rows % 2)
    p[0].view(torch.uint8).copy_(q.to(dtype).view(torch.uint8))
    p[1][scale_places(rows, cols)] = (e + 127).to(torch.uint8)
    return p


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("a_type,b_type", [(E4M3, E4M3), (E5M2, E4M3), (E4M3, E5M2), (E5M2, E5M2)])
def test_exact_sums(m, n, k, a_type, b_type):
    """|terms| <= 9 * 4 in units of 1/4: below 2^24 units up to K = 116000."""
    a, b = whole_numbers(m, k, 1, a_type), whole_numbers(n, k, 2, b_type)
    d = strided(m, n, F32, n + n % 3, fill=5.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ecq.ecq_act8_product(a, b, d, status=status)
    assert torch.equal(d.double(), values(a) @ values(b).T) and status.item() == 0
    around = torch.as_strided(d, (m, d.stride(0)), (d.stride(0), 1))[:, n:]
    assert bool((around == 5.0).all())


def bound(a, b, k):
    """Sums of 32 products, aligned and added to the running sum: at most 2^-22 of all magnitudes each."""
    return (values(a).abs() @ values(b).abs().T) * (k / 32 + 8) * 2.0 ** -22


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("out", ["f32", "bf16", "f16", "e4m3", "e5m2", "add"])
def test_random(m, n, k, out):
    a, b = stored(random(m, k, 3)), stored(random(n, k, 4, 1 / math.sqrt(k) / 8))
    want, err = values(a) @ values(b).T, bound(a, b, k)
    if out in ("e4m3", "e5m2"):
        d = pair(m, n, E4M3 if out == "e4m3" else E5M2)
        ecq.ecq_act8_product(a, b, d)
        check_pair(d, want, err)
    elif out == "add":
        for c_type, d_type in ((F32, F32), (BF16, F32), (F16, BF16), (F32, F16)):
            c = strided(m, n, c_type, n + 1, 1).copy_(random(m, n, 5))
            d = strided(m, n, d_type, n + 2)
            ecq.ecq_act8_product(a, b, d, add=c)
            total = want + c.double()
            check_plain(d, total, err + total.abs() * 2.0 ** -24)
    else:
        dtype = dict(f32=F32, bf16=BF16, f16=F16)[out]
        for stride, offset in ((n, 0), (n + 5, 1), (-(-n // 16) * 16, 0)):
            d = strided(m, n, dtype, stride, offset)
            ecq.ecq_act8_product(a, b, d)
            check_plain(d, want, err)


@pytest.mark.parametrize("m,n,k", [(5, 300, 400), (200, 300, 1300), (1000, 1500, 2000), (2300, 2100, 300), (2304, 2048, 700), (2500, 2333, 90)])
@pytest.mark.parametrize("c_type,d_type", [(F32, F32), (BF16, BF16), (F16, F16), (F32, BF16), (BF16, F32), (F16, BF16)])
def test_additions_of_aligned_rows(m, n, k, c_type, d_type):
    """Rows on 16-byte boundaries, with columns that end anywhere; what lies behind them is left."""
    a, b = stored(random(m, k, 3)), stored(random(n, k, 4, 1 / math.sqrt(k) / 8))
    stride = -(-n // 16) * 16 + 16
    want, err = values(a) @ values(b).T, bound(a, b, k)
    c = strided(m, n, c_type, stride).copy_(random(m, n, 5))
    d = strided(m, n, d_type, stride, fill=7.0)
    total = want + c.double()
    ecq.ecq_act8_product(a, b, d, add=c)
    check_plain(d, total, err + total.abs() * 2.0 ** -24)
    assert bool((torch.as_strided(d, (m, stride), (stride, 1))[:, n:] == 7.0).all())
    if c_type == d_type:
        ecq.ecq_act8_product(a, b, c, add=c)
        assert torch.equal(c, d)


@pytest.mark.parametrize("m,n,k", [(5, 301, 400), (200, 333, 300), (2500, 2333, 90), (2304, 2056, 130)])
@pytest.mark.parametrize("d_type", [F32, BF16, E4M3, E5M2])
def test_what_lies_behind_the_last_column_is_left(m, n, k, d_type):
    a, b = stored(random(m, k, 3)), stored(random(n, k, 4))
    if d_type in (E4M3, E5M2):
        d = pair(m, n, d_type, extra=1)
        ecq.ecq_act8_product(a, b, d)
        whole = torch.as_strided(d[0].view(torch.uint8), (m, d[0].stride(0)), (d[0].stride(0), 1))
        assert bool((whole[:, n:] == 0xA5).all())
        rest = torch.ones_like(d[1], dtype=torch.bool)
        rest[scale_places(m, n)] = False
        assert bool((d[1][rest] == 0xA5).all())
    else:
        stride = -(-n // 16) * 16 + 16
        d = strided(m, n, d_type, stride, fill=7.0)
        ecq.ecq_act8_product(a, b, d)
        whole = torch.as_strided(d, (m, stride), (stride, 1))
        assert bool((whole[:, n:] == 7.0).all())
        check_plain(d, values(a) @ values(b).T, bound(a, b, k))
        once = d.clone()
        ecq.ecq_act8_product(a, b, d, add=d)
        total = values(a) @ values(b).T + once.double()
        check_plain(d, total, bound(a, b, k) + total.abs() * 2.0 ** -24)
        assert bool((whole[:, n:] == 7.0).all())


@pytest.mark.parametrize("m,n,k", [(5, 300, 400), (200, 300, 1300), (2300, 2100, 300)])
def test_in_place_addition(m, n, k):
    a, b = whole_numbers(m, k, 1, E4M3), whole_numbers(n, k, 2, E4M3)
    d = torch.randint(-100, 100, (m, n), device="cuda").float()
    want = d.double() + values(a) @ values(b).T
    ecq.ecq_act8_product(a, b, d, add=d)
    assert torch.equal(d.double(), want)


@pytest.mark.parametrize("m,n,k,stride", [(1, 300, 400, 300), (5, 301, 400, 303), (200, 304, 1300, 304), (200, 301, 300, 301), (2300, 2104, 300, 2104),
                                          (2300, 2101, 300, 2101), (2300, 2102, 300, 2104)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_in_place_is_as_apart(m, n, k, stride, dtype):
    a, b = stored(random(m, k, 1)), stored(random(n, k, 2))
    c, d, e = (strided(m, n, dtype, stride) for _ in range(3))
    c.copy_(random(m, n, 3))
    e.copy_(c)
    ecq.ecq_act8_product(a, b, d, add=c)
    ecq.ecq_act8_product(a, b, e, add=e)
    assert torch.equal(d, e)


@pytest.mark.parametrize("m,n,k", [(5, 300, 700), (200, 300, 1300), (2300, 2100, 300)])
def test_nan_blocks_reach_their_rows_and_columns_alone(m, n, k):
    x, y = random(m, k, 1).float(), random(n, k, 2).float()
    x[m - 2, k - 1], y[7, 0] = math.nan, math.inf
    a, b = stored(x.double()), stored(y.double())
    d = strided(m, n, F32)
    ecq.ecq_act8_product(a, b, d)
    bad = torch.isnan(d)
    want = torch.zeros_like(bad)
    want[m - 2] = True
    want[:, 7] = True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("m,n,k", [(2, 256, 300), (140, 256, 300), (2300, 2100, 300)])
def test_far_scales(m, n, k):
    """Scales at both ends of their range that cancel in the product, and zero blocks (byte 0)."""
    a, b = whole_numbers(m, k, 1, E4M3), whole_numbers(n, k, 2, E4M3)
    a[1][scale_places(m, k)] = 1
    b[1][scale_places(n, k)] = 253
    a[0].view(torch.uint8)[m // 2] = 0
    a[1][scale_places(m, k)[m // 2]] = 0
    d = strided(m, n, F32)
    ecq.ecq_act8_product(a, b, d)
    assert torch.equal(d.double(), values(a) @ values(b).T)


def test_results_repeat():
    a, b = stored(random(300, 5000, 1)), stored(random(400, 5000, 2))
    outs = [torch.empty(300, 400, device="cuda") for _ in range(3)]
    for d in outs:
        ecq.ecq_act8_product(a, b, d)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("m,n,k", [(5, 300, 900), (200, 300, 900), (2300, 2100, 300)])
def test_a_wait_that_runs_out_is_reported(m, n, k):
    """No polls at all: every result is NaN, the status says so, and the next call is sound.  (A single row of A is
    multiplied without waits.)"""
    a, b = whole_numbers(m, k, 1, E4M3), whole_numbers(n, k, 2, E4M3)
    d, status = strided(m, n, F32), torch.zeros(1, dtype=torch.int32, device="cuda")
    ecq.ecq_act8_set_wait_limit(0)
    try:
        ecq.ecq_act8_product(a, b, d, status=status)
        torch.cuda.synchronize()
    finally:
        ecq.ecq_act8_set_wait_limit()
    assert status.item() == 2 and bool(torch.isnan(d).all())
    ecq.ecq_act8_product(a, b, d)
    assert torch.equal(d.double(), values(a) @ values(b).T)


def test_no_rows_and_refusals():
    a, b = pair(0, 300), stored(random(5, 300, 1))
    before = ecq.ecq_launch_count()
    ecq.ecq_act8_product(a, b, torch.empty(0, 5, device="cuda"))
    assert ecq.ecq_launch_count() == before
    a = stored(random(4, 300, 1))
    with pytest.raises(ValueError):
        ecq.ecq_act8_product(a, stored(random(5, 301, 1)), torch.empty(4, 5, device="cuda"))
    with pytest.raises(ValueError):
        ecq.ecq_act8_product(a, b, torch.empty(4, 6, device="cuda"))
    with pytest.raises(ecq.EcqError):
        ecq.ecq_act8_product(a, b, pair(4, 5), add=torch.empty(4, 5, device="cuda"))
    with pytest.raises(ecq.EcqError):
        ecq.ecq_act8_product(a[0].float(), b, torch.empty(4, 5, device="cuda"))
