"""Products in 8 bits whose waits run out at any point: what was on its way is let land, a status says so, and
the next call is right.  (csrc/ecq_ring.h's arithmetic for this: test_ring_cpu.py.)"""
import contextlib

import pytest
import torch

import paper_1806_08054_b200 as ecq
from act8_util import E4M3, strided, values
from test_gpu_product8 import whole_numbers

pytestmark = pytest.mark.gpu
F32 = torch.float32
LIMITS = (0, 1, 2, 3, 5, 10, 30, 100, 1000)
# operands exchanged, tiles by a CTA and by a pair with K in parts, tiles by pairs that stay
SIZES = [(5, 300, 900), (64, 4096, 4096), (200, 300, 900), (128, 4096, 4096), (1024, 1024, 8192), (2300, 2100, 300), (4096, 4096, 1024)]


@contextlib.contextmanager
def limit(polls):
    ecq.ecq_act8_set_wait_limit(polls)
    try:
        yield
        torch.cuda.synchronize()
    finally:
        ecq.ecq_act8_set_wait_limit()


@pytest.mark.parametrize("m,n,k", SIZES)
def test_the_next_call_is_right(m, n, k):
    a, b = whole_numbers(m, k, 1, E4M3), whole_numbers(n, k, 2, E4M3)
    d, status = strided(m, n, F32), torch.zeros(1, dtype=torch.int32, device="cuda")
    want = values(a) @ values(b).T
    for polls in LIMITS:
        status.zero_()
        with limit(polls):
            for _ in range(3):
                ecq.ecq_act8_product(a, b, d, status=status)
        assert status.item() in (0, 2) and (polls or status.item() == 2)
        if status.item() == 0:
            assert torch.equal(d.double(), want)
        d.fill_(7.0)
        status.zero_()
        ecq.ecq_act8_product(a, b, d, status=status)
        assert torch.equal(d.double(), want) and status.item() == 0


def right_or_nan(m, n, k, dtype=F32, add=False, stride=None):
    """Every entry is either the exact sum or NaN, and the status says whether there may be any of these."""
    a, b = whole_numbers(m, k, 1, E4M3), whole_numbers(n, k, 2, E4M3)
    d, status = strided(m, n, dtype, stride or n), torch.zeros(1, dtype=torch.int32, device="cuda")
    c = strided(m, n, dtype, stride or n).copy_(torch.randint(-9, 10, (m, n), device="cuda")) if add else None
    want = (values(a) @ values(b).T + (c.double() if add else 0)).to(dtype)     # one rounding of an exact sum
    for polls in LIMITS:
        d.fill_(7.0)
        status.zero_()
        with limit(polls):
            ecq.ecq_act8_product(a, b, d, add=c, status=status)
        bad = torch.isnan(d)
        assert torch.equal(d[~bad], want[~bad]), polls
        assert status.item() == 2 or (status.item() == 0 and not bool(bad.any()))


@pytest.mark.parametrize("m,n,k", SIZES[:5] + [(33, 200, 5000), (300, 504, 1000), (512, 4096, 1024)])
@pytest.mark.parametrize("add", [False, True])
def test_what_did_not_come_is_nan_where_k_is_shared_out(m, n, k, add):
    right_or_nan(m, n, k, add=add)


@pytest.mark.parametrize("m,n,k", SIZES[5:] + [(8192, 4096, 256), (2304, 2048, 31)])
@pytest.mark.parametrize("dtype,add", [(F32, False), (F32, True), (torch.bfloat16, False)])
def test_what_did_not_come_is_nan_in_tiles_by_pairs(m, n, k, dtype, add):
    for _ in range(3):
        right_or_nan(m, n, k, dtype, add, stride=n + 16)


@pytest.mark.parametrize("m,n,k", [(5, 301, 900), (200, 301, 900), (1024, 1021, 8192), (128, 4095, 4096), (2300, 2101, 300)])
@pytest.mark.parametrize("dtype,add", [(F32, False), (F32, True), (torch.float16, False), (torch.bfloat16, True)])
def test_what_did_not_come_is_nan_in_rows_that_begin_anywhere(m, n, k, dtype, add):
    for _ in range(3):
        right_or_nan(m, n, k, dtype, add)
