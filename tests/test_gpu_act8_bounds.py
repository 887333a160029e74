"""Bounds that include/ecq.h states for matrices in 8 bits, at the entries that reach them."""
import pytest
import torch

import paper_1806_08054_b200 as ecq
from act8_util import E4M3, E5M2, check_plain, expand, pair, random, scale_places, stored, strided, values
from test_gpu_act8 import check_exactly
from test_gpu_product8 import bound, whole_numbers

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16

# The smallest largest entry of a block, unscaled, is the value above half the type's limit: 1.875 2^7 above 1.75 2^7, and 2^15
# above 1.75 2^14.  The largest entry that may change is the one below the smallest normal number that the type's
# subnormals (steps of 2^-9, 2^-16) do not have: 1.875 2^-7 and 1.75 2^-15.
WORST = {E4M3: (1.875 * 2.0 ** 7, 1.875 * 2.0 ** -7, 2.0 ** -14), E5M2: (2.0 ** 15, 1.75 * 2.0 ** -15, 1.75 * 2.0 ** -30)}


@pytest.mark.parametrize("kind", [E4M3, E5M2])
@pytest.mark.parametrize("rows,cols", [(128, 128), (300, 700), (1, 40), (513, 129)])
def test_storing_again_changes_only_small_entries_of_a_block(kind, rows, cols):
    torch.manual_seed(rows)
    sizes = torch.exp2(torch.randint(-40, 1, (rows, cols), device="cuda").double())
    x = random(rows, cols, 4) * sizes
    if rows > 1:                                             # both in one block of the transposed matrix, and apart in this one
        x[:2] = x[:, :1] = 0
        x[0, 0], x[1, 0] = WORST[kind][:2]
    p, t = stored(x, kind), pair(cols, rows, kind)
    ecq.ecq_act8_store(p, None, t)
    check_exactly(t, values(p).T.contiguous())
    v, again = values(p).T.contiguous(), values(t)
    largest = torch.nn.functional.pad(v.abs(), (0, -rows % 128)).view(cols, -1, 128).amax(2)
    share = v.abs() / expand(largest, rows)
    changed = v != again
    assert bool((share[changed] <= WORST[kind][2]).all())
    if rows > 1:
        assert bool(changed[0, 1]) and share[0, 1] == WORST[kind][2]


@pytest.mark.parametrize("m,n,k", [(128, 128, 256), (128, 128, 384), (1024, 1024, 1280), (200, 300, 900), (1, 300, 700), (40, 300, 4096)])
def test_a_products_bits_repeat_and_agree_between_calls_that_differ(m, n, k):
    """K is shared out by how d and c lie too: alone, added from elsewhere, in place, and in rows that begin anywhere agree
    to the sums' rounding (and the addition's and the result's), each repeats its own bits."""
    a, b = stored(random(m, k, 1)), stored(random(n, k, 2))
    c = random(m, n, 3).float()
    want, err = values(a) @ values(b).T, bound(a, b, k)
    total = want + c.double()
    for stride in (n, n + 1):
        for add in (None, "apart", "in place"):
            got = []
            for _ in range(3):
                d = strided(m, n, F32, stride)
                if add == "in place":
                    d.copy_(c)
                ecq.ecq_act8_product(a, b, d, add=None if add is None else d if add == "in place" else c)
                got.append(d)
            assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
            check_plain(got[0], want if add is None else total, err + (0 if add is None else total.abs() * 2.0 ** -24))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [1, 300])
def test_gate_at_the_ends_of_its_range(dtype, rows):
    inf, nan, top = float("inf"), float("nan"), torch.finfo(dtype).max
    g = torch.tensor([inf, -inf, top, -top, 200.0, -200.0, 0.0, inf], device="cuda").repeat(rows, 1).to(dtype)
    u = torch.tensor([2.0, 2.0, 0.5, 2.0, 2.0, 2.0, 2.0, 0.0], device="cuda").repeat(rows, 1).to(dtype)
    d = torch.full_like(g, 0.5)
    out, d_gate, d_up = (torch.empty_like(g) for _ in range(3))
    ecq.ecq_act8_gate(g, u, out)
    ecq.ecq_act8_gate_grad(g, u, d, d_gate, d_up)
    half = (torch.tensor(top, dtype=torch.float64) / 2).item()
    for got, want in ((out, [inf, nan, half, 0, 400, 0, 0, nan]), (d_gate, [nan, nan, 0.25, 0, 1, 0, 0.5, nan]),
                      (d_up, [inf, nan, half, 0, 100, 0, 0, inf])):
        assert torch.equal(got.double().nan_to_num(nan=7.0, posinf=8.0), torch.tensor(want, device="cuda").double().nan_to_num(nan=7.0, posinf=8.0)
                           .to(dtype).double().repeat(rows, 1))


def test_norm_of_rows_whose_squares_underflow():
    x = torch.zeros(3, 40, device="cuda")
    x[1], x[2] = 1e-30, 1e-10
    out, rstd = torch.empty_like(x), torch.empty(3, device="cuda")
    ecq.ecq_act8_norm(x, eps=0.0, out=out, rstd=rstd)
    assert bool(torch.isnan(out[0]).all()) and bool(torch.isinf(out[1]).all()) and bool((out[2] - 1).abs().max() < 1e-6)
    assert bool(torch.isinf(rstd[:2]).all())
    ecq.ecq_act8_norm(x, eps=1e-6, out=out)
    check_plain(out, x.double() / torch.sqrt(x.double().square().mean(1, keepdim=True) + 1e-6), x.double().abs() * 1e3 * 2.0 ** -22)


ROWS = [(300, 400), (256, 4096), (5, 130)]                       # one row of A: K within a warp's step, shared out, and short


@pytest.mark.parametrize("n,k", ROWS)
@pytest.mark.parametrize("low,high", [(1, 253), (0, 254), (254, 0), (127, 127), (100, 1), (254, 254), (0, 0), (1, 0)])
def test_far_scales_of_one_row(n, k, low, high):
    """Scales at both ends of their range, which may cancel, overflow or underflow in the product.  Sums of whole numbers times
    one power of two are exact in 32 bits as long as they are normal.  Below that, each sixteen products' sum is rounded once,
    to a multiple of 2^-149 (by 2^-150 at most), and adding such multiples rounds nothing: ceil(k / 16) 2^-150 in all.  Where
    the magnitudes together pass the range of 32 bits, sums of what is left of them may be anything."""
    a, b = whole_numbers(1, k, 1, E4M3), whole_numbers(n, k, 2, E4M3)
    a[1][scale_places(1, k)] = low
    b[1][scale_places(n, k)] = high
    d = strided(1, n, F32)
    ecq.ecq_act8_product(a, b, d)
    want, size = values(a) @ values(b).T, values(a).abs() @ values(b).abs().T
    inside = size <= torch.finfo(F32).max
    assert bool(((d.double() - want).abs() <= -(-k // 16) * 2.0 ** -150)[inside].all())
    normal = inside & (size >= 2.0 ** -100)                       # units of these are far above 2^-149
    assert torch.equal(d[normal].double(), want[normal])
    assert not bool(torch.isfinite(d[want.abs() > torch.finfo(F32).max]).any())


@pytest.mark.parametrize("n,k", ROWS)
def test_nan_blocks_of_one_row(n, k):
    x, y = random(1, k, 1).float(), random(n, k, 2).float()
    y[n - 2, k - 1], y[1, 0] = float("nan"), float("inf")
    a, b = stored(x.double()), stored(y.double())
    c = random(1, n, 3).float()
    for add in (None, c):
        d = strided(1, n, F32)
        ecq.ecq_act8_product(a, b, d, add=add)
        bad = torch.isnan(d)
        assert bool(bad[0, 1] and bad[0, n - 2]) and int(bad.sum()) == 2
    x[0, k - 1] = float("nan")
    ecq.ecq_act8_product(stored(x.double()), b, d)
    assert bool(torch.isnan(d).all())


@pytest.mark.parametrize("m,n,k", [(2600, 2304, 31), (4196, 4096, 128), (2304, 2148, 200)])
@pytest.mark.parametrize("add", [False, True])
def test_pairs_of_ctas_of_which_one_has_nothing_to_write(m, n, k, add):
    """The last row or column of tiles is less than half inside; calls on top of each other."""
    a, b = whole_numbers(m, k, 1, E4M3), whole_numbers(n, k, 2, E4M3)
    want = values(a) @ values(b).T
    d = torch.zeros(m, n, device="cuda")
    for calls in range(1, 31):
        ecq.ecq_act8_product(a, b, d, add=d if add else None)
    assert torch.equal(d.double(), want * (calls if add else 1))
