"""Matrices in 8 bits: storing, restoring, the gated activation and the norm with their gradients,
against plain restatements in 64 bits."""
import math

import pytest
import torch

import paper_1806_08054_b200 as ecq
from act8_util import (E4M3, E5M2, block_scales, bytes_of, check_pair, check_plain, expand, half_step, pair, random, rounded,
                       scale_bytes, scale_places, stored, strided, values)

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
SIZES = [(1, 1), (1, 128), (3, 127), (5, 129), (128, 128), (127, 255), (129, 513), (300, 1000), (64, 4096), (257, 640)]


def behind_is_left(p, fill=0xA5):
    cols = p[0].shape[1]
    assert bool((bytes_of(p)[:, cols:] == fill).all())
    mask = torch.ones_like(p[1], dtype=torch.bool)
    mask[scale_places(*p[0].shape)] = False
    assert bool((p[1][mask] == fill).all())


def check_exactly(p, x):
    """A pair is x's, bit for bit but for the sign of zeros."""
    b = block_scales(x, p[0].dtype)
    assert torch.equal(scale_bytes(p), b)
    want = rounded(x, b, p[0].dtype)
    assert torch.equal(torch.nan_to_num(values(p), nan=12345.0), torch.nan_to_num(want, nan=12345.0))
    behind_is_left(p)


# ---- store, load ---------------------------------------------------------------------------------

@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("to", [E4M3, E5M2])
def test_store_is_the_definition(rows, cols, dtype, to):
    x = strided(rows, cols, dtype)
    x.copy_(random(rows, cols, rows * cols, 1e-2))
    q, t = pair(rows, cols, to), pair(cols, rows, to, extra=1)
    ecq.ecq_act8_store(x, q, t)
    check_exactly(q, x.double())
    check_exactly(t, x.double().T.contiguous())


@pytest.mark.parametrize("stride,offset", [(131, 0), (131, 1), (136, 3), (160, 8)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_store_any_alignment(stride, offset, dtype):
    x = strided(140, 130, dtype, stride, offset)
    x.copy_(random(140, 130, 5))
    q, t = pair(140, 130, extra=2), pair(130, 140)
    ecq.ecq_act8_store(x, q, t)
    check_exactly(q, x.double())
    check_exactly(t, x.double().T.contiguous())


@pytest.mark.parametrize("only", ["q", "t"])
def test_store_one_way_leaves_the_other(only):
    x = random(200, 300, 3).float()
    p = pair(200, 300) if only == "q" else pair(300, 200)
    ecq.ecq_act8_store(x, *((p, None) if only == "q" else (None, p)))
    check_exactly(p, x.double() if only == "q" else x.double().T.contiguous())


def test_scales_at_the_borders():
    """Blocks whose largest entry is a power of two times 448, the next float above, zero, the smallest
    and the largest floats."""
    tops = [448.0, math.nextafter(448.0, 500), 448.0 * 2 ** -40, 449 * 2.0 ** 60, 0.0, 2.0 ** -149, 2.0 ** -126, 2.0 ** -118,
            448 * 2.0 ** -127, 449 * 2.0 ** -127, 3.4028234663852886e38, 1.0, 1.75, 1.7500001, 57344.0, 57345.0]
    x = torch.zeros(len(tops), 128, dtype=torch.float64, device="cuda")
    x[:, 5] = torch.tensor(tops, dtype=torch.float64, device="cuda").float().double()
    x[:, 77] = -x[:, 5] / 3
    x = x.float()
    for to in (E4M3, E5M2):
        p = pair(len(tops), 128, to)
        ecq.ecq_act8_store(x, p)
        check_exactly(p, x.double())


def test_every_value_of_both_types_comes_back():
    for dtype in (E4M3, E5M2):
        every = torch.arange(256, dtype=torch.uint8, device="cuda").view(dtype).float()
        every = every[torch.isfinite(every)]
        largest = every.max()
        x = torch.zeros(9, 128 * 3, device="cuda")
        x[:, :every.numel()] = every
        x[:, 127] = x[:, 255] = x[:, 383] = largest       # each block's scale is 1 times the row's factor
        x = x * torch.exp2(torch.tensor([-100.0, -20, -7, -1, 0, 1, 9, 40, 100], device="cuda"))[:, None]
        p, out = pair(9, 384, dtype), strided(9, 384, F32)
        ecq.ecq_act8_store(x, p)
        ecq.ecq_act8_load(p, out)
        assert torch.equal(out, x)


def test_nan_and_inf_stay_in_their_block():
    x = random(130, 300, 9).float()
    x[3, 5], x[7, 200], x[129, 299] = math.nan, math.inf, -math.inf
    q, t = pair(130, 300), pair(300, 130)
    ecq.ecq_act8_store(x, q, t)
    check_exactly(q, x.double())
    check_exactly(t, x.double().T.contiguous())
    out = strided(130, 300, F32)
    ecq.ecq_act8_load(q, out)
    bad = torch.isnan(out)
    assert bool(bad[3, :128].all() and bad[7, 128:256].all() and bad[129, 256:].all()) and int(bad.sum()) == 128 + 128 + 44


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("kind", [E4M3, E5M2])
@pytest.mark.parametrize("rows,cols,stride", [(1, 1, 1), (130, 257, 259), (64, 512, 512), (31, 100, 104)])
def test_load(dtype, kind, rows, cols, stride):
    p = stored(random(rows, cols, 11, 0.1), kind)
    out = strided(rows, cols, dtype, stride, fill=7.0)
    ecq.ecq_act8_load(p, out)
    assert torch.equal(out, values(p).to(dtype))
    whole = torch.as_strided(out, (rows, stride), (stride, 1))
    assert bool((whole[:, cols:] == 7.0).all())


@pytest.mark.parametrize("rows,cols", [(128, 128), (300, 700), (1, 40), (513, 129)])
def test_storing_again_transposed_changes_only_what_underflows(rows, cols):
    p = stored(random(rows, cols, 4))
    t = pair(cols, rows)
    ecq.ecq_act8_store(p, None, t)
    check_exactly(t, values(p).T.contiguous())
    v, again = values(p).T, values(t)
    top = torch.exp2(expand(scale_bytes(t).double(), rows) - 127) * 2.0 ** -6
    assert torch.equal(torch.where(v.abs() >= top, v, 0.0), torch.where(v.abs() >= top, again, 0.0))


def test_store_of_an_8_bit_matrix_in_the_other_type():
    p = stored(random(100, 200, 8))
    q = pair(100, 200, E5M2)
    ecq.ecq_act8_store(p, q)
    check_exactly(q, values(p))


# ---- gated activation ------------------------------------------------------------------------------

def gate64(g, u):
    s = torch.sigmoid(g)
    return g * s * u, s


def gate_error(g, u, dtype):
    """sigmoid from exp2 of a rounded product: its argument's rounding (and log2(e)'s) times ln 2, 2^-22 of
    exp2 and a reciprocal's, then three products; in 32 bits the argument's rounding is put back.  A
    sigmoid below the smallest normal number of 32 bits, 2^-126, is 0."""
    rel = 2.0 ** -20 + (0 if dtype == F32 else 1) * g.abs() * 2.0 ** -23
    return (g * torch.sigmoid(g) * u).abs() * rel + (g * u).abs() * 2.0 ** -126 + 2.0 ** -126


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (5, 129), (128, 128), (130, 300), (257, 1001)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("kept", [False, True])
def test_gate(rows, cols, dtype, kept):
    size = 0.05 if dtype == F16 else 1.0
    a, b = random(rows, cols, 1, 2 * size), random(rows, cols, 2, size)
    if kept:
        gate, up = stored(a), stored(b)
        g, u = values(gate), values(up)
    else:
        gate, up = strided(rows, cols, dtype).copy_(a), strided(rows, cols, dtype, cols + 3).copy_(b)
        g, u = gate.double(), up.double()
    out, h, ht = strided(rows, cols, dtype), pair(rows, cols), pair(cols, rows, E5M2)
    g8, u8 = pair(rows, cols), pair(rows, cols, E5M2)
    ecq.ecq_act8_gate(gate, up, out, h, ht, g8, u8)
    want, err = gate64(g, u)[0], gate_error(g, u, dtype)
    check_plain(out, want, err, "out")
    check_pair(h, want, err, "out8")
    check_pair(ht, want.T.contiguous(), err.T.contiguous(), "out8_t")
    check_exactly(g8, g)
    check_exactly(u8, u)
    behind_is_left(h)
    behind_is_left(ht)


def test_gate_far_out():
    """Where exp over- and underflows the sigmoid is 0 or 1."""
    g = torch.tensor([[-3e38, -1e4, -200.0, -104.0, -88.0, 0.0, 88.0, 200.0, 3e38, 1e-40]], device="cuda")
    u, out = torch.ones_like(g), torch.empty_like(g)
    ecq.ecq_act8_gate(g, u, out)
    want = gate64(g.double(), u.double())[0]
    assert bool(((out.double() - want).abs() <= want.abs() * 2.0 ** -18 + 1e-35).all())


def gate_grad64(g, u, d):
    s = torch.sigmoid(g)
    return d * u * s * (1 + g * (1 - s)), d * g * s


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (5, 129), (128, 128), (130, 300), (257, 1001)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("kept", [False, True])
def test_gate_grad(rows, cols, dtype, kept):
    size = 0.1 if dtype == F16 else 1.0
    a, b = random(rows, cols, 3, 2 * size), random(rows, cols, 4, size)
    if kept:
        gate, up = stored(a, E5M2), stored(b, E5M2)
        g, u = values(gate), values(up)
    else:
        gate, up = strided(rows, cols, dtype, cols + 1).copy_(a), strided(rows, cols, dtype).copy_(b)
        g, u = gate.double(), up.double()
    d = strided(rows, cols, dtype).copy_(random(rows, cols, 5, size))
    outs = dict(d_gate=strided(rows, cols, dtype), d_up=strided(rows, cols, dtype, cols + 5), d_gate8=pair(rows, cols),
                d_gate8_t=pair(cols, rows), d_up8=pair(rows, cols, E5M2), d_up8_t=pair(cols, rows))
    ecq.ecq_act8_gate_grad(gate, up, d, **outs)
    dg, du = gate_grad64(g, u, d.double())
    s = torch.sigmoid(g)
    rel = 2.0 ** -20 + (0 if dtype == F32 else 1) * g.abs() * 2.0 ** -23
    # 1 - s and the sum with 1 are rounded (or cancel) at the size of their parts
    eg = (d.double() * u).abs() * s * (1 + g.abs() * (1 - s) + g.abs() * 2.0 ** -2) * rel
    eg = eg + (d.double() * u).abs() * (1 + g.abs()) * 2.0 ** -126 + 2.0 ** -126      # sigmoids below 2^-126 are 0
    eu = du.abs() * rel + (d.double() * g).abs() * 2.0 ** -126 + 2.0 ** -126
    for name, want, err in (("gate", dg, eg), ("up", du, eu)):
        check_plain(outs["d_" + name], want, err, name)
        check_pair(outs["d_%s8" % name], want, err, name + "8")
        check_pair(outs["d_%s8_t" % name], want.T.contiguous(), err.T.contiguous(), name + "8_t")
        behind_is_left(outs["d_%s8_t" % name])


def test_gate_grad_against_differences():
    g, u, d = (random(7, 130, i).float() for i in (20, 21, 22))
    dg, du = torch.empty_like(g), torch.empty_like(g)
    ecq.ecq_act8_gate_grad(g, u, d, dg, du)
    step = 1e-6
    f = lambda g, u: (gate64(g, u)[0] * d.double())
    for got, num in ((dg, (f(g.double() + step, u.double()) - f(g.double() - step, u.double())) / (2 * step)),
                     (du, (f(g.double(), u.double() + step) - f(g.double(), u.double() - step)) / (2 * step))):
        # central differences: step^2 of the third derivative, and 2^-52 / step of the values
        scale = (d.double().abs() * (u.double().abs() + 1) * (g.double().abs() + 1))
        assert bool(((got.double() - num).abs() <= 1e-5 * scale).all())


def test_gate_in_place():
    g, u = random(70, 200, 1).to(BF16), random(70, 200, 2).to(BF16)
    want = torch.empty_like(g)
    ecq.ecq_act8_gate(g, u, want)
    ecq.ecq_act8_gate(g, u, g)
    assert torch.equal(g, want)


def gate_parts(P, lo, hi, kept):
    """Rows lo .. hi - 1 of a plain matrix, or of a pair as one of its own."""
    if not kept:
        return P[lo:hi]
    p = pair(hi - lo, P[0].shape[1], P[0].dtype)
    p[0].view(torch.uint8).copy_(P[0].view(torch.uint8)[lo:hi])
    p[1][scale_places(*p[0].shape)] = scale_bytes(P)[lo:hi]
    return p


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("kept", [False, True])
def test_many_tiles_are_as_few(dtype, kept):
    """Enough tiles that those ahead are on their way, whole ones and ones at both edges: bit for bit what calls on 512 rows
    give (which the tests above hold to 64 bits)."""
    rows, cols = 5000, 4008
    x = strided(rows, cols, dtype).copy_(random(rows, cols, 51))
    u = strided(rows, cols, dtype).copy_(random(rows, cols, 52))
    d = strided(rows, cols, dtype).copy_(random(rows, cols, 53))
    g8, u8 = pair(rows, cols, E5M2), pair(rows, cols, E5M2)
    ecq.ecq_act8_store(x, g8)
    ecq.ecq_act8_store(u, u8)
    a, b = (g8, u8) if kept else (x, u)

    def calls(a, b, d, rows):
        plain = [strided(rows, cols, dtype) for _ in range(4)]
        q = [pair(rows, cols, k) for k in (E4M3, E5M2, E4M3, E5M2, E4M3, E4M3)]
        t = [pair(cols, rows, k) for k in (E4M3, E5M2, E4M3, E5M2)]
        ecq.ecq_act8_store(a, q[0], t[0])
        if kept:
            ecq.ecq_act8_load(a, plain[0])
        else:
            plain[0].copy_(a)
        ecq.ecq_act8_gate(a, b, plain[1], q[1], t[1], q[4], q[5])
        ecq.ecq_act8_gate_grad(a, b, d, plain[2], plain[3], q[2], t[2], q[3], t[3])
        return plain, q, t

    plain, q, t = calls(a, b, d, rows)
    for p in q + t:
        behind_is_left(p)
    for lo in range(0, rows, 512):
        hi = min(rows, lo + 512)
        few = calls(gate_parts(a, lo, hi, kept), gate_parts(b, lo, hi, kept), d[lo:hi], hi - lo)
        for one, all_of in zip(few[0], plain):
            assert torch.equal(one, all_of[lo:hi])
        for one, all_of in zip(few[1], q):
            assert torch.equal(bytes_of(one)[:, :cols], bytes_of(all_of)[lo:hi, :cols])
            assert torch.equal(scale_bytes(one), scale_bytes(all_of)[lo:hi])
        for one, all_of in zip(few[2], t):
            assert torch.equal(bytes_of(one)[:, :hi - lo], bytes_of(all_of)[:, lo:hi])
            assert torch.equal(scale_bytes(one), scale_bytes(all_of)[:, lo // 128:(hi + 127) // 128])


def test_tiles_that_do_not_come_in_time_are_read_from_memory():
    x = random(5000, 4000, 61).to(BF16)
    q, t, late, late_t = pair(5000, 4000), pair(4000, 5000), pair(5000, 4000), pair(4000, 5000)
    ecq.ecq_act8_store(x, q, t)
    ecq.ecq_act8_set_wait_limit(0)
    try:
        ecq.ecq_act8_store(x, late, late_t)
        torch.cuda.synchronize()
    finally:
        ecq.ecq_act8_set_wait_limit()
    for a, b in ((q, late), (t, late_t)):
        assert torch.equal(bytes_of(a), bytes_of(b)) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("rows,cols,stride", [(70, 200, 200), (70, 201, 203), (5000, 1024, 1024)])
def test_gate_gradient_in_place(rows, cols, stride):
    g, u, d = (strided(rows, cols, BF16, stride).copy_(random(rows, cols, k)) for k in (1, 2, 3))
    dg, du = strided(rows, cols, BF16, stride), strided(rows, cols, BF16, stride)
    ecq.ecq_act8_gate_grad(g, u, d, dg, du)
    ecq.ecq_act8_gate_grad(g, u, d, g, u)
    assert torch.equal(g, dg) and torch.equal(u, du)
    ecq.ecq_act8_gate_grad(dg, du, d, g, u)
    ecq.ecq_act8_gate_grad(dg, du, d, d)
    assert torch.equal(d, g)


# ---- norm ------------------------------------------------------------------------------------------

NORM_SIZES = [(1, 1), (1, 7), (3, 8), (2, 200), (9, 256), (33, 513), (700, 1024), (1, 4096), (5, 4097), (3, 8192), (2, 12001),
              (1, 16384), (20000, 64)]
# per thread up to 32 squares one after the other, ten levels of sums, and a few products
NORM_REL = 64 * 2.0 ** -24


@pytest.mark.parametrize("rows,cols", NORM_SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("residual", [False, True])
def test_norm(rows, cols, dtype, residual):
    x = strided(rows, cols, dtype, cols + 1, 1).copy_(random(rows, cols, 31, 0.2))
    r = strided(rows, cols, dtype).copy_(random(rows, cols, 32, 0.2)) if residual else None
    w = random(1, cols, 33)[0].to(dtype if cols % 2 else F32)
    total, y, y8, s8 = strided(rows, cols, dtype, cols + 2), strided(rows, cols, dtype), pair(rows, cols), pair(rows, cols, E5M2)
    rstd = torch.full((rows,), 7.0, device="cuda")
    ecq.ecq_act8_norm(x, r, w, eps=1e-5, sum=total, out=y, out8=y8, sum8=s8, rstd=rstd)
    s = x.double() + (r.double() if residual else 0.0)
    s_err = s.abs() * 2.0 ** -24
    f = 1 / torch.sqrt(s.square().mean(1) + 1e-5)
    assert bool(((rstd.double() - f).abs() <= f * NORM_REL).all())
    want = s * f[:, None] * w.double()
    check_plain(total, s, s_err, "sum")
    check_plain(y, want, want.abs() * NORM_REL, "out")
    check_pair(y8, want, want.abs() * NORM_REL, "out8")
    check_pair(s8, s, s_err, "sum8")
    behind_is_left(y8)
    behind_is_left(s8)


@pytest.mark.parametrize("rows,cols", [(2600, 1024), (1300, 4096), (700, 5128), (700, 8192), (500, 16384), (6000, 200), (4000, 520), (1500, 2560)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("coded", [False, True])
def test_norm_of_many_aligned_rows(rows, cols, dtype, residual, coded):
    x = strided(rows, cols, dtype).copy_(random(rows, cols, 31, 0.2))
    r = strided(rows, cols, dtype, cols + 8).copy_(random(rows, cols, 32, 0.2)) if residual else None
    w = random(1, cols, 33)[0].float()
    total, y, rstd = strided(rows, cols, dtype), strided(rows, cols, dtype, cols + 16), torch.full((rows,), 7.0, device="cuda")
    y8 = pair(rows, cols) if coded else None
    ecq.ecq_act8_norm(x, r, w, eps=1e-5, sum=total, out=y, out8=y8, rstd=rstd)
    s = x.double() + (r.double() if residual else 0.0)
    f = 1 / torch.sqrt(s.square().mean(1) + 1e-5)
    want = s * f[:, None] * w.double()
    assert bool(((rstd.double() - f).abs() <= f * NORM_REL).all())
    check_plain(total, s, s.abs() * 2.0 ** -24, "sum")
    check_plain(y, want, want.abs() * NORM_REL, "out")
    if coded:
        check_pair(y8, want, want.abs() * NORM_REL, "out8")


def test_norm_without_a_weight_and_zero_rows():
    x = random(5, 300, 1).float()
    x[2] = 0.0
    y, y8, rstd = torch.empty_like(x), pair(5, 300), torch.empty(5, device="cuda")
    ecq.ecq_act8_norm(x, eps=1e-6, out=y, out8=y8, rstd=rstd)
    assert bool((y[2] == 0).all()) and abs(rstd[2].item() - 1000.0) < 0.01
    want = x.double() / torch.sqrt(x.double().square().mean(1, keepdim=True) + 1e-6)
    check_plain(y, want, want.abs() * NORM_REL)
    assert bool((scale_bytes(y8)[2] == 0).all())


def test_norm_of_rows_with_nan_leaves_the_others():
    x = random(40, 700, 1).float()
    clean = x.clone()
    x[3, 9], x[20, 699] = math.nan, math.inf
    y, z, y8 = torch.empty_like(x), torch.empty_like(x), pair(40, 700)
    ecq.ecq_act8_norm(x, out=y, out8=y8)
    ecq.ecq_act8_norm(clean, out=z)
    rest = [i for i in range(40) if i not in (3, 20)]
    assert torch.equal(y[rest], z[rest]) and bool(torch.isnan(y[3]).all()) and bool((scale_bytes(y8)[3] == 255).all())
    assert bool((scale_bytes(y8)[rest] < 255).all())


def test_norm_in_place():
    x, r = random(300, 500, 1).to(BF16), random(300, 500, 2).to(BF16)
    s, y = torch.empty_like(x), torch.empty_like(x)
    ecq.ecq_act8_norm(x, r, sum=s, out=y)
    ecq.ecq_act8_norm(x, r, sum=r, out=x)
    assert torch.equal(s, r) and torch.equal(x, y)


@pytest.mark.parametrize("rows,cols", NORM_SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("kept", [False, True])
def test_norm_grad(rows, cols, dtype, kept):
    x = random(rows, cols, 41, 0.3)
    if kept:
        saved = stored(x)
        s = values(saved)
    else:
        saved = strided(rows, cols, dtype, cols + 1).copy_(x)
        s = saved.double()
    w = random(1, cols, 42)[0].float()
    d = strided(rows, cols, dtype, cols + 3, 3).copy_(random(rows, cols, 43, 0.1))
    d_sum = strided(rows, cols, dtype).copy_(random(rows, cols, 44, 0.1)) if rows % 2 else None
    rstd = (1 / torch.sqrt(s.square().mean(1) + 1e-5)).float()
    d_x, d_w = strided(rows, cols, dtype, cols + 2), torch.full((cols,), 7.0, device="cuda")
    work = torch.full((ecq.ecq_act8_norm_grad_workspace_bytes(rows, cols),), 0xFF, dtype=torch.uint8, device="cuda")
    ecq.ecq_act8_norm_grad(saved, w, rstd, d, d_x, d_w, work, d_sum=d_sum)
    f = rstd.double()[:, None]
    n, g = s * f, d.double() * w.double()
    want = f * (g - n * (g * n).mean(1, keepdim=True))
    err = f * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True)) * NORM_REL
    if d_sum is not None:
        want = want + d_sum.double()
    check_plain(d_x, want, err + want.abs() * 2.0 ** -23, "d_x")
    terms = d.double() * n
    assert bool(((d_w.double() - terms.sum(0)).abs() <= terms.abs().sum(0) * (rows + 64) * 2.0 ** -24 + 1e-37).all())
    again = torch.empty_like(d_w)
    ecq.ecq_act8_norm_grad(saved, w, rstd, d, None, again, work)
    assert torch.equal(d_w, again)


@pytest.mark.parametrize("rows,cols", [(2600, 1024), (700, 4096), (500, 5128), (300, 8192), (300, 16384), (6000, 200), (4000, 520), (1500, 2560)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("kept", [False, True])
def test_norm_gradient_of_many_aligned_rows(rows, cols, dtype, kept):
    x = random(rows, cols, 41, 0.3)
    saved = stored(x) if kept else strided(rows, cols, dtype, cols + 8).copy_(x)
    s = values(saved) if kept else saved.double()
    w = random(1, cols, 42)[0].float()
    d, d_sum = strided(rows, cols, dtype).copy_(random(rows, cols, 43, 0.1)), strided(rows, cols, dtype).copy_(random(rows, cols, 44, 0.1))
    rstd = (1 / torch.sqrt(s.square().mean(1) + 1e-5)).float()
    d_x, d_w = strided(rows, cols, dtype), torch.full((cols,), 7.0, device="cuda")
    work = torch.full((ecq.ecq_act8_norm_grad_workspace_bytes(rows, cols),), 0xFF, dtype=torch.uint8, device="cuda")
    ecq.ecq_act8_norm_grad(saved, w, rstd, d, d_x, d_w, work, d_sum=d_sum)
    f = rstd.double()[:, None]
    n, g = s * f, d.double() * w.double()
    want = f * (g - n * (g * n).mean(1, keepdim=True)) + d_sum.double()
    err = f * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True)) * NORM_REL
    check_plain(d_x, want, err + want.abs() * 2.0 ** -23, "d_x")
    terms = d.double() * n
    assert bool(((d_w.double() - terms.sum(0)).abs() <= terms.abs().sum(0) * (rows + 64) * 2.0 ** -24 + 1e-37).all())


@pytest.mark.parametrize("rows,cols,stride", [(300, 500, 500), (300, 1001, 1003), (3000, 1024, 1024), (2, 9000, 9001)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_gradient_in_place(rows, cols, stride, dtype):
    s, d, e = (strided(rows, cols, dtype, stride).copy_(random(rows, cols, k)) for k in (1, 2, 3))
    w, rstd = random(1, cols, 4)[0].float(), torch.rand(rows, device="cuda") + 0.5
    work = torch.empty(ecq.ecq_act8_norm_grad_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    want, dw = strided(rows, cols, dtype, stride), torch.empty(cols, device="cuda")
    ecq.ecq_act8_norm_grad(s, w, rstd, d, want, dw, work, d_sum=e)
    for place in (0, 1, 2):
        x = [strided(rows, cols, dtype, stride).copy_(y) for y in (s, d, e)]
        again = torch.empty_like(dw)
        ecq.ecq_act8_norm_grad(x[0], w, rstd, x[1], x[place], again, work, d_sum=x[2])
        assert torch.equal(x[place], want) and torch.equal(again, dw)


def test_norm_grad_is_the_formulas_derivative():
    """Against autograd in 64 bits of the norm itself."""
    x = random(6, 300, 1)
    w = random(1, 300, 2)[0]
    d = random(6, 300, 3)
    leaf, wl = x.float().double().requires_grad_(), w.float().double().requires_grad_()
    f = 1 / torch.sqrt(leaf.square().mean(1, keepdim=True) + 1e-6)
    (leaf * f * wl * d.float().double()).sum().backward()
    d_x, d_w = torch.empty(6, 300, device="cuda"), torch.empty(300, device="cuda")
    work = torch.empty(ecq.ecq_act8_norm_grad_workspace_bytes(6, 300), dtype=torch.uint8, device="cuda")
    ecq.ecq_act8_norm_grad(x.float(), w.float(), f.detach()[:, 0].float(), d.float(), d_x, d_w, work)
    assert bool(((d_x.double() - leaf.grad).norm() <= 1e-6 * leaf.grad.norm()))
    assert bool(((d_w.double() - wl.grad).norm() <= 1e-6 * wl.grad.norm()))


def test_norm_grad_of_no_rows_zeroes_the_weights():
    d_w = torch.full((300,), 3.0, device="cuda")
    e = torch.empty(0, 300, device="cuda")
    ecq.ecq_act8_norm_grad(e, None, torch.empty(0, device="cuda"), e, None, d_w, None)
    assert bool((d_w == 0).all())


# ---- no rows, refusals -----------------------------------------------------------------------------

def test_no_rows_is_nothing_to_do():
    e, q, t = torch.empty(0, 300, device="cuda"), pair(0, 300), (torch.empty(300, 0, dtype=torch.uint8, device="cuda").view(E4M3),
                                                                torch.empty(0, dtype=torch.uint8, device="cuda"))
    before = ecq.ecq_launch_count()
    ecq.ecq_act8_store(e, q, t)
    ecq.ecq_act8_gate(e, e, out8=q)
    ecq.ecq_act8_norm(e, out8=q)
    assert ecq.ecq_launch_count() == before


def test_binding_refuses_wrong_shapes_types_and_devices():
    x, q = torch.zeros(40, 300, device="cuda"), pair(40, 300)
    for call in (lambda: ecq.ecq_act8_store(x, pair(40, 301)), lambda: ecq.ecq_act8_store(x.double(), q),
                 lambda: ecq.ecq_act8_store(x.cpu(), q), lambda: ecq.ecq_act8_store(x, (q[0], q[1][:-1])),
                 lambda: ecq.ecq_act8_store(x, (q[0].view(torch.uint8), q[1])), lambda: ecq.ecq_act8_store(x.T, pair(300, 40)),
                 lambda: ecq.ecq_act8_store(x, q, pair(40, 300)), lambda: ecq.ecq_act8_norm(x, out=torch.zeros(40, 299, device="cuda")),
                 lambda: ecq.ecq_act8_norm(x, weight=torch.ones(299, device="cuda"), out=x),
                 lambda: ecq.ecq_act8_store(torch.zeros(1, 300, device="cuda").expand(40, 300), q)):
        with pytest.raises(ValueError):
            call()
    odd = (torch.zeros(40, 300, dtype=torch.uint8, device="cuda").view(E4M3), q[1])            # rows not on 16 bytes
    for call in (lambda: ecq.ecq_act8_store(x, odd), lambda: ecq.ecq_act8_store(x, None, None),
                 lambda: ecq.ecq_act8_gate(x, x.to(BF16), x), lambda: ecq.ecq_act8_norm(x, out=x.to(BF16)),
                 lambda: ecq.ecq_act8_norm(x, eps=-1.0, out=x)):
        with pytest.raises(ecq.EcqError):
            call()
