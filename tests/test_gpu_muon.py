"""Newton-Schulz orthogonalisation and the momentum step around it against the definitions in 64 bits.

Tolerances, relative in the 2-norm.  ECQ_MUON_HALF: the operands of the products carry 2^-12 of
rounding each; emulated in 64 bits on spectra from flat to 1/i^1.5 the result is 3e-4 to 1.1e-3 off
with five default steps: 3e-3, and the output type's own rounding on top.  ECQ_MUON_SPLIT: operands
carry 2^-23, which scales to 5e-7, and the fp32 accumulators of sums of up to 2048 terms and the
fp32 epilogues a few 1e-6 after five steps: 2e-5.
"""
import math

import pytest
import torch

import paper_1806_08054_b200 as ecq

pytestmark = pytest.mark.gpu
QUINTIC = (3.4445, -4.7750, 2.0315)
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ROUND = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
HALF, SPLIT = 3e-3, 2e-5
TILES = {"256x256": ecq.ECQ_MUON_TILES_256X256, "128x128": ecq.ECQ_MUON_TILES_128X128,
         "128x64": ecq.ECQ_MUON_TILES_128X64}


def polar(u, coefficients):
    u = u.double()
    norm = u.norm()
    x = u / norm if norm > 0 else u
    for a, b, c in coefficients:
        if x.shape[0] <= x.shape[1]:
            g = x @ x.T
            x = a * x + (b * g + c * g @ g) @ x
        else:
            g = x.T @ x
            x = a * x + x @ (b * g + c * g @ g)
    return x


class Plan:
    def __init__(self, shapes, gap=0, strides=None, tiles=0, precision=0, scales=None, steps=5, coefficients=None, first=0):
        self.shapes, self.offsets, at = shapes, [], first
        self.strides = strides or [c for _, c in shapes]
        for (r, c), s in zip(shapes, self.strides):
            self.offsets.append(at)
            at += (r - 1) * s + c + gap
        self.length = at
        self.coefficients = coefficients or [QUINTIC] * steps
        self.scales = scales or [1.0] * len(shapes)
        self.h = ecq.ecq_muon_create(self.offsets, [s[0] for s in shapes], [s[1] for s in shapes], strides=strides,
                                     scales=scales, steps=steps, coefficients=coefficients, precision=precision)
        ecq.ecq_muon_set_tiles(self.h, tiles)
        n = ecq.ecq_muon_workspace_bytes(self.h)
        self.guarded = torch.full((n + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        # what an earlier use may have left there: NaN patterns everywhere
        self.guarded[256:256 + n] = 0xFF
        ecq.ecq_muon_bind(self.h, self.guarded[256:256 + n])

    def views(self, flat):
        return [flat[o:].as_strided((r, c), (s, 1)) for (r, c), o, s in zip(self.shapes, self.offsets, self.strides)]

    def outside(self):
        mask = torch.ones(self.length, dtype=torch.bool, device="cuda")
        for v in self.views(mask):
            v.fill_(False)
        return mask

    def close(self):
        assert torch.all(self.guarded[:256] == 0xA5) and torch.all(self.guarded[-256:] == 0xA5), "write outside the workspace"
        assert ecq.ecq_muon_status(self.h) == ecq.ECQ_OK
        ecq.ecq_muon_destroy(self.h)


def data(plan, seed=0, kind="real", dtype=torch.float32):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    flat = torch.randn(plan.length, generator=gen, device="cuda") * 1e-4
    if kind == "real":
        for v in plan.views(flat):
            k = min(4, *v.shape)
            v += 3e-4 * torch.randn(v.shape[0], k, generator=gen, device="cuda") @ torch.randn(k, v.shape[1], generator=gen, device="cuda")
    return flat.to(dtype)


def far(x, ref):
    return ((x.double() - ref).norm() / ref.norm()).item()


def check_orth(plan, src, dst="f32", tol=SPLIT):
    out = torch.full((plan.length,), 5.0, dtype=DT[dst], device="cuda")
    ecq.ecq_muon_orthogonalize(plan.h, src, out)
    for x, y in zip(plan.views(src), plan.views(out)):
        assert far(y, polar(x, plan.coefficients)) <= tol + ROUND[dst], x.shape
    assert torch.all(out[plan.outside()] == 5.0), "write outside the matrices"
    return out


SIZES = [(1, 1), (1, 9), (9, 1), (2, 2), (3, 65), (64, 64), (65, 64), (127, 129), (128, 128), (129, 257), (257, 127),
         (300, 1000), (1000, 300), (512, 512), (611, 1537)]


@pytest.mark.parametrize("tiles", list(TILES))
@pytest.mark.parametrize("rows,cols", SIZES)
def test_sizes(rows, cols, tiles):
    for precision, dst, tol in ((ecq.ECQ_MUON_HALF, "bf16", HALF), (ecq.ECQ_MUON_SPLIT, "f32", SPLIT)):
        plan = Plan([(rows, cols)], tiles=TILES[tiles], precision=precision)
        check_orth(plan, data(plan, rows + cols), dst, tol)
        plan.close()


@pytest.mark.parametrize("shapes", [[(2497, 85)], [(40, 9001)], [(9001, 40)], [(128, 4096)], [(1000, 1333)], [(64, 7000)],
                                    [(70, 5000), (5000, 130), (1, 9000), (129, 4100)]], ids=str)
def test_few_tiles_and_long_products(shapes):
    """Where two CTAs share the sums of a tile; for the smallest of them one of the two has nothing to add."""
    for precision, dst, tol in ((ecq.ECQ_MUON_HALF, "bf16", HALF), (ecq.ECQ_MUON_SPLIT, "f32", SPLIT)):
        plan = Plan(shapes, gap=3, precision=precision)
        src = data(plan, 11)
        first = check_orth(plan, src, dst, tol)
        for _ in range(20):
            again = torch.full_like(first, 5.0)
            ecq.ecq_muon_orthogonalize(plan.h, src, again)
            assert torch.equal(first, again)
        plan.close()


@pytest.mark.parametrize("tiles", list(TILES))
def test_many_matrices_odd_offsets_and_strides(tiles):
    shapes = [(96, 160), (31, 700), (260, 130), (1, 50), (64, 64), (513, 300), (17, 17), (300, 513)]
    strides = [c + k for (_, c), k in zip(shapes, (0, 4, 1, 3, 0, 5, 64, 0))]
    plan = Plan(shapes, gap=37, strides=strides, tiles=TILES[tiles], first=3)
    for dtype in DT:
        check_orth(plan, data(plan, 5, dtype=DT[dtype]), "f32", SPLIT)
    plan.close()


@pytest.mark.parametrize("src", list(DT))
@pytest.mark.parametrize("dst", list(DT))
def test_types(src, dst):
    plan = Plan([(200, 333), (333, 200)], gap=1)
    a = check_orth(plan, data(plan, 1, dtype=DT[src]), dst, HALF if dst == "bf16" else SPLIT)
    if src == dst:                                          # in place
        x = data(plan, 1, dtype=DT[src])
        ecq.ecq_muon_orthogonalize(plan.h, x, x)
        for u, v in zip(plan.views(x), plan.views(a)):
            assert torch.equal(u, v)
    plan.close()


@pytest.mark.parametrize("size", [1e-30, 1e-18, 1.0, 1e18, 1e30])
def test_any_magnitude(size):
    """Squares of the entries would vanish or overflow in 32 bits; the result does not depend on them."""
    plan = Plan([(70, 190)])
    src = data(plan, 2)
    want = [polar(v, plan.coefficients) for v in plan.views(src)]
    out = torch.empty_like(src)
    ecq.ecq_muon_orthogonalize(plan.h, src / 1e-4 * size, out)
    assert far(plan.views(out)[0], want[0]) <= 2 * SPLIT
    plan.close()


@pytest.mark.parametrize("spectrum", ["flat", "1/i^0.5", "1/i", "1/i^1.5", "rank one"])
def test_spectra(spectrum):
    m, n = 256, 640
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    u, _ = torch.linalg.qr(torch.randn(m, m, generator=gen, device="cuda", dtype=torch.float64))
    v, _ = torch.linalg.qr(torch.randn(n, m, generator=gen, device="cuda", dtype=torch.float64))
    i = torch.arange(1, m + 1, device="cuda", dtype=torch.float64)
    s = {"flat": i ** 0, "1/i^0.5": i ** -0.5, "1/i": 1 / i, "1/i^1.5": i ** -1.5, "rank one": (i == 1).double()}[spectrum]
    x = ((u * s) @ v.T).float()
    for precision, tol in ((ecq.ECQ_MUON_HALF, HALF), (ecq.ECQ_MUON_SPLIT, SPLIT)):
        if spectrum == "rank one":
            tol *= 20       # the rest of the spectrum is the input's own rounding, amplified 480 times
        plan = Plan([(m, n)], precision=precision)
        check_orth(plan, x.reshape(-1).contiguous(), "f32", tol)
        plan.close()


def test_steps_and_coefficients():
    other = [(1.5, -0.5, 0.0), (2.0, -1.5, 0.5), (3.4445, -4.7750, 2.0315), (15 / 8, -10 / 8, 3 / 8)]
    for coefficients in (other[:1], other[1:3], other, [(1.875, -1.25, 0.375)] * 12):
        plan = Plan([(90, 140), (140, 90)], steps=len(coefficients), coefficients=coefficients)
        check_orth(plan, data(plan, 6), "f32", 2 * SPLIT)
        plan.close()


@pytest.mark.parametrize("coefficients", [[(0.1, 0.0, 0.0), (1.0, 0.0, 0.0), (10.0, 5000.0, 0.0)],
                                          [(0.1, 0.0, 0.0), (2.0, 0.0, 0.0), (3.0, 400.0, -300.0), (0.5, -0.02, 0.001)],
                                          [(0.05, 0.0, 0.0), (1.0, 0.0, 0.0), (10.0, 100.0, 0.0)],
                                          [(0.2, 0.0, 0.0), (1.0, 0.0, 0.0), (1.0, 60.0, 60.0)]], ids=str)
def test_coefficients_whose_iterates_stay_small(coefficients):
    """The last steps' polynomial is large only for singular values that do not occur: it is neither to
    leave the range of the 16-bit copies nor to take their rounding to the result."""
    for precision, tol in ((ecq.ECQ_MUON_HALF, HALF), (ecq.ECQ_MUON_SPLIT, SPLIT)):
        plan = Plan([(90, 140), (300, 700)], steps=len(coefficients), coefficients=coefficients, precision=precision)
        check_orth(plan, data(plan, 6), "f32", tol)
        plan.close()


def test_zero_matrix_and_nan_matrix():
    plan = Plan([(40, 50), (64, 64), (50, 40), (30, 30)], gap=3)
    grad, mom, par = data(plan, 1), data(plan, 2), data(plan, 3)
    plan.views(grad)[0].zero_(); plan.views(mom)[0].zero_()
    plan.views(grad)[1][3, 5] = math.nan
    plan.views(mom)[2][7, 7] = math.inf
    before = [t.clone() for t in (grad, mom, par)]
    upd = torch.full_like(grad, 5.0)
    ecq.ecq_muon_step(plan.h, grad, mom, par, upd, mu=0.9, lr=0.1, decay=0.1)
    assert ecq.ecq_muon_status(plan.h) == ecq.ECQ_ERR_NONFINITE
    assert ecq.ecq_muon_status(plan.h) == ecq.ECQ_OK
    for k in (1, 2):                                        # left alone
        assert torch.equal(plan.views(mom)[k].isfinite(), plan.views(before[1])[k].isfinite())
        assert torch.equal(plan.views(par)[k], plan.views(before[2])[k])
        assert torch.equal(torch.nan_to_num(plan.views(mom)[k]), torch.nan_to_num(plan.views(before[1])[k]))
        assert torch.all(plan.views(upd)[k] == 0)
    assert torch.all(plan.views(upd)[0] == 0) and torch.all(plan.views(mom)[0] == 0)
    assert torch.allclose(plan.views(par)[0], plan.views(before[2])[0] * 0.99, rtol=1e-6, atol=0)
    m3 = 0.9 * plan.views(before[1])[3].double() + plan.views(grad)[3].double()
    assert far(plan.views(upd)[3], polar(plan.views(grad)[3].double() + 0.9 * m3, plan.coefficients)) <= SPLIT
    assert torch.equal(torch.nan_to_num(grad), torch.nan_to_num(before[0]))
    plan.close()


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("gap", [0, 3])
def test_step(nesterov, gap):
    """Three steps: momentum, weights and the emitted update, and nothing beside the matrices."""
    shapes = [(100, 260), (260, 100), (64, 128), (33, 47)]
    scales = [0.2 * math.sqrt(max(s)) for s in shapes]
    plan = Plan(shapes, gap=gap, scales=scales)
    mom, par = data(plan, 1), 0.02 * torch.randn(plan.length, device="cuda")
    upd = torch.full((plan.length,), 5.0, device="cuda")
    m64, p64 = mom.double(), par.double()
    outside = plan.outside()
    keep = [t[outside].clone() for t in (mom, par, upd)]
    for t in range(3):
        grad = data(plan, 10 + t)
        ecq.ecq_muon_step(plan.h, grad, mom, par, upd, mu=0.95, nesterov=nesterov, lr=0.02, decay=0.1)
        for v, w, g, mv, pv, uv, s in zip(plan.views(m64), plan.views(p64), plan.views(grad), plan.views(mom),
                                          plan.views(par), plan.views(upd), scales):
            v.mul_(0.95).add_(g.double())
            o = s * polar(g.double() + 0.95 * v if nesterov else v, plan.coefficients)
            w.mul_(1 - 0.02 * 0.1).sub_(0.02 * o)
            assert far(mv, v) <= 4 * 2.0 ** -24 * (t + 1)
            assert far(uv, o) <= SPLIT
            # lr times the update's error, and 3 roundings of the weights a step
            assert (pv.double() - w).norm() <= (t + 1) * (0.02 * SPLIT * o.norm() + 3 * 2.0 ** -24 * w.norm())
    assert all(torch.equal(t[outside], k) for t, k in zip((mom, par, upd), keep))
    only = torch.zeros_like(par)
    m2, p2 = mom.clone(), par.clone()
    grad = data(plan, 99)
    ecq.ecq_muon_step(plan.h, grad, m2, p2, None, mu=0.95, nesterov=nesterov, lr=0.02, decay=0.1)
    m3, p3 = mom.clone(), par.clone()
    ecq.ecq_muon_step(plan.h, grad, m3, p3, only, mu=0.95, nesterov=nesterov, lr=0.02, decay=0.1)
    assert torch.equal(m2, m3) and torch.equal(p2, p3)
    bf = torch.zeros(plan.length, dtype=torch.bfloat16, device="cuda")
    m4 = mom.clone()
    ecq.ecq_muon_step(plan.h, grad, m4, None, bf, mu=0.95, nesterov=nesterov)
    assert torch.equal(m4, m3)
    for u, v in zip(plan.views(bf), plan.views(only)):
        assert far(u, v.double()) <= HALF + ROUND["bf16"]
    plan.close()


@pytest.mark.parametrize("tiles", list(TILES))
def test_repeatable_back_to_back_and_on_another_stream(tiles):
    """Calls enqueued one after the other on a plan's workspace give what each gives alone."""
    plan = Plan([(384, 1100), (500, 500), (257, 130)], gap=1, tiles=TILES[tiles])
    srcs = [data(plan, k) for k in range(3)]
    alone = [check_orth(plan, s) for s in srcs]
    outs = [torch.full_like(a, 5.0) for a in alone]
    for _ in range(3):
        for s, o in zip(srcs, outs):
            ecq.ecq_muon_orthogonalize(plan.h, s, o)
    assert all(torch.equal(a, o) for a, o in zip(alone, outs))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        ecq.ecq_muon_orthogonalize(plan.h, srcs[1], outs[0])
    stream.synchronize()
    assert torch.equal(outs[0], alone[1])
    plan.close()


@pytest.mark.parametrize("rows,cols", [(64, 200_001), (64, 1 << 20), (1 << 20, 50)])
def test_very_long_sums(rows, cols):
    """The rounding errors of long sums do not reach the result, whatever the operands' precision."""
    for precision, tol in ((ecq.ECQ_MUON_HALF, HALF), (ecq.ECQ_MUON_SPLIT, SPLIT)):
        plan = Plan([(rows, cols)], precision=precision)
        src = data(plan, 7, kind="flat")
        check_orth(plan, src, "f32", tol)
        plan.close()


@pytest.mark.parametrize("tiles,precision", [(0, 1), (0, 2), (1, 1), (1, 2), (3, 1), (3, 2)])
def test_many_tiles_of_many_sizes_over_and_over(tiles, precision):
    """Numbers of tiles that two CTAs hand each other, with tiles that take from one step along K to dozens:
    200 calls with the same bits."""
    shapes = [(64, 147), (64, 64), (64, 576), (256, 64), (128, 1152), (512, 128), (256, 2304), (1024, 256), (85, 2497), (3, 4000),
              (700, 700)]
    plan = Plan(shapes, gap=1, tiles=tiles, precision=precision)
    src = data(plan, 4)
    first = torch.full_like(src, 5.0)
    ecq.ecq_muon_orthogonalize(plan.h, src, first)
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(200):
        again = torch.full_like(src, 5.0)
        ecq.ecq_muon_orthogonalize(plan.h, src, again)
        wrong += (again != first).sum()
    assert wrong.item() == 0
    plan.close()


@pytest.mark.parametrize("tiles", list(TILES))
def test_a_wait_that_runs_out_is_reported(tiles):
    plan = Plan([(300, 400)], tiles=TILES[tiles])
    src = data(plan, 1)
    want = check_orth(plan, src)
    ecq.ecq_muon_set_wait_limit(plan.h, 0)
    ecq.ecq_muon_orthogonalize(plan.h, src, torch.empty_like(src))
    assert ecq.ecq_muon_status(plan.h) == ecq.ECQ_ERR_TIMEOUT
    ecq.ecq_muon_set_wait_limit(plan.h, ecq.ECQ_WAIT_LIMIT_DEFAULT)
    assert torch.equal(check_orth(plan, src), want)
    plan.close()


@pytest.mark.parametrize("shape,tiles", [((2497, 85), 0), ((300, 1000), 1), ((128, 4096), 0), ((300, 1000), 2)])
def test_waits_that_run_out_in_the_middle_of_a_call(shape, tiles):
    """Whatever was on its way then is let land: the call ends with a status, and the next is right."""
    for precision in (ecq.ECQ_MUON_HALF, ecq.ECQ_MUON_SPLIT):
        plan = Plan([shape], tiles=tiles, precision=precision)
        src = data(plan, 1)
        want, out = torch.empty_like(src), torch.empty_like(src)
        ecq.ecq_muon_orthogonalize(plan.h, src, want)
        for limit in (0, 1, 5, 30, 200, 1000):
            ecq.ecq_muon_set_wait_limit(plan.h, limit)
            ecq.ecq_muon_orthogonalize(plan.h, src, out)
            status = ecq.ecq_muon_status(plan.h)
            assert status in (ecq.ECQ_OK, ecq.ECQ_ERR_TIMEOUT) and (limit or status == ecq.ECQ_ERR_TIMEOUT)
            ecq.ecq_muon_set_wait_limit(plan.h, ecq.ECQ_WAIT_LIMIT_DEFAULT)
            ecq.ecq_muon_orthogonalize(plan.h, src, out)
            assert torch.equal(out, want)
        plan.close()


def test_offsets_beyond_32_bits():
    first = (1 << 32) + 12345
    need = (first + 200 * 300) * 2
    if torch.cuda.mem_get_info()[0] < 3 * need:
        pytest.skip("not enough free memory")
    plan = Plan([(200, 300)], first=first)
    flat = torch.zeros(plan.length, dtype=torch.bfloat16, device="cuda")
    plan.views(flat)[0].copy_(torch.randn(200, 300, device="cuda"))
    want = polar(plan.views(flat)[0], plan.coefficients)
    ecq.ecq_muon_orthogonalize(plan.h, flat, flat)
    assert far(plan.views(flat)[0], want) <= HALF + ROUND["bf16"]
    plan.close()


def test_refusals():
    plan = Plan([(20, 30)])
    ok = data(plan)
    for bad in (ok[:-1], ok.double(), ok.cpu(), ok[1:]):
        with pytest.raises((ValueError, ecq.EcqError)):
            ecq.ecq_muon_orthogonalize(plan.h, bad, ok.clone())
    with pytest.raises(ecq.EcqError):
        ecq.ecq_muon_step(plan.h, ok, ok.clone(), None, None)
    with pytest.raises(ecq.EcqError):
        ecq.ecq_muon_step(plan.h, ok, ok, ok.clone(), None)
    for bad in (dict(mu=1.5), dict(mu=math.nan), dict(lr=-1.0), dict(decay=math.inf)):
        with pytest.raises(ecq.EcqError):
            ecq.ecq_muon_step(plan.h, ok, ok.clone(), ok.clone(), None, **bad)
    plan.close()
    loose = ecq.ecq_muon_create([0], [20], [30])
    with pytest.raises(ecq.EcqError):                       # not bound yet
        ecq.ecq_muon_orthogonalize(loose, ok, ok.clone())
    n = ecq.ecq_muon_workspace_bytes(loose)
    for bad in (torch.empty(n - 1, dtype=torch.uint8, device="cuda"), torch.empty(n + 512, dtype=torch.uint8, device="cuda")[16:]):
        with pytest.raises(ecq.EcqError):
            ecq.ecq_muon_bind(loose, bad)
    ecq.ecq_muon_destroy(loose)
    for bad in (dict(coefficients=[(40.0, 0.0, 0.0)] * 5), dict(coefficients=[(1.0, math.nan, 0.0)] * 5), dict(steps=0),
                dict(steps=65), dict(precision=3), dict(strides=[29]), dict(scales=[math.inf])):
        with pytest.raises(ecq.EcqError):
            ecq.ecq_muon_create([0], [20], [30], **bad)
    for rows, cols in ((0, 5), (5, 0), ((1 << 22) + 1, 2), (40000, 40000)):
        with pytest.raises(ecq.EcqError):
            ecq.ecq_muon_create([0], [rows], [cols])
