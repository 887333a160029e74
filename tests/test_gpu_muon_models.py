"""The orthogonaliser at the sizes of models and in the ways that programs call it: every tile shape
held to the error of its precision, plans of many groups, all of the step's outputs from every tile
shape, CUDA graphs, two plans at once.

Tolerances, relative in the 2-norm, against the definition in 64 bits.  11-bit operands: each is off by
2^-12 / sqrt(3) of itself on average, 1.4e-4; five steps of three products with two operands each
add up to sqrt(30) * 1.4e-4 = 8e-4 where all count alike, and small singular values are amplified while they
are rounded: twice that, 2e-3 with the sums' own.  Rank one: all of U in one singular value, whose
polynomial cancels (merged steps lose a factor of 41 of 2^-12): 1e-2, which is what the header says.
22-bit operands: 2e-5.
"""
import math

import pytest
import torch

import paper_1806_08054_b200 as ecq
from test_gpu_muon import DT, ROUND, SPLIT, TILES, Plan, check_orth, data, far, polar

pytestmark = pytest.mark.gpu
HALF = 2e-3


@pytest.mark.parametrize("tiles", list(TILES))
@pytest.mark.parametrize("rows,cols", [(512, 1300), (1024, 1024), (2048, 700), (1537, 1611), (128, 4096)])
@pytest.mark.parametrize("kind", ["real", "flat"])
def test_half_precision_of_every_tile_shape(rows, cols, tiles, kind):
    plan = Plan([(rows, cols)], tiles=TILES[tiles], precision=ecq.ECQ_MUON_HALF)
    check_orth(plan, data(plan, 3, kind), "f32", HALF)
    plan.close()


@pytest.mark.parametrize("rows,cols", [(4096, 4096), (4096, 11000), (20000, 4096), (8192, 1024)])
def test_wide_layers(rows, cols):
    for precision, tol in ((ecq.ECQ_MUON_HALF, HALF), (ecq.ECQ_MUON_SPLIT, SPLIT)):
        plan = Plan([(rows, cols)], precision=precision)
        check_orth(plan, data(plan, 5), "f32", tol)
        plan.close()


@pytest.mark.parametrize("rows,cols", [(256, 640), (640, 256), (200, 300), (1024, 4096), (1024, 1024)])
def test_rank_one(rows, cols):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(8)
    x = torch.randn(rows, 1, generator=gen, device="cuda") * torch.randn(1, cols, generator=gen, device="cuda")
    for dst in ("f32", "bf16"):
        plan = Plan([(rows, cols)], precision=ecq.ECQ_MUON_HALF)
        out = torch.empty(rows * cols, dtype=DT[dst], device="cuda")
        ecq.ecq_muon_orthogonalize(plan.h, x.reshape(-1), out)
        u = x.double() / x.double().norm()                  # only its direction: the rest is the input's rounding
        want = polar(u, plan.coefficients)
        along = (out.view(rows, cols).double() * u).sum()
        assert abs(along - (want * u).sum()) <= (1e-2 + ROUND[dst]) * want.norm()
        plan.close()


def steps_against_definition(plan, scales, dtype, tol, bad=None, sample=None, steps=2):
    """`steps` steps with weights, update and momentum; matrix `bad` holds a NaN and stays as it is."""
    mu, lr, decay = 0.95, 0.02, 0.1
    mom, par = data(plan, 1), 0.02 * torch.randn(plan.length, device="cuda")
    upd = torch.full((plan.length,), 5.0, dtype=DT[dtype], device="cuda")
    outside = plan.outside()
    keep = [t[outside].clone() for t in (mom, par, upd)]
    sample = range(len(plan.shapes)) if sample is None else sample
    m64 = {k: plan.views(mom)[k].double() for k in sample}
    p64 = {k: plan.views(par)[k].double() for k in sample}
    if bad is not None:
        left = [plan.views(t)[bad].clone() for t in (mom, par)]
    with_params = dtype == "f32"
    for t in range(steps):
        grad = data(plan, 10 + t)
        if bad is not None:
            plan.views(grad)[bad][-1, -1] = math.nan
        ecq.ecq_muon_step(plan.h, grad, mom, par if with_params else None, upd, mu=mu, lr=lr, decay=decay)
        assert ecq.ecq_muon_status(plan.h) == (ecq.ECQ_OK if bad is None else ecq.ECQ_ERR_NONFINITE)
        for k in sample:
            if k == bad:
                assert torch.equal(plan.views(mom)[k], left[0]) and torch.equal(plan.views(par)[k], left[1])
                assert torch.all(plan.views(upd)[k] == 0)
                continue
            g = plan.views(grad)[k].double()
            m64[k].mul_(mu).add_(g)
            o = scales[k] * polar(g + mu * m64[k], plan.coefficients)
            assert far(plan.views(mom)[k], m64[k]) <= 4 * 2.0 ** -24 * (t + 1)
            assert far(plan.views(upd)[k], o) <= tol + ROUND[dtype], (k, plan.shapes[k])
            if with_params:
                p64[k].mul_(1 - lr * decay).sub_(lr * o)
                # lr times the update's error, and 3 roundings of the weights a step
                assert (plan.views(par)[k].double() - p64[k]).norm() <= (t + 1) * (lr * tol * o.norm() + 3 * 2.0 ** -24 * p64[k].norm())
    assert all(torch.equal(t[outside], k) for t, k in zip((mom, par, upd), keep))


@pytest.mark.parametrize("tiles", [0] + list(TILES.values()))
@pytest.mark.parametrize("dtype,precision", [("f32", ecq.ECQ_MUON_AUTO), ("f32", ecq.ECQ_MUON_HALF), ("bf16", ecq.ECQ_MUON_AUTO)])
def test_step_of_a_models_layer(tiles, dtype, precision):
    """The matrices of a language model's layer: the passes over the vectors are two launches, and one
    matrix holds a NaN."""
    shapes = [(1024, 4096), (1024, 1024), (4096, 1024), (257, 1030)]
    scales = [0.2 * math.sqrt(max(s)) for s in shapes]
    plan = Plan(shapes, gap=37, tiles=tiles, scales=scales, precision=precision)
    half = dtype == "bf16" or precision == ecq.ECQ_MUON_HALF
    steps_against_definition(plan, scales, dtype, HALF if half else SPLIT, bad=1)
    plan.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_step_of_more_groups_than_are_under_way_at_a_time(dtype):
    """66 M entries: groups of matrices that wait for a turn of the groups before them."""
    shapes = [(1024, 4096), (2048, 2048)] * 6 + [(100, 300)] * 9 + [(4096, 1024)] * 4
    scales = [0.2 * math.sqrt(max(s)) for s in shapes]
    plan = Plan(shapes, gap=3, scales=scales)
    steps_against_definition(plan, scales, dtype, SPLIT if dtype == "f32" else HALF, sample=(0, 1, 5, 11, 15, 20, 21, 24))
    plan.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tiles", list(TILES.values()))
def test_weights_and_a_narrow_update_in_one_call(tiles, dtype):
    """The weights are the ones that a call without the update gives, the update is the fp32 one rounded."""
    plan = Plan([(300, 520), (520, 300), (64, 131)], gap=1, tiles=tiles, scales=[1.0, 0.5, 2.0])
    grad, mom, par = data(plan, 1), data(plan, 2), data(plan, 3)
    got = []
    for out in (torch.float32, DT[dtype]):
        m, p, u = mom.clone(), par.clone(), torch.full((plan.length,), 5.0, dtype=out, device="cuda")
        ecq.ecq_muon_step(plan.h, grad, m, p, u, mu=0.9, lr=0.1, decay=0.1)
        got.append((m, p, u.to(DT[dtype])))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    plan.close()


def test_in_a_graph():
    """Captured once, replayed on other data: the same bits as the calls themselves."""
    shapes = [(1024, 512), (300, 200), (512, 512)]
    plan = Plan(shapes, gap=1, scales=[1.0, 2.0, 3.0])
    grad, mom, par = data(plan, 1), data(plan, 2), data(plan, 3)
    logits = torch.randn(70, 5003, device="cuda").bfloat16()
    y = torch.randint(0, 5003, (70,), device="cuda")
    lp, ent, lse = (torch.empty(70, device="cuda") for _ in range(3))
    d = torch.empty_like(logits)

    def work():
        ecq.ecq_token_logprob(logits, y, lp, ent, lse)
        ecq.ecq_token_logprob_grad(logits, y, lse, ent, lp, ent, d)
        ecq.ecq_muon_step(plan.h, grad, mom, par, mu=0.9, lr=0.1)

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for seed in range(3):
        grad.copy_(data(plan, 20 + seed))
        logits.copy_(torch.randn(70, 5003, device="cuda"))
        start = [t.clone() for t in (mom, par)]
        work()
        want = [t.clone() for t in (mom, par, lp, ent, lse, d)]
        for t, s in zip((mom, par), start):
            t.copy_(s)
        for t in (lp, ent, lse, d):
            t.fill_(7.0)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(want, (mom, par, lp, ent, lse, d)))
    plan.close()


@pytest.mark.parametrize("shapes", [([(1024, 1024)], [(2497, 85), (300, 1000)]), ([(512, 512)] * 20, [(1024, 2048)] * 4)], ids=str)
def test_two_plans_on_two_streams(shapes):
    plans = [Plan(s) for s in shapes]
    srcs = [data(p, k) for k, p in enumerate(plans)]
    want = [check_orth(p, s) for p, s in zip(plans, srcs)]
    outs = [torch.full_like(w, 5.0) for w in want]
    streams = [torch.cuda.Stream() for _ in plans]
    torch.cuda.synchronize()
    for _ in range(30):
        for p, s, o, st in zip(plans, srcs, outs, streams):
            with torch.cuda.stream(st):
                ecq.ecq_muon_orthogonalize(p.h, s, o)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    for p in plans:
        p.close()
