"""The operators on matrices in 8 bits as a program uses them: a gated layer's forward and backward pass run
together, captured and replayed, on two streams, beside the codec, and beyond 2^32 bytes."""
import math
import os
import subprocess
import sys

import pytest
import torch

import paper_1806_08054_b200 as ecq
from act8_util import E5M2, check_plain, pair, random, scale_places, stored, strided, values

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


class Layer:
    """y = s + W_down (silu(W_gate n) * (W_up n)), n = norm(s), s = x + residual: all buffers of one step."""

    def __init__(self, tokens, width, hidden, seed, dtype=BF16):
        T, d, f = tokens, width, hidden
        r = lambda a, b, k, size=1.0: random(a, b, seed + k, size)
        self.x, self.residual = r(T, d, 0, 0.3).to(dtype), r(T, d, 1, 0.3).to(dtype)
        self.norm_w = (1 + r(1, d, 2, 0.05)[0]).float()
        self.weights = [r(f, d, 3, 0.5 / math.sqrt(d)).float(), r(f, d, 4, 0.5 / math.sqrt(d)).float(), r(d, f, 5, 0.5 / math.sqrt(f)).float()]
        self.d_y = r(T, d, 6, 1e-3).to(dtype)
        self.w8 = [pair(*w.shape) for w in self.weights]
        self.w8_t = [pair(*reversed(w.shape)) for w in self.weights]
        self.sum, self.sum8, self.n8, self.n8_t = torch.empty_like(self.x), pair(T, d), pair(T, d), pair(d, T)
        self.rstd = torch.empty(T, device="cuda")
        self.gate, self.up = (torch.empty(T, f, dtype=dtype, device="cuda") for _ in range(2))
        self.h8, self.gate8, self.up8, self.h8_t = pair(T, f), pair(T, f), pair(T, f), pair(f, T)
        self.y = torch.empty_like(self.x)
        self.d_y8, self.d_y8_t = pair(T, d, E5M2), pair(d, T)
        self.d_h = torch.empty(T, f, dtype=dtype, device="cuda")
        self.d_gate8, self.d_up8, self.d_gate8_t, self.d_up8_t = pair(T, f), pair(T, f, E5M2), pair(f, T), pair(f, T)
        self.d_n, self.d_x = torch.empty(T, d, device="cuda"), torch.empty(T, d, device="cuda")
        self.grads = [torch.zeros_like(w) for w in self.weights]
        self.d_norm_w = torch.empty(d, device="cuda")
        self.sum32 = torch.empty(T, d, device="cuda")
        self.work = torch.empty(ecq.ecq_act8_norm_grad_workspace_bytes(T, d), dtype=torch.uint8, device="cuda")

    def step(self):
        for w, q, t in zip(self.weights, self.w8, self.w8_t):
            ecq.ecq_act8_store(w, q, t)
        ecq.ecq_act8_norm(self.x, self.residual, self.norm_w, eps=1e-5, sum=self.sum, sum8=self.sum8, out8=self.n8, rstd=self.rstd)
        ecq.ecq_act8_product(self.n8, self.w8[0], self.gate)
        ecq.ecq_act8_product(self.n8, self.w8[1], self.up)
        ecq.ecq_act8_gate(self.gate, self.up, out8=self.h8, gate8=self.gate8, up8=self.up8)
        ecq.ecq_act8_product(self.h8, self.w8[2], self.y, add=self.sum)
        # backward
        ecq.ecq_act8_store(self.d_y, self.d_y8, self.d_y8_t)
        ecq.ecq_act8_product(self.d_y8, self.w8_t[2], self.d_h)
        ecq.ecq_act8_gate_grad(self.gate8, self.up8, self.d_h, d_gate8=self.d_gate8, d_gate8_t=self.d_gate8_t, d_up8=self.d_up8,
                               d_up8_t=self.d_up8_t)
        ecq.ecq_act8_store(self.h8, None, self.h8_t)
        ecq.ecq_act8_store(self.n8, None, self.n8_t)
        for g, left, right in zip(self.grads, (self.d_gate8_t, self.d_up8_t, self.d_y8_t), (self.n8_t, self.n8_t, self.h8_t)):
            ecq.ecq_act8_product(left, right, g, add=g)
        ecq.ecq_act8_product(self.d_gate8, self.w8_t[0], self.d_n)
        ecq.ecq_act8_product(self.d_up8, self.w8_t[1], self.d_n, add=self.d_n)
        ecq.ecq_act8_load(self.sum8, self.sum32)
        ecq.ecq_act8_norm_grad(self.sum8, self.norm_w, self.rstd, self.d_n, self.d_x, self.d_norm_w, self.work)

    def results(self):
        return [self.y, self.sum, self.d_x, self.d_norm_w, *self.grads]


def product_error(a, b):
    return (values(a).abs() @ values(b).abs().T) * (a[0].shape[1] / 32 + 8) * 2.0 ** -22


SIZES = [(1, 64, 100), (37, 200, 333), (300, 512, 1024), (257, 130, 700)]


@pytest.mark.parametrize("tokens,width,hidden", SIZES)
def test_a_layers_step_is_its_parts_in_64_bits(tokens, width, hidden):
    """Each product and sum from what was stored before it: shapes, transposes and additions in place."""
    L = Layer(tokens, width, hidden, 11)
    L.step()
    V = values
    s = L.x.double() + L.residual.double()
    check_plain(L.sum, s, s.abs() * 2.0 ** -24, "sum")
    for out, w in ((L.gate, L.w8[0]), (L.up, L.w8[1])):
        check_plain(out, V(L.n8) @ V(w).T, product_error(L.n8, w), "gate, up")
    want = V(L.h8) @ V(L.w8[2]).T + L.sum.double()
    check_plain(L.y, want, product_error(L.h8, L.w8[2]) + want.abs() * 2.0 ** -24, "y")
    check_plain(L.d_h, V(L.d_y8) @ V(L.w8_t[2]).T, product_error(L.d_y8, L.w8_t[2]), "d_h")
    for g, left, right in zip(L.grads, (L.d_gate8_t, L.d_up8_t, L.d_y8_t), (L.n8_t, L.n8_t, L.h8_t)):
        check_plain(g, V(left) @ V(right).T, product_error(left, right), "weights")
    want = V(L.d_gate8) @ V(L.w8_t[0]).T + V(L.d_up8) @ V(L.w8_t[1]).T
    err = product_error(L.d_gate8, L.w8_t[0]) + product_error(L.d_up8, L.w8_t[1])
    check_plain(L.d_n, want, err + want.abs() * 2.0 ** -22, "d_n")
    assert torch.equal(L.sum32.double(), V(L.sum8))
    f = L.rstd.double()[:, None]
    n, g = V(L.sum8) * f, L.d_n.double() * L.norm_w.double()
    want = f * (g - n * (g * n).mean(1, keepdim=True))
    check_plain(L.d_x, want, f * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True)) * 2.0 ** -18, "d_x")


def test_a_layers_gradient_is_near_the_unrounded_layers():
    """Against autograd in 64 bits of the same layer without 8 bits.  An operand's rounding is 2^-4 of an
    entry at most, 2^-4 / sqrt(3) of its norm where errors spread evenly (e5m2: twice that); a product has two such
    operands, and up to four products follow each other: sqrt(8) / sqrt(3) / 16 = 0.10, 0.15 with e5m2 among them."""
    L = Layer(512, 384, 640, 5, dtype=F32)
    L.step()
    ps = [t.double().requires_grad_() for t in (L.x, L.norm_w, *L.weights)]
    x, nw, wg, wu, wd = ps
    s = x + L.residual.double()
    n = s / torch.sqrt(s.square().mean(1, keepdim=True) + 1e-5) * nw
    g = n @ wg.T
    ((g * torch.sigmoid(g) * (n @ wu.T)) @ wd.T * L.d_y.double()).sum().backward()
    for got, p in zip((L.d_x, L.d_norm_w, *L.grads), ps):
        assert (got.double() - p.grad).norm() <= 0.15 * p.grad.norm()


@pytest.mark.parametrize("tokens,width,hidden", [(37, 200, 333), (2100, 512, 1024)])
def test_captured_and_replayed(tokens, width, hidden):
    eager, L = Layer(tokens, width, hidden, 3), Layer(tokens, width, hidden, 3)
    eager.step()
    want = [t.clone() for t in eager.results()]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        L.step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for g in L.grads:
            g.zero_()
        L.step()
    for _ in range(3):
        for t in (L.y, L.sum, L.d_x, L.d_norm_w):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(L.results(), want):
            assert torch.equal(a, b)
    L.x.copy_(random(tokens, width, 99))                      # new inputs in the captured buffers
    eager.x.copy_(L.x)
    for g in eager.grads:
        g.zero_()
    graph.replay()
    eager.step()
    for a, b in zip(L.results(), eager.results()):
        assert torch.equal(a, b)


FIRST = """
import torch
import paper_1806_08054_b200 as ecq
from act8_util import pair, random, stored
x = random(300, 520, 1).bfloat16()
q, t, out = pair(300, 520), pair(520, 300), torch.zeros_like(x)
a, b, rstd = stored(random(2000, 700, 2)), stored(random(900, 700, 3)), torch.ones(300, device="cuda")
d, one, dw = torch.zeros(2000, 900, device="cuda"), torch.zeros(200, 900, device="cuda"), torch.zeros(520, device="cuda")
few = stored(random(200, 700, 4))
work = torch.empty(ecq.ecq_act8_norm_grad_workspace_bytes(300, 520), dtype=torch.uint8, device="cuda")
torch.cuda.synchronize()

def calls():
    ecq.ecq_act8_store(x, q, t)
    ecq.ecq_act8_load(q, out)
    ecq.ecq_act8_gate(x, x, out)
    ecq.ecq_act8_norm(x, out, sum=out)
    ecq.ecq_act8_norm_grad(x, None, rstd, x, out, dw, work)
    ecq.ecq_act8_product(a, b, d)
    ecq.ecq_act8_product(few, b, one)

graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    calls()
graph.replay()
torch.cuda.synchronize()
got = [y.clone() for y in (out, d, one, dw)]
calls()
for y, z in zip((out, d, one, dw), got):
    assert torch.equal(y, z) and bool(z.any())
"""


def test_the_first_calls_of_a_process_may_be_captured():
    """Nothing that a first call sets up (kernels' limits, what the GPU holds at once) is refused while a stream is captured."""
    here = os.path.dirname(os.path.abspath(__file__))
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([here, os.path.dirname(here)]))
    run = subprocess.run([sys.executable, "-c", FIRST], env=env, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]


def test_two_streams_at_once():
    layers = [Layer(700, 512, 1536, k) for k in (1, 2)]
    want = []
    for L in layers:
        L.step()
        want.append([t.clone() for t in L.results()])
    torch.cuda.synchronize()
    for L in layers:
        for g in L.grads:
            g.zero_()
    streams = [torch.cuda.Stream() for _ in layers]
    torch.cuda.synchronize()
    for _ in range(5):
        for L, st in zip(layers, streams):
            with torch.cuda.stream(st):
                for g in L.grads:
                    g.zero_()
                L.step()
    torch.cuda.synchronize()
    for L, w in zip(layers, want):
        for a, b in zip(L.results(), w):
            assert torch.equal(a, b)


def test_the_gradient_goes_on_to_the_codec():
    """Weights' gradients added into the flat vector that is encoded, at offsets that are no multiple of 16 bytes."""
    T, a, b = 300, 257, 130
    flat = torch.zeros(4096 * 9, device="cuda")
    left, right = stored(random(a, T, 1)), stored(random(b, T, 2))
    for at in (0, 1, 37, 1024):
        flat.zero_()
        g = flat[at:at + a * b].view(a, b)
        ecq.ecq_act8_product(left, right, g, add=g)
        ecq.ecq_act8_product(left, right, g, add=g)
        want = 2 * (values(left) @ values(right).T)
        err = 2 * (values(left).abs() @ values(right).abs().T) * (T / 32 + 8) * 2.0 ** -22
        check_plain(g, want, err + want.abs() * 2.0 ** -24)
        assert bool((flat[:at] == 0).all() and (flat[at + a * b:] == 0).all())
    ctx = ecq.ecq_create(flat.numel(), 512, 4, 1.0, 0.9, 7)
    err = torch.zeros_like(flat)
    codes = torch.zeros(ecq.ecq_codes_words(ctx), dtype=torch.int32, device="cuda")
    scales = torch.zeros(ecq.ecq_num_buckets(ctx), device="cuda")
    ecq.ecq_encode(ctx, 0, 0, flat, err, codes, scales)
    assert ecq.ecq_status(ctx) == ecq.ECQ_OK
    ecq.ecq_destroy(ctx)


def test_beyond_4_gb():
    """Rows behind 2^32 bytes of a plain matrix and of a product's result."""
    rows, cols = 300_000, 8192
    x = torch.zeros(rows, cols, dtype=BF16, device="cuda")
    tail = random(300, cols, 1).to(BF16)
    x[-300:] = tail
    q = pair(rows, cols)
    ecq.ecq_act8_store(x, q)
    want = stored(tail.double())
    last = (q[0][-300:], None)
    assert torch.equal(last[0].float(), want[0].float())
    places = scale_places(rows, cols)[-300:]
    assert torch.equal(q[1][places], want[1][scale_places(300, cols)])
    x.fill_(7.0)
    ecq.ecq_act8_load(q, x)
    assert torch.equal(x[-300:], values(want).to(BF16)) and bool((x[:1000] == 0).all())
    y = torch.empty_like(x)
    ecq.ecq_act8_norm(x, out=y)
    f = 1 / torch.sqrt(x[-300:].double().square().mean(1, keepdim=True) + 1e-6)
    check_plain(y[-300:], x[-300:].double() * f, (x[-300:].double() * f).abs() * 2.0 ** -18)
    a, b = stored(random(rows, 40, 3)), stored(random(cols, 40, 4))
    y.fill_(7.0)
    ecq.ecq_act8_product(a, b, y)
    av = a[0][-300:].double() * torch.exp2(a[1][scale_places(rows, 40)[-300:]].double() - 127)
    check_plain(y[-300:], av @ values(b).T, av.abs() @ values(b).abs().T * 12 * 2.0 ** -22)
