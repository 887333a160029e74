"""Refusals of the C entries on matrices in 8 bits that need no GPU: every one is checked before any CUDA
call; and the format's sizes."""
import ctypes

import pytest
import torch

import paper_1806_08054_b200 as ecq
from paper_1806_08054_b200 import binding

P = 4096          # a non-null, aligned stand-in for a device address; refused calls never touch it
F32, BF16, F16, E4M3, E5M2 = ecq.ECQ_F32, ecq.ECQ_BF16, ecq.ECQ_F16, ecq.ECQ_E4M3, ecq.ECQ_E5M2


def mat(dtype=F32, stride=256, data=P, scales=None):
    return binding._PACK(data, stride, P if scales is None and dtype in (E4M3, E5M2) else scales or 0, dtype)


def test_scale_bytes():
    assert ecq.ecq_act8_scale_bytes(0, 5) == 0 and ecq.ecq_act8_scale_bytes(1, 1) == 512
    assert ecq.ecq_act8_scale_bytes(128, 512) == 512 and ecq.ecq_act8_scale_bytes(129, 513) == 2048
    assert ecq.ecq_act8_scale_bytes((1 << 28) + 1, 1) == 0
    with pytest.raises(ValueError):
        ecq.ecq_act8_scale_bytes(-1, 1)


def store(rows=4, cols=200, x=mat(), q=mat(E4M3), q_t=None):
    return binding.lib().ecq_act8_store(rows, cols, x, q, q_t, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(q=None), dict(x=mat(data=0)), dict(x=mat(5)), dict(x=mat(-1)), dict(x=mat(stride=199)), dict(x=mat(data=P + 2)),
    dict(x=mat(stride=(1 << 36) + 1)), dict(x=mat(BF16, data=P + 1)), dict(q=mat(F32)), dict(q=mat(E4M3, stride=200)),
    dict(q=mat(E4M3, stride=192)), dict(q=mat(E4M3, data=P + 8)), dict(q=mat(E5M2, scales=P + 8)),
    dict(q=binding._PACK(P, 256, 0, E4M3)), dict(q_t=mat(E4M3, stride=8)), dict(q_t=mat(BF16)), dict(cols=0),
    dict(rows=(1 << 28) + 1), dict(cols=(1 << 28) + 1), dict(x=mat(E4M3, stride=192)),
    dict(rows=1 << 28, cols=1 << 28, x=mat(stride=1 << 28), q=mat(E4M3, stride=1 << 28))])
def test_store_refuses(bad):
    assert store(**bad) == binding.ECQ_ERR_ARG


def test_load_refuses():
    L = binding.lib()
    good = dict(q=mat(E4M3), x=mat(BF16))
    for bad in (dict(q=mat(BF16)), dict(x=mat(E4M3)), dict(q=None), dict(x=None), dict(x=mat(BF16, stride=100))):
        a = {**good, **bad}
        assert L.ecq_act8_load(4, 200, a["q"], a["x"], None) == binding.ECQ_ERR_ARG


GATE = ("gate", "up", "out", "out8", "out8_t", "gate8", "up8")


@pytest.mark.parametrize("bad", [
    dict(gate=None), dict(up=None), dict(up=mat(BF16)), dict(out=None), dict(out=mat(BF16)), dict(out=mat(E4M3)), dict(out8=mat(F32)),
    dict(out8_t=mat(E4M3, stride=0)), dict(gate8=mat(F16)), dict(up8=mat(E5M2, stride=100)), dict(gate=mat(E4M3), up=mat(E5M2)),
    dict(gate=mat(E4M3), up=mat(E4M3), out=mat(9))])
def test_gate_refuses(bad):
    a = {**dict.fromkeys(GATE), "gate": mat(), "up": mat(), "out": mat(), **bad}
    assert binding.lib().ecq_act8_gate(4, 200, *[a[n] for n in GATE], None) == binding.ECQ_ERR_ARG


GRAD = ("gate", "up", "d_out", "d_gate", "d_up", "d_gate8", "d_gate8_t", "d_up8", "d_up8_t")


@pytest.mark.parametrize("bad", [
    dict(gate=None), dict(up=None), dict(d_out=None), dict(d_out=mat(E4M3)), dict(d_out=mat(BF16)), dict(d_gate=None), dict(d_gate=mat(F16)),
    dict(d_up=mat(E4M3)), dict(d_gate8=mat(F32)), dict(d_gate8_t=mat(E4M3, stride=2)), dict(d_up8=mat(E4M3, stride=201)),
    dict(d_up8_t=mat(BF16))])
def test_gate_grad_refuses(bad):
    a = {**dict.fromkeys(GRAD), "gate": mat(), "up": mat(), "d_out": mat(), "d_gate": mat(), **bad}
    assert binding.lib().ecq_act8_gate_grad(4, 200, *[a[n] for n in GRAD], None) == binding.ECQ_ERR_ARG


def norm(rows=4, cols=200, x=mat(), residual=None, weight=P, wd=F32, eps=1e-6, total=None, out=mat(), out8=None, sum8=None, rstd=None):
    return binding.lib().ecq_act8_norm(rows, cols, x, residual, weight, wd, eps, total, out, out8, sum8, rstd, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(x=mat(E4M3)), dict(residual=mat(BF16)), dict(residual=mat(stride=100)), dict(weight=P + 2), dict(wd=3), dict(eps=-1.0),
    dict(eps=float("nan")), dict(eps=float("inf")), dict(out=None), dict(out=mat(F16)), dict(total=mat(BF16)), dict(out8=mat(F32)),
    dict(sum8=mat(E4M3, stride=100)), dict(rstd=P + 2), dict(cols=16385, x=mat(stride=20000), out=mat(stride=20000)), dict(cols=0)])
def test_norm_refuses(bad):
    assert norm(**bad) == binding.ECQ_ERR_ARG


def norm_grad(rows=4, cols=200, s=mat(), weight=P, wd=F32, rstd=P, d_out=mat(), d_sum=None, d_x=mat(), d_weight=None, ws=None, size=0):
    return binding.lib().ecq_act8_norm_grad(rows, cols, s, weight, wd, rstd, d_out, d_sum, d_x, d_weight, ws, size, None)


@pytest.mark.parametrize("bad", [
    dict(s=None), dict(s=mat(BF16)), dict(weight=P + 1), dict(wd=-1), dict(rstd=None), dict(rstd=P + 1), dict(d_out=None), dict(d_out=mat(E4M3)),
    dict(d_sum=mat(F16)), dict(d_x=None), dict(d_x=mat(BF16)), dict(d_weight=P), dict(d_weight=P + 2, ws=P, size=1 << 30),
    dict(d_weight=P, ws=P + 8, size=1 << 30), dict(cols=16385, s=mat(stride=20000), d_out=mat(stride=20000), d_x=mat(stride=20000))])
def test_norm_grad_refuses(bad):
    assert norm_grad(**bad) == binding.ECQ_ERR_ARG


def product(m=4, n=8, k=200, a=mat(E4M3), b=mat(E4M3), c=None, d=mat(), status=None):
    return binding.lib().ecq_act8_product(m, n, k, a, b, c, d, status, None)


@pytest.mark.parametrize("bad", [
    dict(a=None), dict(b=None), dict(d=None), dict(a=mat(F32)), dict(b=mat(BF16)), dict(a=mat(E4M3, stride=192)), dict(b=mat(E4M3, data=P + 4)),
    dict(c=mat(E4M3)), dict(c=mat(), d=mat(E4M3)), dict(d=mat(stride=7)), dict(n=0), dict(k=0), dict(status=P + 2), dict(m=(1 << 28) + 1),
    dict(c=mat(stride=4)), dict(d=mat(E5M2, stride=8))])
def test_product_refuses(bad):
    assert product(**bad) == binding.ECQ_ERR_ARG


def test_no_rows_is_nothing_to_do():
    empty = lambda dtype: binding._PACK(0, 0, 0, dtype)
    L = binding.lib()
    assert L.ecq_act8_store(0, 200, empty(F32), empty(E4M3), empty(E5M2), None) == binding.ECQ_OK
    assert L.ecq_act8_load(0, 200, empty(E4M3), empty(F32), None) == binding.ECQ_OK
    assert L.ecq_act8_norm(0, 200, empty(F32), None, None, 0, 0.0, None, empty(F32), None, None, None, None) == binding.ECQ_OK
    assert L.ecq_act8_norm_grad(0, 200, empty(E4M3), None, 0, None, empty(F32), None, empty(F32), None, None, 0, None) == binding.ECQ_OK
    assert L.ecq_act8_product(0, 8, 200, empty(E4M3), mat(E4M3), None, empty(F32), None, None) == binding.ECQ_OK
    assert L.ecq_act8_store(0, 200, empty(7), empty(E4M3), None, None) == binding.ECQ_ERR_ARG


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 200)
    q = (torch.zeros(4, 208, dtype=torch.uint8).view(torch.float8_e4m3fn)[:, :200], torch.zeros(512, dtype=torch.uint8))
    for call in (lambda: ecq.ecq_act8_store(x, q), lambda: ecq.ecq_act8_load(q, x), lambda: ecq.ecq_act8_gate(x, x, x),
                 lambda: ecq.ecq_act8_norm(x, out=x), lambda: ecq.ecq_act8_product(q, q, x)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        ecq.ecq_act8_set_wait_limit(1 << 32)


def test_the_struct_is_the_headers():
    class Matrix(ctypes.Structure):
        _fields_ = [("data", ctypes.c_void_p), ("stride", ctypes.c_uint64), ("scales", ctypes.c_void_p), ("dtype", ctypes.c_int32)]
    packed = binding._PACK(1 << 40, 7, 9, 3)
    assert len(packed) == ctypes.sizeof(Matrix)
    m = Matrix.from_buffer_copy(packed)
    assert (m.data, m.stride, m.scales, m.dtype) == (1 << 40, 7, 9, 3)


def outcome(f, *args):
    try:
        return f(*args)
    except (ValueError, AttributeError, TypeError) as e:
        return type(e), str(e)


def test_marshalling_is_the_same_compiled_and_in_python():
    """On host tensors with their device's number, -1, in place of the current GPU's."""
    from paper_1806_08054_b200.build import build_marshal
    if not build_marshal():
        pytest.skip("no headers of Python or torch")
    from paper_1806_08054_b200 import _marshal
    q8 = lambda r, c, stride, kind=torch.float8_e4m3fn: torch.zeros(r, stride, dtype=torch.uint8).view(kind)[:, :c]
    scales = torch.zeros(512 * 2, dtype=torch.uint8)
    matrices = [None, torch.zeros(4, 200), torch.zeros(4, 200, dtype=torch.bfloat16), torch.zeros(4, 300, dtype=torch.float16)[:, :200],
                torch.zeros(4, 201), torch.zeros(5, 200), torch.zeros(200, 4).T, torch.zeros(1, 200).expand(4, 200), torch.zeros(4, 200).double(),
                (q8(4, 200, 208), scales), [q8(4, 200, 256, torch.float8_e5m2), scales], (q8(4, 200, 208), scales[:511]),
                (q8(4, 200, 208), scales[::2]), (q8(4, 200, 208), scales.float()), (torch.zeros(4, 200), scales),
                (torch.zeros(4, 200, dtype=torch.uint8), scales), (q8(4, 201, 208), scales)]
    for m in matrices:
        for device in (-1, 0):
            args = (m, "some", 4, 200, device)
            assert outcome(_marshal.matrix, *args) == outcome(binding._in_python[0], *args)
    one = torch.zeros(7, 33)[3:4, :17]
    assert _marshal.matrix(one, "one", 1, 17, -1) == binding._in_python[0](one, "one", 1, 17, -1)
    for m in (torch.zeros(4, 200), (q8(4, 200, 208), scales)):
        assert outcome(_marshal.size, m, "some") == outcome(binding._in_python[1], m, "some")
    for t, dtype, n in ((None, torch.float32, 5), (torch.zeros(5), torch.float32, 5), (torch.zeros(5), torch.float32, 6),
                        (torch.zeros(5), torch.int32, 5), (torch.zeros(10)[::2], torch.float32, 5), (torch.zeros(5).half(), torch.float16, 5)):
        for device in (-1, 0):
            assert outcome(_marshal.vector, t, dtype, n, "some", device) == outcome(binding._in_python[2], t, dtype, n, "some", device)
    for f in (_marshal.matrix, _marshal.size, _marshal.vector):
        with pytest.raises(TypeError):
            f(1)
    with pytest.raises(ValueError):
        _marshal.matrix(7, "some", 4, 200, -1)
