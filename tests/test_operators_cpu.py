"""Refusals of the operators' C entries that need no GPU: every one is checked before any CUDA call."""
import ctypes

import pytest

import paper_1806_08054_b200 as ecq
from paper_1806_08054_b200 import binding

P = 4096          # a non-null, aligned stand-in for a device address; refused calls never touch it


def logprob(logits=P, dtype=ecq.ECQ_F32, rows=2, vocab=8, stride=8, targets=P, tau=1.0, top=0, lp=P, ent=None,
            lse=None, tl=None, ti=None):
    return binding.lib().ecq_token_logprob(logits, dtype, rows, vocab, stride, targets, tau, top, lp, ent, lse, tl, ti, None)


def grad(logits=P, dtype=ecq.ECQ_BF16, rows=2, vocab=8, stride=8, targets=P, tau=1.0, lse=P, ent=None, glp=P, gent=None,
         d=P, d_stride=8):
    return binding.lib().ecq_token_logprob_grad(logits, dtype, rows, vocab, stride, targets, tau, lse, ent, glp, gent, d,
                                                d_stride, None)


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(dtype=3), dict(dtype=-1), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(stride=7),
    dict(tau=0.0), dict(tau=-1.0), dict(tau=float("inf")), dict(tau=float("nan")), dict(top=33, tl=P, ti=P),
    dict(top=9, tl=P, ti=P), dict(top=2, tl=P), dict(top=2, ti=P), dict(tl=P, ti=P), dict(targets=None), dict(lp=None),
    dict(lp=None, targets=None), dict(logits=P + 2), dict(targets=P + 4), dict(lp=P + 2), dict(ent=P + 1), dict(lse=P + 3),
    dict(rows=(1 << 28) + 1), dict(dtype=ecq.ECQ_F16, logits=P + 1)])
def test_logprob_refuses(bad):
    assert logprob(**bad) == ecq.ECQ_ERR_ARG


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(d=None), dict(dtype=7), dict(vocab=0), dict(stride=7), dict(d_stride=7), dict(tau=0.0),
    dict(lse=None), dict(targets=None), dict(glp=None), dict(glp=None, targets=None), dict(gent=P), dict(d=P + 1),
    dict(lse=P + 2), dict(d=P, d_stride=9)])
def test_logprob_grad_refuses(bad):
    assert grad(**bad) == ecq.ECQ_ERR_ARG


@pytest.mark.parametrize("tau", [2.4e38, 3.4e38])
def test_a_temperature_beyond_the_range_of_its_powers_of_two_is_refused(tau):
    assert logprob(tau=tau) == ecq.ECQ_ERR_ARG and grad(tau=tau) == ecq.ECQ_ERR_ARG


def test_no_rows_is_nothing_to_do():
    assert logprob(rows=0) == ecq.ECQ_OK and grad(rows=0) == ecq.ECQ_OK
    assert logprob(rows=0, dtype=9) == ecq.ECQ_ERR_ARG


def create(offsets=(0,), rows=(8,), cols=(6,), strides=None, scales=None, steps=5, coefficients=None, precision=0, out=True,
           count=None):
    n = len(offsets)
    u64, u32, f32 = ctypes.c_uint64 * n, ctypes.c_uint32 * n, ctypes.c_float * n
    h = ctypes.c_void_p()
    rc = binding.lib().ecq_muon_create(
        ctypes.byref(h) if out else None, n if count is None else count, u64(*offsets), u32(*rows), u32(*cols),
        None if strides is None else u64(*strides), None if scales is None else f32(*scales), steps,
        None if coefficients is None else (ctypes.c_float * len(coefficients))(*coefficients), precision)
    assert h.value is None
    return rc


@pytest.mark.parametrize("bad", [
    dict(out=False), dict(count=0), dict(count=65537), dict(rows=(0,)), dict(cols=(0,)), dict(rows=((1 << 22) + 1,)),
    dict(rows=(32769,), cols=(32769,)), dict(strides=(5,)), dict(offsets=((1 << 48) + 1,)), dict(scales=(float("nan"),)),
    dict(steps=0), dict(steps=65), dict(precision=-1), dict(precision=3), dict(coefficients=[float("inf")] * 15),
    dict(coefficients=[30.0, 0.0, 0.0] * 5), dict(coefficients=[1.0, 200.0, -200.0] * 5)])
def test_muon_create_refuses(bad):
    assert create(**bad) == ecq.ECQ_ERR_ARG


def test_muon_calls_refuse_no_plan():
    L = binding.lib()
    assert L.ecq_muon_orthogonalize(None, P, 0, P, 0, None) == ecq.ECQ_ERR_ARG
    assert L.ecq_muon_step(None, P, P, 0.9, 1, 0.1, 0.0, P, None, 0, None) == ecq.ECQ_ERR_ARG
    assert L.ecq_muon_bind(None, P, 0, None) == ecq.ECQ_ERR_ARG
    assert L.ecq_muon_set_tiles(None, 0) == ecq.ECQ_ERR_ARG
    assert L.ecq_muon_set_wait_limit(None, 1) == ecq.ECQ_ERR_ARG
    assert L.ecq_muon_status(None, None) == ecq.ECQ_ERR_ARG
    assert L.ecq_muon_workspace_bytes(None) == 0
    L.ecq_muon_destroy(None)


def test_binding_refuses_before_the_library():
    import torch
    for bad in (dict(rows=[8, 8]), dict(strides=[6, 6]), dict(scales=[]), dict(coefficients=[(1.0, 1.0, 1.0)] * 4),
                dict(offsets=[-1])):
        args = dict(offsets=[0], rows=[8], cols=[6])
        args.update(bad)
        with pytest.raises(ValueError):
            ecq.ecq_muon_create(**args)
    with pytest.raises(ValueError):
        ecq.ecq_token_logprob(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64), torch.zeros(2))


def test_binding_refuses_sizes_whose_low_bits_would_pass():
    """ctypes passes a number modulo 2^32 or 2^64: 2^32 + 8 rows would be taken for 8."""
    import torch
    from unittest import mock
    for bad in (dict(rows=[(1 << 32) + 8]), dict(cols=[(1 << 32) + 6]), dict(offsets=[1 << 64]), dict(strides=[(1 << 64) + 6]),
                dict(steps=(1 << 32) + 5)):
        args = dict(offsets=[0], rows=[8], cols=[6])
        args.update(bad)
        with mock.patch.object(binding.lib(), "ecq_muon_create", side_effect=AssertionError("reached the library")):
            with pytest.raises(ValueError):
                ecq.ecq_muon_create(**args)
    wide = torch.zeros(1, dtype=torch.bfloat16).expand(1, (1 << 32) + 8)

    class OnGpu:                                            # a CUDA tensor of that shape, as the binding sees it
        is_cuda, dtype, shape = True, wide.dtype, wide.shape
        stride = staticmethod(lambda: ((1 << 32) + 8, 1))
        data_ptr = staticmethod(lambda: P)

    with pytest.raises(ValueError):
        binding._rows(OnGpu, "logits")
