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


def test_no_rows_is_nothing_to_do():
    assert logprob(rows=0) == ecq.ECQ_OK and grad(rows=0) == ecq.ECQ_OK
    assert logprob(rows=0, dtype=9) == ecq.ECQ_ERR_ARG
