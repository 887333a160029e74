"""Results in 8 bits alone of many tiles, which come one ahead where there is room for one: bit for bit what calls on
few rows give, which test_gpu_act8.py holds to 64 bits; with tiles that come in time and without."""
import pytest
import torch

import paper_1806_08054_b200 as ecq
from act8_util import E4M3, E5M2, bytes_of, pair, random, scale_bytes, strided
from test_gpu_act8 import behind_is_left, gate_parts

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.mark.parametrize("polls", [ecq.binding.ECQ_WAIT_LIMIT_DEFAULT, 0, 1])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("kept", [False, True])
def test_many_tiles_to_8_bits_are_as_few(dtype, kept, polls):
    rows, cols = 5000, 4008
    x, u, d = (strided(rows, cols, dtype).copy_(random(rows, cols, 61 + k)) for k in range(3))
    g8, u8 = pair(rows, cols, E5M2), pair(rows, cols, E5M2)
    ecq.ecq_act8_store(x, g8)
    ecq.ecq_act8_store(u, u8)
    a, b = (g8, u8) if kept else (x, u)

    def calls(a, b, d, rows):
        q = [pair(rows, cols, k) for k in (E4M3, E5M2, E4M3, E5M2, E4M3, E4M3, E4M3, E5M2)]
        t = [pair(cols, rows, k) for k in (E4M3, E5M2, E4M3, E5M2)]
        ecq.ecq_act8_gate(a, b, None, q[0], None, q[1], q[2])
        ecq.ecq_act8_gate(a, b, None, None, t[0], q[3], None)
        ecq.ecq_act8_gate_grad(a, b, d, None, None, q[4], t[1], q[5], t[2])
        ecq.ecq_act8_gate_grad(a, b, d, None, None, q[6], None, q[7], None)
        ecq.ecq_act8_gate_grad(a, b, d, None, None, None, t[3], None, None)
        return q, t

    ecq.ecq_act8_set_wait_limit(polls)
    try:
        q, t = calls(a, b, d, rows)
        torch.cuda.synchronize()
    finally:
        ecq.ecq_act8_set_wait_limit()
    for p in q + t:
        behind_is_left(p)
    for lo in range(0, rows, 512):
        hi = min(rows, lo + 512)
        few = calls(gate_parts(a, lo, hi, kept), gate_parts(b, lo, hi, kept), d[lo:hi], hi - lo)
        for one, all_of in zip(few[0], q):
            assert torch.equal(bytes_of(one)[:, :cols], bytes_of(all_of)[lo:hi, :cols])
            assert torch.equal(scale_bytes(one), scale_bytes(all_of)[lo:hi])
        for one, all_of in zip(few[1], t):
            assert torch.equal(bytes_of(one)[:, :hi - lo], bytes_of(all_of)[:, lo:hi])
            assert torch.equal(scale_bytes(one), scale_bytes(all_of)[:, lo // 128:(hi + 127) // 128])
