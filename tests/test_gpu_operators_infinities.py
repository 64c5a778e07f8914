"""Infinite states, inputs and gradients of the gated recurrence over long sequences: what the formula gives, step after step."""
import math

import numpy as np
import pytest
import torch

from paper_2010_16248_amd import binding as B
from tests import operators_plain as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF = torch.float32, torch.bfloat16


def _check(gate, x, h0, dout, dlast):
    out, last = torch.empty_like(x), torch.empty_like(h0)
    B.recurrence_forward(gate, x, out, h0=h0, h_last=last)
    ref, ref_last, off, last_off = P.recurrence(gate, x, h0)
    P.assert_within(out, ref, off, "out")
    P.assert_within(last, ref_last, last_off, "last")
    dgate, dinput, dh0 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(h0)
    B.recurrence_backward(gate, x, out, dout, dgate, dinput, h0=h0, grad_last=dlast, grad_h0=dh0)
    ref, off = P.recurrence_gradients(gate, x, out, h0, dout, dlast)
    for got, r, o, what in zip((dgate, dinput, dh0), ref, off, ("dgate", "dinput", "dh0")):
        P.assert_within(got, r, o, what)
    return out, last, dh0


# steps, gate: the gates' product over 128 steps (a workgroup), over 1024 (a group of them) or over 16 (a wave) is below what 64 bits hold
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("steps,at", [(3000, -1.0), (3000, -10.0), (200, -10.0), (3000, -60.0), (12, -60.0)])
def test_what_is_infinite_stays_infinite_through_open_gates(steps, at, dtype):
    print(f"case infinite {steps} {at} {dtype}", flush=True)
    gen = torch.Generator().manual_seed(steps)
    r = lambda *s: torch.randn(*s, generator=gen)
    gate, x, dout = ((at + 0.5 * r(2, steps, 70)).to(dtype).to(DEV), r(2, steps, 70).to(dtype).to(DEV), r(2, steps, 70).to(dtype).to(DEV))
    h0, dlast = r(2, 70).to(DEV), r(2, 70).to(DEV)
    h0[0, 3], h0[1, 69], x[0, steps // 3, 10], x[1, 1, 64] = math.inf, -math.inf, math.inf, -math.inf
    dlast[0, 5], dlast[1, 68], dout[0, steps // 2, 12], dout[1, steps - 2, 66] = math.inf, -math.inf, math.inf, -math.inf
    out, last, dh0 = _check(gate, x, h0, dout, dlast)
    assert out[0, :, 3].eq(math.inf).all() and last[1, 69] == -math.inf and last[0, 10] == math.inf and last[1, 64] == -math.inf
    assert dh0[0, 5] == math.inf and dh0[1, 68] == -math.inf and dh0[0, 12] == math.inf and dh0[1, 66] == -math.inf


@pytest.mark.parametrize("steps", [12, 200, 3000])
def test_a_shut_gate_makes_nan_of_infinity(steps):
    gen = torch.Generator().manual_seed(steps)
    r = lambda *s: torch.randn(*s, generator=gen)
    gate, x, dout = (r(1, steps, 65).to(DEV) - 3 for _ in range(3))
    h0, dlast = r(1, 65).to(DEV), r(1, 65).to(DEV)
    h0[0, 64], dlast[0, 0] = math.inf, math.inf
    gate[:, steps // 2] = -math.inf
    out, last, dh0 = _check(gate, x, h0, dout, dlast)
    assert out[0, :steps // 2, 64].eq(math.inf).all() and out[0, steps // 2:, 64].isnan().all() and dh0[0, 0].isnan()


@pytest.mark.parametrize("steps", [9, 40, 300])
def test_gates_below_the_normal_numbers_count(steps):
    """sigmoid(-f) for f from 87.4 to 103.9 lies between 1e-38 and the smallest fp32 number: it shows beside large inputs, states and
    gradients.  One step has such a gate for each channel, all others keep what is there."""
    print(f"case subnormal gates {steps}", flush=True)
    f = torch.linspace(80.0, 103.9, 70, device=DEV)
    for sign in (1.0, -1.0):
        gate = torch.full((1, steps, 70), math.inf, device=DEV)
        gate[:, 5] = sign * f
        x, dout = torch.zeros(1, steps, 70, device=DEV), torch.zeros(1, steps, 70, device=DEV)
        h0, dlast = torch.zeros(1, 70, device=DEV), torch.full((1, 70), 1e38, device=DEV)
        (x[:, 5] if sign > 0 else h0).fill_(1e38)
        out, last = torch.empty_like(x), torch.empty_like(h0)
        B.recurrence_forward(gate, x, out, h0=h0, h_last=last)
        # the gate is rounded to a multiple of 2^-149, which acts on 1e38
        coarse = 2.0 ** -149 * 1e38
        ref, ref_last, off, last_off = P.recurrence(gate, x, h0)
        P.assert_within(out, ref, off + coarse * (np.arange(steps) >= 5)[None, :, None], "out")
        P.assert_within(last, ref_last, last_off + coarse, "last")
        assert last.min() > 0
        dgate, dinput, dh0 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(h0)
        B.recurrence_backward(gate, x, out, dout, dgate, dinput, h0=h0, grad_last=dlast, grad_h0=dh0)
        ref, off = P.recurrence_gradients(gate, x, out, h0, dout, dlast)
        P.assert_within(dinput, ref[1], off[1] + coarse, "dinput")
        P.assert_within(dh0, ref[2], off[2] + coarse, "dh0")
        assert (dinput[:, 5] if sign > 0 else dh0).min() > 0
    h0 = torch.full((1, 70), math.inf, device=DEV)
    gate[:, 5] = -f
    B.recurrence_forward(gate, torch.zeros_like(x), out, h0=h0)
    assert out.eq(math.inf).all()
