"""The gated linear recurrence against the formula, step after step in 64 bits, and its gradients against differences."""
import math

import numpy as np
import pytest
import torch

from paper_2010_16248_amd import binding as B
from tests import operators_plain as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF = torch.float32, torch.bfloat16

# batch, steps, channels
SIZES = [(1, 1, 1), (64, 1, 672), (3, 2, 5), (2, 7, 64), (1, 8, 65), (5, 9, 127), (20, 35, 672), (2, 255, 33), (2, 256, 130), (1, 257, 64),
         (3, 511, 3), (1, 513, 200), (1, 1025, 64), (2, 3000, 70), (1, 16385, 66), (130, 40, 300)]


def _inputs(batch, steps, channels, dtype, seed=0):
    gen = torch.Generator().manual_seed(batch * 7 + steps * 3 + channels + seed)
    shape = (batch, steps, channels)
    gate = torch.randn(*shape, generator=gen) * 2 + torch.empty(channels).uniform_(-2, 7, generator=gen)
    gate[torch.rand(*shape[:2], generator=gen) < 0.01] = -math.inf
    gate[torch.rand(*shape, generator=gen) < 0.01] = math.inf
    x = torch.randn(*shape, generator=gen)
    h0, dlast = torch.randn(batch, channels, generator=gen), torch.randn(batch, channels, generator=gen)
    dout = torch.randn(*shape, generator=gen)
    return [t.to(DEV) for t in (gate.to(dtype), x.to(dtype), h0, dout.to(dtype), dlast)]


def _lengths(batch, steps, kind):
    if kind is None:
        return None
    gen = torch.Generator().manual_seed(batch + steps)
    n = torch.randint(0, steps + 1, (batch,), generator=gen, dtype=torch.int32)
    n[0] = 0 if kind == "empty" else steps
    if batch > 1:
        n[1] = steps + 5
    if batch > 2:
        n[2] = -1
    return n.to(DEV)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("kind", [None, "empty", "whole"])
@pytest.mark.parametrize("batch,steps,channels", SIZES)
def test_forward_and_backward(batch, steps, channels, kind, dtype):
    print(f"case recurrence {batch} {steps} {channels} {kind} {dtype}", flush=True)
    gate, x, h0, dout, dlast = _inputs(batch, steps, channels, dtype)
    lengths = _lengths(batch, steps, kind)
    if kind is not None:                                   # what lies behind a sequence's end plays no role
        for b in range(batch):
            n = min(max(int(lengths[b]), 0), steps)
            gate[b, n:], x[b, n:], dout[b, n:] = math.nan, math.inf, math.nan
    out, last = torch.full_like(gate, 9.0), torch.empty_like(h0)
    B.recurrence_forward(gate, x, out, h0=h0, h_last=last, lengths=lengths)
    ref, ref_last, off, last_off = P.recurrence(gate, x, h0, lengths)
    P.assert_within(out, ref, off, "out")
    P.assert_within(last, ref_last, last_off, "last")
    dgate, dinput, dh0 = torch.full_like(gate, 9.0), torch.full_like(gate, 9.0), torch.empty_like(h0)
    B.recurrence_backward(gate, x, out, dout, dgate, dinput, h0=h0, grad_last=dlast, grad_h0=dh0, lengths=lengths)
    ref, off = P.recurrence_gradients(gate, x, out, h0, dout, dlast, lengths)
    P.assert_within(dgate, ref[0], off[0], "dgate")
    P.assert_within(dinput, ref[1], off[1], "dinput")
    P.assert_within(dh0, ref[2], off[2], "dh0")
    again = [torch.empty_like(t) for t in (out, last, dgate, dinput, dh0)]
    B.recurrence_forward(gate, x, again[0], h0=h0, h_last=again[1], lengths=lengths)
    B.recurrence_backward(gate, x, out, dout, again[2], again[3], h0=h0, grad_last=dlast, grad_h0=again[4], lengths=lengths)
    for a, b in zip(again, (out, last, dgate, dinput, dh0)):
        assert torch.equal(a, b), "the same call gave other bits"


@pytest.mark.parametrize("batch,steps,channels", [(2, 5, 64), (3, 700, 33)])
def test_without_the_optional_tensors(batch, steps, channels):
    gate, x, _, dout, _ = _inputs(batch, steps, channels, F32)
    out = torch.empty_like(gate)
    B.recurrence_forward(gate, x, out)
    ref, _, off, _ = P.recurrence(gate, x, None)
    P.assert_within(out, ref, off, "out")
    dgate, dinput = torch.empty_like(gate), torch.empty_like(gate)
    B.recurrence_backward(gate, x, out, dout, dgate, dinput)
    ref, off = P.recurrence_gradients(gate, x, out, None, dout, None)
    P.assert_within(dgate, ref[0], off[0], "dgate")
    P.assert_within(dinput, ref[1], off[1], "dinput")


@pytest.mark.parametrize("steps", [1, 6, 600])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_slices_of_a_projection_and_time_first_tensors(steps, dtype):
    batch, channels = 3, 77
    gate, x, h0, dout, dlast = _inputs(batch, steps, channels, dtype)
    both = torch.full((batch, steps, 2 * channels + 3), 4.0, dtype=dtype, device=DEV)
    g, v = both[:, :, 1:1 + channels], both[:, :, 2 + channels:2 + 2 * channels]
    g.copy_(gate), v.copy_(x)
    out = torch.empty(steps, batch, channels, dtype=dtype, device=DEV).transpose(0, 1)
    plain, last, last2 = torch.empty_like(gate), torch.empty_like(h0), torch.empty_like(h0)
    B.recurrence_forward(gate, x, plain, h0=h0, h_last=last)
    B.recurrence_forward(g, v, out, h0=h0, h_last=last2)
    assert torch.equal(out, plain) and torch.equal(last, last2)
    d1 = [torch.empty_like(gate), torch.empty_like(gate), torch.empty_like(h0)]
    B.recurrence_backward(gate, x, plain, dout, d1[0], d1[1], h0=h0, grad_last=dlast, grad_h0=d1[2])
    grads = torch.full_like(both, 4.0)
    dg, dv, dh = grads[:, :, 1:1 + channels], grads[:, :, 2 + channels:2 + 2 * channels], torch.empty_like(h0)
    B.recurrence_backward(g, v, out, dout, dg, dv, h0=h0, grad_last=dlast, grad_h0=dh)
    assert torch.equal(dg, d1[0]) and torch.equal(dv, d1[1]) and torch.equal(dh, d1[2])
    for edge in (0, 1 + channels, 2 + 2 * channels):
        assert (grads[:, :, edge] == 4).all() and (both[:, :, edge] == 4).all()


def test_a_gate_for_all_channels_of_a_step_by_stride_zero_batches():
    gate, x, h0, _, _ = _inputs(1, 300, 50, F32)
    shared = gate.expand(4, 300, 50)
    inputs = torch.randn(4, 300, 50, device=DEV)
    out = torch.empty(4, 300, 50, device=DEV)
    B.recurrence_forward(shared, inputs, out)
    ref, _, off, _ = P.recurrence(shared, inputs, None)
    P.assert_within(out, ref, off, "out")


@pytest.mark.parametrize("steps", [1, 5, 90, 700])
def test_one_token_after_the_other_is_the_whole_sequence(steps):
    gate, x, h0, _, _ = _inputs(4, steps, 100, F32)
    out, last = torch.empty_like(gate), torch.empty_like(h0)
    B.recurrence_forward(gate, x, out, h0=h0, h_last=last)
    state, one = h0.clone(), torch.empty(4, 1, 100, device=DEV)
    outs = []
    for t in range(steps):
        B.recurrence_forward(gate[:, t:t + 1], x[:, t:t + 1], one, h0=state, h_last=state)   # the state in place
        outs.append(one.clone())
    ref, ref_last, off, last_off = P.recurrence(gate, x, h0)
    P.assert_within(torch.cat(outs, 1), ref, off, "tokens")
    P.assert_within(state, ref_last, last_off, "state")
    P.assert_within(out, ref, off, "sequence")


def test_no_steps_and_no_sequences():
    h0, last = torch.randn(3, 40, device=DEV), torch.empty(3, 40, device=DEV)
    nothing = torch.empty(3, 0, 40, device=DEV)
    B.recurrence_forward(nothing, nothing, torch.empty_like(nothing), h0=h0, h_last=last)
    assert torch.equal(last, h0)
    dh0 = torch.empty(3, 40, device=DEV)
    B.recurrence_backward(nothing, nothing, nothing, nothing, torch.empty_like(nothing), torch.empty_like(nothing), h0=h0, grad_last=h0,
                          grad_h0=dh0)
    assert torch.equal(dh0, h0)
    none = torch.empty(0, 5, 40, device=DEV)
    B.recurrence_forward(none, none, torch.empty_like(none))


def test_gates_at_the_ends_of_their_range():
    f = torch.tensor([math.inf, -math.inf, 3.4e38, -3.4e38, 200.0, -200.0, 104.0, -104.0, 88.0, -88.0, 0.0, -0.0, 1e-30, 16.7, -16.7, 30.0],
                     device=DEV)
    gate = f.repeat(3, 6, 5)
    x, h0 = torch.randn(3, 6, 80, device=DEV), torch.randn(3, 80, device=DEV)
    out = torch.empty_like(x)
    B.recurrence_forward(gate, x, out, h0=h0)
    ref, _, off, _ = P.recurrence(gate, x, h0)
    P.assert_within(out, ref, off, "out")
    assert torch.equal(out[:, :, 0], h0[:, 0:1].expand(3, 6)) and torch.equal(out[:, :, 1], x[:, :, 1])


def test_a_nan_spoils_its_channel_from_its_step_on():
    gate, x, h0, _, _ = _inputs(2, 700, 64, F32)
    gate = gate.clamp(-5, 5)
    gate[0, 300, 7], x[1, 650, 9] = math.nan, math.nan
    out = torch.empty_like(gate)
    B.recurrence_forward(gate, x, out, h0=h0)
    bad = torch.zeros_like(gate, dtype=torch.bool)
    bad[0, 300:, 7], bad[1, 650:, 9] = True, True
    assert torch.equal(out.isnan(), bad)


def test_gradients_against_differences():
    batch, steps, channels, h = 2, 40, 3, 1e-5
    gen = torch.Generator().manual_seed(3)
    gate, x = (torch.randn(batch, steps, channels, generator=gen).to(DEV) for _ in range(2))
    h0, dlast = (torch.randn(batch, channels, generator=gen).to(DEV) for _ in range(2))
    dout = torch.randn(batch, steps, channels, generator=gen).to(DEV)
    out = torch.empty_like(gate)
    B.recurrence_forward(gate, x, out, h0=h0)
    dg, dx, dh = torch.empty_like(gate), torch.empty_like(gate), torch.empty_like(h0)
    B.recurrence_backward(gate, x, out, dout, dg, dx, h0=h0, grad_last=dlast, grad_h0=dh)

    def loss(gate_, x_, h0_):
        o, last, _, _ = P.recurrence(gate_, x_, h0_)
        return float((o * P.f64(dout)).sum() + (last * P.f64(dlast)).sum())

    for k, grad in enumerate((dg, dx, dh)):
        at = [t.double() for t in (gate, x, h0)]
        for _ in range(5):
            d = torch.randn(at[k].shape, generator=gen, dtype=torch.float64).to(DEV)
            up, down = list(at), list(at)
            up[k], down[k] = at[k] + h * d, at[k] - h * d
            slope = (loss(*up) - loss(*down)) / (2 * h)
            size = float((grad.double().abs() * d.abs()).sum())
            assert abs(float((grad.double() * d).sum()) - slope) <= 1e-5 * size + 1e-7


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("batch,steps,channels", [(3, 17, 65), (4, 200, 129), (5, 1100, 33), (3, 3000, 131), (1, 1024, 64)])
def test_the_state_in_place_over_many_steps(batch, steps, channels, dtype):
    print(f"case in place {batch} {steps} {channels} {dtype}", flush=True)
    gate, x, h0, _, _ = _inputs(batch, steps, channels, dtype, 4)
    for kind in (None, "empty", "whole"):
        lengths = _lengths(batch, steps, kind)
        out, last = torch.empty_like(gate), torch.empty_like(h0)
        B.recurrence_forward(gate, x, out, h0=h0, h_last=last, lengths=lengths)
        for _ in range(3):
            state, again = h0.clone(), torch.empty_like(gate)
            B.recurrence_forward(gate, x, again, h0=state, h_last=state, lengths=lengths)
            assert torch.equal(again, out) and torch.equal(state, last)


@pytest.mark.parametrize("batch,steps,channels", [(2, 40, 129), (1, 300, 257), (2, 130, 385), (3, 9, 129)])
def test_a_last_channel_alone_in_its_block(batch, steps, channels):
    """bf16, two channels per lane, 128 per block: the last block has one channel."""
    print(f"case alone {batch} {steps} {channels}", flush=True)
    gate, x, h0, dout, dlast = _inputs(batch, steps, channels, BF, 7)
    whole = [torch.full((batch, steps, channels + 2), 9.0, dtype=BF, device=DEV) for _ in range(3)]
    out, dgate, dinput = (w[:, :, :channels] for w in whole)
    last, dh0 = torch.empty_like(h0), torch.empty_like(h0)
    B.recurrence_forward(gate, x, out, h0=h0, h_last=last)
    ref, ref_last, off, last_off = P.recurrence(gate, x, h0)
    P.assert_within(out, ref, off, "out")
    P.assert_within(last, ref_last, last_off, "last")
    B.recurrence_backward(gate, x, out, dout, dgate, dinput, h0=h0, grad_last=dlast, grad_h0=dh0)
    ref, off = P.recurrence_gradients(gate, x, out, h0, dout, dlast)
    for got, r, o, what in zip((dgate, dinput, dh0), ref, off, ("dgate", "dinput", "dh0")):
        P.assert_within(got, r, o, what)
    for w in whole:
        assert w[:, :, channels:].eq(9).all()
