"""Offsets beyond 2^31 elements: the last rows, steps and blocks of large buffers are the right ones."""
import math

import numpy as np
import pytest
import torch

from paper_2010_16248_amd import binding as B
from tests import operators_plain as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16
ROWS, DIM = 2_200_000, 1024          # 2.25e9 elements


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def test_embedding():
    print("case large embedding", flush=True)
    table = torch.zeros(ROWS, DIM, dtype=BF, device=DEV)
    ids = torch.tensor([ROWS - 1, 0, ROWS - 2, 2_097_152, 2_097_151, ROWS], device=DEV)
    table[ids[:5]] = torch.arange(1, 6, device=DEV, dtype=BF)[:, None].expand(5, DIM)
    out = torch.empty(6, DIM, dtype=BF, device=DEV)
    B.embedding_forward(ids, table, out, 2.0)
    assert torch.equal(out.float(), torch.tensor([2.0, 4, 6, 8, 10, 0], device=DEV)[:, None].expand(6, DIM))
    del table
    grad = torch.full((ROWS, DIM), 7.0, device=DEV)
    B.embedding_backward(ids, out, grad, 0.5)
    for i, v in zip(ids[:5].tolist(), (1.0, 2, 3, 4, 5)):
        assert grad[i].eq(v).all()
    assert grad[ROWS - 3].eq(0).all() and grad[2_097_150].eq(0).all() and grad[1].eq(0).all()
    assert float(grad.sum(dtype=torch.float64)) == 15.0 * DIM


def test_embedding_with_more_gradients_than_31_bits_of_elements():
    print("case large embedding gradients", flush=True)
    g = torch.zeros(ROWS, DIM, dtype=BF, device=DEV)
    ids = torch.full((ROWS,), 3, dtype=torch.int32, device=DEV)
    g[-1], g[0], ids[-1], ids[0] = 5.0, 2.0, 8, 1
    table = torch.empty(10, DIM, device=DEV)
    B.embedding_backward(ids, g, table)
    ref = torch.zeros(10, device=DEV)
    ref[8], ref[1] = 5.0, 2.0
    assert torch.equal(table, ref[:, None].expand(10, DIM))


def test_layernorm():
    print("case large layer norm", flush=True)
    x = torch.ones(ROWS, DIM, dtype=BF, device=DEV)
    gen = torch.Generator().manual_seed(1)
    last = torch.randn(3, DIM, generator=gen).to(BF)
    x[-3:] = last.to(DEV)
    w, b = torch.ones(DIM, device=DEV), torch.zeros(DIM, device=DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty(ROWS, device=DEV), torch.empty(ROWS, device=DEV)
    B.layernorm_forward(x, w, b, y, mean, rstd)
    ref = P.layernorm(last, w, b, float(np.float32(1e-5)))
    P.assert_within(y[-3:], ref[0], P.layernorm_bounds(last, w, b, 1e-5)[0], "y")
    assert y[:-3].eq(0).all() and mean[:-3].eq(1).all()
    dx, dw, db = torch.full_like(x, 3.0), torch.empty(DIM, device=DEV), torch.empty(DIM, device=DEV)
    dy = y.mul_(0)                   # a gradient in the last rows alone
    dy[-3:] = 1.0
    B.layernorm_backward(dy, x, w, mean, rstd, dx, dw, db)
    ref, off = P.layernorm_gradients(dy[-3:], x[-3:], w, mean[-3:], rstd[-3:])
    P.assert_within(dx[-3:], ref[0], off[0], "dx")
    P.assert_within(dw, ref[1], off[1], "dw")
    assert db.eq(3).all() and dx[:-3].eq(0).all()


def test_recurrence():
    print("case large recurrence", flush=True)
    steps, tail = ROWS, 40
    gate = torch.full((1, steps, DIM), 3.0, dtype=BF, device=DEV)
    x = torch.ones(1, steps, DIM, dtype=BF, device=DEV)
    gen = torch.Generator().manual_seed(2)
    # a shut gate cuts the last steps off from everything before them
    gate[:, -tail] = -math.inf
    x[:, -tail:] = torch.randn(1, tail, DIM, generator=gen).to(BF).to(DEV)
    out, last = torch.empty_like(x), torch.empty(1, DIM, device=DEV)
    B.recurrence_forward(gate, x, out, h_last=last)
    ref, ref_last, off, last_off = P.recurrence(gate[:, -tail:], x[:, -tail:], None)
    P.assert_within(out[:, -tail:], ref, off, "out")
    P.assert_within(last, ref_last, last_off, "last")
    assert (out[:, -tail - 1].float() - 1).abs().max() < 0.01 and (out[:, steps // 2].float() - 1).abs().max() < 0.01
    # backward: the gradient of the last steps alone, which the shut gate keeps there
    dout = torch.zeros_like(x)
    dout[:, -tail:] = torch.randn(1, tail, DIM, generator=gen).to(BF).to(DEV)
    dgate, dinput, dh0 = torch.full_like(x, 3.0), torch.full_like(x, 3.0), torch.empty(1, DIM, device=DEV)
    B.recurrence_backward(gate, x, out, dout, dgate, dinput, grad_h0=dh0)
    first = out[:, -tail - 1].float()
    ref, off = P.recurrence_gradients(gate[:, -tail:], x[:, -tail:], out[:, -tail:], first, dout[:, -tail:], None)
    P.assert_within(dgate[:, -tail:], ref[0], off[0], "dgate")
    P.assert_within(dinput[:, -tail:], ref[1], off[1], "dinput")
    assert dgate[:, :-tail].eq(0).all() and dinput[:, :-tail].eq(0).all() and dh0.eq(0).all()


def test_adamw():
    print("case large adamw", flush=True)
    n = ROWS * DIM
    w, g = torch.zeros(n, dtype=BF, device=DEV), torch.zeros(n, dtype=BF, device=DEV)
    g[-5:], g[2 ** 31 + 3] = 1.0, 1.0
    small_w, small_g = torch.zeros(100, dtype=BF, device=DEV), torch.ones(100, dtype=BF, device=DEV)
    state = B.adamw_state([n, 100], 8)
    B.adamw_step([w, small_w], [g, small_g], state, 0.5, 1)
    assert w[-5:].eq(-0.5).all() and w[2 ** 31 + 3] == -0.5 and int(w.ne(0).sum()) == 6
    assert small_w.eq(-0.5).all() and state[0][-256:].float()[:100].eq(448).all()
