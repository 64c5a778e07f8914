"""Layer norm's forward and backward pass against the formula and, for the gradients, against differences."""
import math

import numpy as np
import pytest
import torch

from paper_2010_16248_amd import binding as B
from tests import operators_plain as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF = torch.float32, torch.bfloat16

# rows, dim: one element, one lane, vectors that end inside a request, every width of the register kernels and beyond it
SIZES = [(1, 1), (3, 2), (5, 63), (130, 64), (7, 255), (64, 256), (33, 257), (700, 672), (21, 1000), (9, 1001), (6, 1025), (5, 2047),
         (4, 2049), (11, 4096), (3, 4100), (5, 8191), (2, 8193), (3, 16384), (2, 16385), (2, 40001), (5003, 40)]


def _inputs(rows, dim, dtype, seed=0):
    gen = torch.Generator().manual_seed(rows * 131 + dim + seed)
    x = (torch.randn(rows, dim, generator=gen) * torch.exp(torch.randn(rows, 1, generator=gen)) + torch.randn(rows, 1, generator=gen))
    w, b = 1 + 0.3 * torch.randn(dim, generator=gen), torch.randn(dim, generator=gen)
    return gen, x.to(dtype).to(DEV), w.to(DEV), b.to(DEV)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,dim", SIZES)
def test_forward(rows, dim, dtype):
    print(f"case layernorm forward {rows} {dim} {dtype}", flush=True)
    _, x, w, b = _inputs(rows, dim, dtype)
    eps = 1e-5
    for bias in (b, None):
        y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
        B.layernorm_forward(x, w, bias, y, mean, rstd, eps=eps)
        ref_y, ref_m, ref_r, _ = P.layernorm(x, w, bias, float(np.float32(eps)))
        y_off, m_off, r_off = P.layernorm_bounds(x, w, bias, float(np.float32(eps)))
        P.assert_within(mean, ref_m, m_off, "mean")
        P.assert_within(rstd, ref_r, r_off, "rstd")
        P.assert_within(y, ref_y, y_off, "y")
    y2 = torch.empty_like(x)
    B.layernorm_forward(x, w, None, y2, eps=eps)
    assert torch.equal(y2, y)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,dim", SIZES + [(40000, 24)])
def test_backward(rows, dim, dtype):
    print(f"case layernorm backward {rows} {dim} {dtype}", flush=True)
    gen, x, w, b = _inputs(rows, dim, dtype)
    dy = torch.randn(rows, dim, generator=gen).to(dtype).to(DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    B.layernorm_forward(x, w, b, y, mean, rstd)
    dx, dw, db = torch.empty_like(x), torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)
    B.layernorm_backward(dy, x, w, mean, rstd, dx, dw, db)
    ref, off = P.layernorm_gradients(dy, x, w, mean, rstd)
    P.assert_within(dx, ref[0], off[0], "dx")
    P.assert_within(dw, ref[1], off[1], "dw")
    P.assert_within(db, ref[2], off[2], "db")
    # without a bias, and on top of what is there
    dx2, dw2 = torch.empty_like(x), dw.clone()
    B.layernorm_backward(dy, x, w, mean, rstd, dx2, dw2, None, accumulate=True)
    assert torch.equal(dx2, dx) and torch.equal(dw2, dw + dw)


def test_gradients_against_differences():
    rows, dim, eps, h = 6, 37, 1e-5, 1e-5
    gen, x, w, b = _inputs(rows, dim, F32, 5)
    dy = torch.randn(rows, dim, generator=gen).to(DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    B.layernorm_forward(x, w, b, y, mean, rstd, eps=eps)
    dx, dw, db = torch.empty_like(x), torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)
    B.layernorm_backward(dy, x, w, mean, rstd, dx, dw, db)

    def loss(x_, w_, b_):
        return float((P.layernorm(x_, w_, b_, eps)[0] * P.f64(dy)).sum())

    for k, grad in enumerate((dx, dw, db)):
        at = [t.double() for t in (x, w, b)]
        for _ in range(5):
            d = torch.randn(at[k].shape, generator=gen, dtype=torch.float64).to(DEV)
            up, down = list(at), list(at)
            up[k], down[k] = at[k] + h * d, at[k] - h * d
            slope = (loss(*up) - loss(*down)) / (2 * h)
            # the difference is off by h^2 times third derivatives (of the order of the slopes' own size) and by 1e-16 / h
            size = float((grad.double().abs() * d.abs()).sum())
            assert abs(float((grad.double() * d).sum()) - slope) <= 1e-5 * size + 1e-7


def test_rows_apart_leave_what_lies_between():
    gen, x, w, b = _inputs(30, 50, F32)
    big, out = torch.randn(30, 80, generator=gen).to(DEV), torch.full((30, 70), 3.0, device=DEV)
    mean, rstd = torch.empty(30, device=DEV), torch.empty(30, device=DEV)
    B.layernorm_forward(big[:, 3:53], w, b, out[:, 11:61], mean, rstd)
    ref = P.layernorm(big[:, 3:53], w, b, float(np.float32(1e-5)))[0]
    P.assert_within(out[:, 11:61], ref, P.layernorm_bounds(big[:, 3:53], w, b, 1e-5)[0], "y")
    assert (out[:, :11] == 3).all() and (out[:, 61:] == 3).all()
    dx = torch.full((30, 60), 5.0, device=DEV)
    dw, db = torch.empty(50, device=DEV), torch.empty(50, device=DEV)
    B.layernorm_backward(big[:, 20:70], big[:, 3:53], w, mean, rstd, dx[:, 2:52], dw, db)
    ref, off = P.layernorm_gradients(big[:, 20:70], big[:, 3:53], w, mean, rstd)
    P.assert_within(dx[:, 2:52], ref[0], off[0], "dx")
    P.assert_within(dw, ref[1], off[1], "dw")
    assert (dx[:, :2] == 5).all() and (dx[:, 52:] == 5).all()


def test_special_rows():
    # a constant row, a row with an infinity, one with NaN; no rows
    x = torch.randn(4, 100, device=DEV)
    x[0], x[1, 7], x[2, 99] = 2.0, math.inf, math.nan
    w, b = torch.ones(100, device=DEV), torch.full((100,), 0.5, device=DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty(4, device=DEV), torch.empty(4, device=DEV)
    B.layernorm_forward(x, w, b, y, mean, rstd)
    assert y[0].eq(0.5).all() and y[1].isnan().any() and y[2].isnan().all() and y[3].isfinite().all()
    empty = torch.empty(0, 100, device=DEV)
    none = torch.empty(0, device=DEV)
    B.layernorm_forward(empty, w, b, torch.empty_like(empty), none, none)
    dw, db = torch.full((100,), 3.0, device=DEV), torch.full((100,), 3.0, device=DEV)
    B.layernorm_backward(empty, empty, w, none, none, torch.empty_like(empty), dw, db)
    assert dw.eq(0).all() and db.eq(0).all()


# Rows beyond what all workgroups of the backward pass have under way at once, with dense gradients, in every form of it: 16 lanes per
# row with one and two requests each, a wave with one, two and four, a workgroup of 256, 512 and 1024, and rows beyond the registers
TURNS = [(9000, 53), (9000, 67), (9000, 100), (4500, 201), (4500, 300), (5000, 1001), (4500, 1501), (600, 1801), (600, 2049), (600, 4100),
         (530, 8193), (530, 16385)]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,dim", TURNS)
def test_backward_where_workgroups_take_several_rows(rows, dim, dtype):
    print(f"case layernorm turns {rows} {dim} {dtype}", flush=True)
    gen, x, w, b = _inputs(rows, dim, dtype, 9)
    dy = torch.randn(rows, dim, generator=gen).to(dtype).to(DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    B.layernorm_forward(x, w, b, y, mean, rstd)
    ref_y, ref_m, ref_r, _ = P.layernorm(x, w, b, float(np.float32(1e-5)))
    y_off, m_off, r_off = P.layernorm_bounds(x, w, b, float(np.float32(1e-5)))
    P.assert_within(y, ref_y, y_off, "y")
    P.assert_within(mean, ref_m, m_off, "mean")
    P.assert_within(rstd, ref_r, r_off, "rstd")
    dx, dw, db = torch.empty_like(x), torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)
    B.layernorm_backward(dy, x, w, mean, rstd, dx, dw, db)
    ref, off = P.layernorm_gradients(dy, x, w, mean, rstd)
    P.assert_within(dx, ref[0], off[0], "dx")
    P.assert_within(dw, ref[1], off[1], "dw")
    P.assert_within(db, ref[2], off[2], "db")
