"""The language-model operators in 64 bits on the host, with bounds of what 32-bit arithmetic may differ by.

U is the rounding unit of fp32.  Every bound counts the roundings between an input and a result and charges each with U times the
magnitude it acts on.  A result stored as bf16 has to be the bf16 rounding of a value within its bound.
"""
from __future__ import annotations

import numpy as np
import torch

U = 2.0 ** -24
TINY = 1e-37        # below it fp32 and bf16 lose digits


def f64(t):
    return t.detach().double().cpu().numpy()


def assert_within(got, ref, bound, what):
    """got is ref to within bound, rounded to got's type."""
    kind = got.dtype
    got = f64(got)
    assert got.shape == ref.shape, f"{what}: shape {got.shape}, not {ref.shape}"
    nan = np.isnan(ref)
    assert np.array_equal(np.isnan(got), nan), f"{what}: NaN in other places"
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf]), f"{what}: infinities differ"
    fine = ~nan & ~inf
    far = np.broadcast_to(bound, ref.shape)[fine] + U * np.abs(ref[fine]) + TINY

    def rounded(v):
        return torch.from_numpy(v).float().to(kind).double().numpy() if kind == torch.bfloat16 else v

    low, high = rounded(ref[fine] - far), rounded(ref[fine] + far)
    off = np.maximum(low - got[fine], got[fine] - high)
    assert off.size == 0 or off.max() <= 0, f"{what}: {np.sum(off > 0)} of {off.size} beyond their bound, the worst by {off.max():.3e}"


def tree_depth(n):
    """Roundings on the way of one term through a sum of n terms: up to 32 in a lane's registers, one every 256 beyond them, then the
    lanes, the waves and the workgroups."""
    return 32 + n / 256 + 16


# ---- embedding ------------------------------------------------------------------------------------------

def embedding_gradient(ids, grad_out, vocab, scale, start=None):
    """(gradient, bound)."""
    g, ids = f64(grad_out), ids.cpu().numpy().reshape(-1).astype(np.int64)
    ok = (ids >= 0) & (ids < vocab)
    total, size, count = (np.zeros((vocab, g.shape[-1])) for _ in range(3))
    g = g.reshape(-1, g.shape[-1])
    np.add.at(total, ids[ok], g[ok])
    np.add.at(size, ids[ok], np.abs(g[ok]))
    np.add.at(count, ids[ok], 1.0)
    ref, bound = total * scale, (count + 2) * U * size * abs(scale)
    if start is not None:
        ref = ref + f64(start)
        bound = bound + U * np.abs(ref)
    return ref, bound


# ---- layer norm -----------------------------------------------------------------------------------------

def layernorm(x, weight, bias, eps):
    x, w = f64(x), f64(weight)
    mean = x.mean(-1, keepdims=True)
    rstd = 1 / np.sqrt(x.var(-1, keepdims=True) + eps)
    xh = (x - mean) * rstd
    y = xh * w + (0 if bias is None else f64(bias))
    return y, mean[..., 0], rstd[..., 0], xh


def layernorm_bounds(x, weight, bias, eps):
    """Bounds of y, mean and rstd."""
    y, mean, rstd, xh = layernorm(x, weight, bias, eps)
    n = x.shape[-1]
    d = tree_depth(n)
    mean_off = (d + 2) * U * np.abs(f64(x)).mean(-1, keepdims=True)
    # the deviations' common shift enters their squares in second order only; their own roundings in first order
    shift = mean_off * rstd[..., None]
    rstd_rel = (d + 12) * U + shift ** 2 + 2 * U * np.abs(mean[..., None]) * rstd[..., None]
    off = np.abs(f64(weight)) * (shift + np.abs(xh) * (rstd_rel + 4 * U) + 2 * U * np.abs(mean[..., None]) * rstd[..., None])
    off = off + 2 * U * (np.abs(y) + (0 if bias is None else np.abs(f64(bias))))
    return off, mean_off[..., 0] + U * np.abs(mean), rstd * rstd_rel[..., 0]


def layernorm_gradients(dy, x, weight, mean, rstd):
    """((dx, dw, db), bounds); mean and rstd are taken as they are."""
    dy, x, w = f64(dy), f64(x), f64(weight)
    mean, rstd = f64(mean)[:, None], f64(rstd)[:, None]
    n, rows = x.shape[1], x.shape[0]
    xh = (x - mean) * rstd
    xh_off = 3 * U * (np.abs(x) + np.abs(mean)) * rstd
    g = dy * w
    sg, sgx = g.mean(1, keepdims=True), (g * xh).mean(1, keepdims=True)
    dx = rstd * (g - sg - xh * sgx)
    d = tree_depth(n) + 4
    sg_off = d * U * np.abs(g).mean(1, keepdims=True)
    sgx_off = d * U * np.abs(g * xh).mean(1, keepdims=True) + (np.abs(g) * xh_off).mean(1, keepdims=True)
    dx_off = rstd * (6 * U * (np.abs(g) + np.abs(sg) + np.abs(xh * sgx)) + sg_off + np.abs(xh) * sgx_off + xh_off * np.abs(sgx))
    d = rows + 40 if rows < 4096 else rows / 64 + 200     # a lane's rows, then groups and workgroups
    dw_off = d * U * np.abs(dy * xh).sum(0) + (np.abs(dy) * xh_off).sum(0)
    db_off = d * U * np.abs(dy).sum(0)
    return (dx, (dy * xh).sum(0), dy.sum(0)), (dx_off, dw_off, db_off)


# ---- recurrence -----------------------------------------------------------------------------------------

def _gates(gate, lengths):
    f = f64(gate)
    with np.errstate(over="ignore"):
        a, z = 1 / (1 + np.exp(-f)), 1 / (1 + np.exp(f))
    on = np.ones(f.shape[:2] + (1,), bool)
    if lengths is not None:
        on = (np.arange(f.shape[1])[None, :] < np.clip(lengths.cpu().numpy(), 0, f.shape[1])[:, None])[:, :, None]
    return a, z, np.broadcast_to(on, f.shape)


# Roundings of one step: the gates (an exponential of two units, a reciprocal, a product: six), their product with the state or the
# input and the sum; twice that, because chunks carry the gates' product and the state apart.
STEP = 16 * U


def recurrence(gate, x, h0, lengths=None):
    """(out, last, bound of out, bound of last)."""
    a, z, on = _gates(gate, lengths)
    x = f64(x)
    h = np.zeros((a.shape[0], a.shape[2])) if h0 is None else f64(h0)
    off, out, bound = np.zeros_like(h), np.zeros_like(a), np.zeros_like(a)
    for t in range(a.shape[1]):
        m = on[:, t]
        with np.errstate(invalid="ignore"):
            new_off = a[:, t] * off + STEP * (a[:, t] * np.abs(h) + z[:, t] * np.abs(x[:, t]))
            new = a[:, t] * h + z[:, t] * x[:, t]
        h, off = np.where(m, new, h), np.where(m, new_off, off)
        out[:, t], bound[:, t] = np.where(m, h, 0), np.where(m, off, 0)
    return out, h, bound, off


def recurrence_gradients(gate, x, out, h0, dout, dlast, lengths=None):
    """((dgate, dinput, dh0), bounds); out is taken as it is."""
    a, z, on = _gates(gate, lengths)
    x, d = f64(x), f64(dout)
    zeros = np.zeros((a.shape[0], 1, a.shape[2]))
    before = np.concatenate([zeros if h0 is None else f64(h0)[:, None], f64(out)[:, :-1]], 1)
    g = np.zeros_like(zeros[:, 0]) if dlast is None else f64(dlast)
    off = np.zeros_like(g)
    dgate, dinput, dgate_off, dinput_off = (np.zeros_like(a) for _ in range(4))
    for t in reversed(range(a.shape[1])):
        m = on[:, t]
        total = g + d[:, t]
        toff = off + U * np.abs(total)
        az = a[:, t] * z[:, t]
        dinput[:, t] = np.where(m, z[:, t] * total, 0)
        dinput_off[:, t] = np.where(m, z[:, t] * (toff + STEP * np.abs(total)), 0)
        dgate[:, t] = np.where(m, total * (before[:, t] - x[:, t]) * az, 0)
        dgate_off[:, t] = np.where(m, (toff + STEP * np.abs(total)) * (np.abs(before[:, t]) + np.abs(x[:, t])) * az, 0)
        off = np.where(m, a[:, t] * toff + STEP * a[:, t] * np.abs(total), off)
        g = np.where(m, a[:, t] * total, g)
    return (dgate, dinput, g), (dgate_off, dinput_off, off)


# ---- AdamW ----------------------------------------------------------------------------------------------

def adamw_scalars(lr, step, betas, eps, decay):
    f = np.float32
    return dict(b1=f(betas[0]), c1=f(1 - betas[0]), b2=f(betas[1]), c2=f(1 - betas[1]), rate=f(lr / (1 - betas[0] ** step)),
                up=f(1 / np.sqrt(1 - betas[1] ** step)), eps=f(eps), keep=f(1 - lr * float(f(decay))))


def adamw32(w, g, m, v, lr, step, betas, eps, decay, grad_scale=None):
    """One tensor's step in fp32, every product and sum rounded on its own: (w, m, v, sqrt(v)) of fp32 arrays."""
    k = adamw_scalars(lr, step, betas, eps, decay)
    if grad_scale is not None:
        g = g * np.float32(grad_scale)
    m = k["b1"] * m + k["c1"] * g
    v = k["b2"] * v + (k["c2"] * g) * g
    root = np.sqrt(v)
    w = w * k["keep"] - (k["rate"] * m) / (root * k["up"] + k["eps"])
    return w, m, v, root


def adamw64(w, g, m, v, lr, step, betas, eps, decay, grad_scale=None):
    """The textbook step in 64 bits: (w, m, v)."""
    w, g, m, v = (np.asarray(t, np.float64) for t in (w, g, m, v))
    g = g * (1 if grad_scale is None else grad_scale)
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    mh, vh = m / (1 - betas[0] ** step), v / (1 - betas[1] ** step)
    return w - lr * decay * w - lr * mh / (np.sqrt(vh) + eps), m, v


def encode(x, root):
    """(codes as uint8, scales) of an fp32 array, blocks of 256, zeros up to a whole block."""
    f = np.float32
    x = np.concatenate([x, np.zeros(-len(x) % 256, f)]).reshape(-1, 256)
    top = np.max(np.abs(x), axis=1, keepdims=True)            # NaN if there is one
    held = ~(top < f(2.0 ** -100))
    with np.errstate(invalid="ignore", divide="ignore"):
        y = x * np.where(held, f(448) / top, f(0))
    if root:
        y = np.where(held & (x > 0) & (y < f(2.0 ** -9)), f(2.0 ** -9), y)
    codes = torch.from_numpy(np.ascontiguousarray(y, f)).to(torch.float8_e4m3fn).view(torch.uint8).numpy().reshape(-1)
    return codes, np.where(held, top * f(1 / 448), f(0))[:, 0]


def decode(codes, scales):
    v = torch.from_numpy(codes).view(torch.float8_e4m3fn).float().numpy().reshape(-1, 256)
    return (v * scales[:, None]).reshape(-1)
