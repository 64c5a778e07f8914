"""The convolution, the scan and the log probabilities in 64 bits on the host, with bounds of what 32-bit arithmetic may differ by.

U is the rounding unit of fp32.  Every bound counts the roundings between an input and a result and charges each with U times the magnitude
it acts on; errors of intermediate values are carried through the derivatives of what follows.  SIGMOID: roundings of a sigmoid (an exponential of
up to seven units, a sum, a reciprocal and a product).
"""
from __future__ import annotations

import numpy as np

from tests.operators_plain import U, f64

SIGMOID = 12 * U


def _sigmoid(v):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-v))


def _lengths(lengths, batch, steps):
    return np.full(batch, steps) if lengths is None else np.clip(lengths.cpu().numpy().astype(np.int64), 0, steps)


# ---- convolution ----------------------------------------------------------------------------------------

def _windows(x, weight, bias, state, n):
    """(inputs behind the state's, u, bound of u) of one sequence's n steps."""
    k = weight.shape[1]
    front = np.zeros((k - 1, x.shape[1])) if state is None else state
    xs = np.concatenate([front, x[:n]])
    u, size = (np.zeros((n, x.shape[1])) + (0 if bias is None else b) for b in (bias, None if bias is None else np.abs(bias)))
    for j in range(k):
        u = u + weight[:, j] * xs[j:j + n]
        size = size + np.abs(weight[:, j] * xs[j:j + n])
    return xs, u, (k + 2) * U * size


def convolution(x, weight, bias, state, lengths, silu):
    """((out, last), bound of out); last is exact."""
    x, w, b, st = f64(x), f64(weight), None if bias is None else f64(bias), None if state is None else f64(state)
    out, off = np.zeros_like(x), np.zeros_like(x)
    last = np.zeros((x.shape[0], w.shape[1] - 1, x.shape[2]))
    for i, n in enumerate(_lengths(lengths, x.shape[0], x.shape[1])):
        xs, u, u_off = _windows(x[i], w, b, None if st is None else st[i], n)
        z = _sigmoid(u) if silu else 1.0
        out[i, :n] = u * z
        off[i, :n] = (1.1 * u_off if silu else u_off) + (SIGMOID + 2 * U if silu else U) * np.abs(out[i, :n])
        last[i] = xs[n:]
    return (out, last), off


def convolution_gradients(x, weight, bias, state, lengths, silu, dout, dlast):
    """((dx, dw, db, dstate), bounds)."""
    x, w, b, st = f64(x), f64(weight), None if bias is None else f64(bias), None if state is None else f64(state)
    go, k = f64(dout), w.shape[1]
    dx, dx_off = np.zeros_like(x), np.zeros_like(x)
    dw, dw_off, dw_size = (np.zeros_like(w) for _ in range(3))
    db, db_off, db_size = (np.zeros(w.shape[0]) for _ in range(3))
    ds, ds_off = (np.zeros((x.shape[0], k - 1, x.shape[2])) for _ in range(2))
    for i, n in enumerate(_lengths(lengths, x.shape[0], x.shape[1])):
        xs, u, u_off = _windows(x[i], w, b, None if st is None else st[i], n)
        g, g_off = go[i, :n], np.zeros_like(u)
        if silu:
            a, z = _sigmoid(u), _sigmoid(-u)
            # the derivative's own derivative is at most 1/2
            g_off = np.abs(g) * (0.5 * u_off + (2 * SIGMOID + 6 * U) * a * (1 + np.abs(u) * z))
            g = g * a * (1 + u * z)
        total, off = np.zeros_like(xs), np.zeros_like(xs)
        if dlast is not None:
            total[n:] = f64(dlast)[i]
            off[n:] = U * np.abs(total[n:])
        for j in range(k):
            total[j:j + n] += w[:, j] * g
            off[j:j + n] += (k + 3) * U * np.abs(w[:, j] * g) + np.abs(w[:, j]) * g_off
            dw[:, j] += (g * xs[j:j + n]).sum(0)
            dw_off[:, j] += (g_off * np.abs(xs[j:j + n])).sum(0)
            dw_size[:, j] += np.abs(g * xs[j:j + n]).sum(0)
        off[n:] += U * np.abs(total[n:])
        db, db_off, db_size = db + g.sum(0), db_off + g_off.sum(0), db_size + np.abs(g).sum(0)
        dx[i, :n], dx_off[i, :n] = total[k - 1:], off[k - 1:]
        ds[i], ds_off[i] = total[:k - 1], off[:k - 1]
    # a run's steps (up to 128), the runs of a workgroup (up to 64), the parts: 16 waves' shares of them, and the waves
    depth = 128 + 64 + x.shape[0] * x.shape[1] / 256 + 24
    return (dx, dw, db, ds), (dx_off, dw_off + depth * U * dw_size, db_off + depth * U * db_size, ds_off)


# ---- scan -----------------------------------------------------------------------------------------------

CHUNK = 256      # steps of a chunk at most, at the sizes of these tests: the roundings of a sum of its dt


class Scan:
    """Everything of one call, in 64 bits, with bounds; arrays are [batch, steps, channels(, states)]."""

    def __init__(self, x, delta, a, b, c, d=None, gate=None, delta_bias=None, softplus=False, h0=None, lengths=None):
        self.x, self.a = f64(x), f64(a)
        batch, steps, channels = self.x.shape
        n = self.a.shape[1]
        b, c = f64(b), f64(c)
        groups = b.shape[2] if b.ndim == 4 else 1
        self.groups = groups
        self.owner = np.arange(channels) // (channels // groups)
        self.b, self.c = (v.reshape(batch, steps, groups, n)[:, :, self.owner] for v in (b, c))
        self.on = (np.arange(steps)[None, :] < _lengths(lengths, batch, steps)[:, None])[:, :, None]
        clean = lambda v: np.where(self.on, v, 0.0)
        self.x = clean(self.x)
        self.b, self.c = (np.where(self.on[..., None], v, 0.0) for v in (self.b, self.c))
        self.d = np.zeros(channels) if d is None else f64(d)
        self.raw = clean(f64(delta)) + (0 if delta_bias is None else f64(delta_bias))
        self.soft = softplus
        self.sig = _sigmoid(self.raw)
        raw_off = U * np.abs(self.raw)
        if softplus:
            dt = np.logaddexp(self.raw, 0.0)
            dt_off = self.sig * raw_off + 14 * U * dt
        else:
            dt, dt_off = self.raw, raw_off
        self.dt, self.dt_off = clean(dt), clean(dt_off)
        self.u = self.dt * self.x
        self.u_off = self.dt_off * np.abs(self.x) + U * np.abs(self.u)
        self.gate = None if gate is None else clean(f64(gate))
        self.h0 = np.zeros((batch, channels, n)) if h0 is None else f64(h0)
        z = self.dt[..., None] * self.a
        self.e = np.exp(z)
        # the exponent's own roundings (a log2(e), its product with dt, the sums of a chunk), dt's error, and the power's
        self.e_rel = np.abs(z) * (4 + CHUNK) * U + np.abs(self.a) * self.dt_off[..., None] + 3 * U
        h, off = self.h0, np.zeros_like(self.h0)
        self.h, self.h_off = np.zeros(z.shape), np.zeros(z.shape)
        for t in range(steps):
            push = self.u[:, t, :, None] * self.b[:, t]
            new = self.e[:, t] * h + push
            off = self.e[:, t] * (off + np.abs(h) * self.e_rel[:, t]) + self.u_off[:, t, :, None] * np.abs(self.b[:, t]) + 2 * U * np.abs(push) \
                + 2 * U * (self.e[:, t] * np.abs(h) + np.abs(push))
            m = self.on[:, t, :, None]
            h, off = np.where(m, new, h), np.where(m, off, 0 * off + off)
            self.h[:, t], self.h_off[:, t] = h, off
        self.last, self.last_off = h, off
        terms = np.abs(self.c * self.h).sum(3) + np.abs(self.d * self.x)
        self.y = (self.c * self.h).sum(3) + self.d * self.x
        self.y_off = (np.abs(self.c) * self.h_off).sum(3) + (n + 3) * U * terms
        if gate is None:
            self.out, self.out_off = self.y, self.y_off
        else:
            s = self.gate * _sigmoid(self.gate)
            self.out, self.out_off = self.y * s, self.y_off * np.abs(s) + (SIGMOID + 3 * U) * np.abs(self.y * s)
        self.out, self.out_off = clean(self.out), clean(self.out_off)

    def gradients(self, dout, dlast=None):
        """({name: gradient}, {name: bound})."""
        go = np.where(self.on, f64(dout), 0.0)
        batch, steps, channels = self.x.shape
        n = self.a.shape[1]
        r, o = {}, {}
        if self.gate is None:
            dy, dy_off = go, 0 * go
        else:
            p, q = _sigmoid(self.gate), _sigmoid(-self.gate)
            dy = go * self.gate * p
            dy_off = (SIGMOID + 3 * U) * np.abs(dy)
            slope, size = p * (1 + self.gate * q), p * (1 + np.abs(self.gate) * q)
            r["gate"] = go * self.y * slope
            o["gate"] = np.abs(go) * (np.abs(slope) * self.y_off + (2 * SIGMOID + 8 * U) * np.abs(self.y) * size)
        before = np.concatenate([self.h0[:, None], self.h[:, :-1]], 1)
        before_off = np.concatenate([0 * self.h0[:, None], self.h_off[:, :-1]], 1)
        g = np.zeros_like(self.h0) if dlast is None else f64(dlast)
        off = np.zeros_like(g)
        G, G_off = np.zeros_like(self.e), np.zeros_like(self.e)
        for t in reversed(range(steps)):
            m = self.on[:, t, :, None]
            push = self.c[:, t] * dy[:, t, :, None]
            total = push + g
            total_off = off + np.abs(self.c[:, t]) * dy_off[:, t, :, None] + 3 * U * (np.abs(push) + np.abs(g))
            G[:, t], G_off[:, t] = np.where(m, total, 0), np.where(m, total_off, 0)
            back = self.e[:, t] * total
            back_off = self.e[:, t] * (total_off + np.abs(total) * (self.e_rel[:, t] + 2 * U))
            g, off = np.where(m, back, g), np.where(m, back_off, off)
        r["h0"], o["h0"] = g, off
        dt, dt_off = self.dt[..., None], self.dt_off[..., None]
        gb = G * self.b
        along, along_off = gb.sum(3), (G_off * np.abs(self.b)).sum(3) + (n + 2) * U * np.abs(gb).sum(3)
        r["x"] = self.dt * along + self.d * dy
        o["x"] = self.dt * along_off + self.dt_off * np.abs(along) + np.abs(self.d) * dy_off + 3 * U * (np.abs(self.dt * along) + np.abs(self.d * dy))
        back = G * self.e * before
        back_off = self.e * (G_off * np.abs(before) + np.abs(G) * before_off) + np.abs(back) * (self.e_rel + 3 * U)
        step = (back * self.a).sum(3) + along * self.x
        step_off = (back_off * np.abs(self.a)).sum(3) + (n + 5) * U * np.abs(back * self.a).sum(3) + along_off * np.abs(self.x) + 2 * U * np.abs(along * self.x)
        if self.soft:
            # (the sigmoid's own argument is rounded once)
            rel = SIGMOID + U * np.abs(self.raw)
            step, step_off = step * self.sig, step_off * self.sig + rel * np.abs(step * self.sig)
        r["delta"], o["delta"] = np.where(self.on, step, 0), np.where(self.on, step_off + U * np.abs(step), 0)
        by = np.eye(self.groups)[self.owner]                # [channels, groups]
        spread = channels // self.groups / 64 + 10          # roundings of a sum over the channels
        u, u_off = self.u[..., None], self.u_off[..., None]
        gather = lambda v: np.einsum("btcn,cg->btgn", v, by)
        r["b"], o["b"] = gather(G * u), gather(G_off * np.abs(u) + np.abs(G) * u_off + spread * U * np.abs(G * u))
        hy = dy[..., None] * self.h
        r["c"] = gather(hy)
        o["c"] = gather(np.abs(dy[..., None]) * self.h_off + dy_off[..., None] * np.abs(self.h) + spread * U * np.abs(hy))
        depth = CHUNK + 16 + batch * (steps / 16 + 1) / 16 + 8       # a chunk's steps, the shares of the chunks, the waves
        sums = (0, 1)
        r["a"] = (back * dt).sum(sums)
        o["a"] = (back_off * dt + np.abs(back) * dt_off + depth * U * np.abs(back * dt)).sum(sums)
        r["d"] = (dy * self.x).sum(sums)
        o["d"] = ((dy_off + depth * U * np.abs(dy)) * np.abs(self.x)).sum(sums)
        r["delta_bias"] = r["delta"].sum(sums)
        o["delta_bias"] = (o["delta"] + depth * U * np.abs(r["delta"])).sum(sums)
        return r, o


# ---- log probabilities ----------------------------------------------------------------------------------

def logprob(logits):
    """(lse, log probabilities, entropy, and the bounds of lse, of log probabilities and of entropy) of rows."""
    x = f64(logits)
    v = x.shape[1]
    with np.errstate(invalid="ignore", divide="ignore"):
        top = x.max(1, keepdims=True)
        d = x - top
        e = np.where(x == -np.inf, 0.0, np.exp(d))
        s = e.sum(1, keepdims=True)
        lse = np.where(s > 0, top + np.log(s), -np.inf)
        lp = d - np.log(s)           # (not x - lse: next to logits of 1e38 even 64 bits hold no log s)
        p = e / s
        pd = np.where(p > 0, p * d, 0.0)
        t = pd.sum(1, keepdims=True)
        entropy = np.log(s) - t
        # an exponential's argument is rounded twice, it itself by two units; a lane's sums, their scaling where a larger logit comes, the
        # lanes', the waves' and the parts' sums
        depth = v / 256 + 3 * (v / 4096 + 1) + 60
        far = np.where(p > 0, np.abs(d), 0.0)
        rel = (p * (4 * far + 4)).sum(1, keepdims=True) * U + depth * U
        log_s = np.abs(np.log(s))
        base = rel + 3 * U * log_s
        lse_off = base + U * np.abs(lse)
        lp_off = base + U * np.abs(d) + U * np.abs(lp)
        ent_off = base + np.abs(t) * (rel + (depth + 4) * U) + (p * far * (4 * far + 8)).sum(1, keepdims=True) * U + U * np.abs(entropy)
    empty = top[:, 0] == -np.inf          # (without a token: by definition)
    lse[empty], lp[empty], entropy[empty] = -np.inf, -np.inf, 0.0
    lse_off[empty], lp_off[empty], ent_off[empty] = 0.0, np.inf, 0.0
    return lse[:, 0], lp, entropy[:, 0], lse_off[:, 0], lp_off, ent_off[:, 0]


def logprob_gradient(logits, targets, lse, g, entropy=None, ge=None):
    """(gradient, bound); lse and entropy as they are."""
    x, lse = f64(logits), f64(lse)[:, None]
    rows, v = x.shape
    ids = np.full(rows, -1) if targets is None else targets.cpu().numpy().astype(np.int64)
    named = (ids >= 0) & (ids < v)
    g = np.where(named, np.zeros(rows) if g is None else f64(g), 0.0)[:, None]
    hit = (np.arange(v)[None, :] == ids[:, None]) & named[:, None]
    with np.errstate(invalid="ignore"):
        lp = x - lse
        p = np.exp(lp)
        rel = (np.where(p > 0, np.abs(lp), 0.0) + 10) * U
        grad = g * (hit - p)
        off = np.abs(g) * p * rel + U * np.abs(grad)
        if ge is not None:
            ge, h = f64(ge)[:, None], f64(entropy)[:, None]
            inner = np.where(p > 0, p * (lp + h), 0.0)
            grad = grad - ge * inner
            off = off + np.abs(ge) * np.where(p > 0, p * (np.abs(lp) + np.abs(h)), 0.0) * (rel + 6 * U) + U * np.abs(grad)
    dead = lse[:, 0] == -np.inf
    grad[dead], off[dead] = 0, 0
    return grad, off


def best(logits, k):
    """Ids of the k largest of every row, of equal ones the lowest index first, a NaN the least."""
    x = f64(logits)
    order = np.where(np.isnan(x), -np.inf, x)
    ids = np.argsort(np.stack([np.isnan(x), np.zeros_like(x)], -1)[..., 0] * 0 - order, axis=1, kind="stable")
    nan = np.take_along_axis(np.isnan(x), ids, 1)
    # NaN behind -infinity
    return np.stack([np.concatenate([r[~m], r[m]]) for r, m in zip(ids, nan)])[:, :k]
