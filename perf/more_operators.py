"""More operators of a language model, as cases that can be timed and compared: a mixing layer's convolution and scan, and the
log probabilities of its tokens.

One pass is one call of one operator:

  convolution  out_t = act(bias + sum_j weight_j x_{t-width+1+j}) per channel along a sequence; forward with the inputs that the next
               call starts from (one step: its serving form); backward: gradients of inputs, weight, bias and first state
  scan         h_t = exp(dt_t a) h_{t-1} + dt_t b_t x_t with dt = softplus(delta + bias), out_t = (c_t . h_t + d x_t) silu(gate_t), a state
               of `states` numbers per channel; forward with the last state (one step: its serving form); backward: all gradients
  logprob      log probability of a given token per row of logits, the row's entropy and its most probable tokens; backward: the
               logits' gradient

`type` is the type of activations and their gradients (f32, bf16); `dir` the direction.  Where `own` is set the passes go through
the library's entry points, otherwise through elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}


def listed():
    return [
        # serving: one token for each of 64 sequences
        dict(name="convolution_forward_token", op="convolution", dir="forward", batch=64, steps=1, channels=1344, width=4, type="bf16",
             silu=True, bias=True, ragged=False),
        # prompts of different lengths, odd number of channels: rows that start off 16-byte boundaries
        dict(name="convolution_forward_ragged", op="convolution", dir="forward", batch=7, steps=1999, channels=1001, width=3, type="f32",
             silu=False, bias=False, ragged=True),
        # a training batch in bf16
        dict(name="convolution_backward_large", op="convolution", dir="backward", batch=8, steps=4096, channels=4096, width=4,
             type="bf16", silu=True, bias=True, ragged=False),
        # serving: one token for each of 64 sequences
        dict(name="scan_forward_token", op="scan", dir="forward", batch=64, steps=1, channels=1344, states=16, groups=1, type="bf16",
             gate=True, softplus=True, ragged=False),
        # one long document: the parallel work has to come from the sequence
        dict(name="scan_forward_long", op="scan", dir="forward", batch=1, steps=65536, channels=672, states=16, groups=1, type="f32",
             gate=False, softplus=True, ragged=False),
        # prompts in bf16 for serving, padded to the longest
        dict(name="scan_forward_prompts", op="scan", dir="forward", batch=8, steps=4096, channels=2048, states=16, groups=1,
             type="bf16", gate=True, softplus=True, ragged=True),
        # odd sizes, groups of channels with their own b and c, steps given as they are
        dict(name="scan_backward_odd", op="scan", dir="backward", batch=3, steps=777, channels=333, states=5, groups=3, type="f32",
             gate=False, softplus=False, ragged=True),
        # a training batch in bf16
        dict(name="scan_backward_large", op="scan", dir="backward", batch=8, steps=4096, channels=2048, states=16, groups=1,
             type="bf16", gate=True, softplus=True, ragged=False),
        # serving: the tokens just sampled, with 20 alternatives each
        dict(name="logprob_forward_tokens", op="logprob", dir="forward", rows=16, vocab=131072, top=20, type="bf16", index="i64",
             entropy=True, masked=0.25),
        # scoring the language model's micro-batch
        dict(name="logprob_forward_batch", op="logprob", dir="forward", rows=700, vocab=32768, top=5, type="f32", index="i64",
             entropy=True, masked=0.0),
        # the same micro-batch's loss: an odd vocabulary, padded rows
        dict(name="logprob_backward_odd", op="logprob", dir="backward", rows=700, vocab=32771, top=0, type="f32", index="i32",
             entropy=True, masked=0.0),
        # a long batch in bf16
        dict(name="logprob_backward_large", op="logprob", dir="backward", rows=16384, vocab=65536, top=0, type="bf16", index="i64",
             entropy=False, masked=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    """What a drawn case is held to: bytes, and for the scan its states."""
    if case["op"] == "scan":
        return case["batch"] * case["steps"] * case["channels"] * case["states"] * (1 if case["dir"] == "forward" else 4)
    return work(case)["bytes"]


def draw(rng):
    op = rng.choice(["convolution", "scan", "logprob"])
    case = dict(op=op, dir=rng.choice(["forward", "backward"]), type=rng.choice(["f32", "bf16"]))
    if op == "logprob":
        case.update(rows=_log(rng, 1, 16384), vocab=_log(rng, 64, 131072), top=0, index=rng.choice(["i32", "i64"]),
                    entropy=rng.random() < 0.5, masked=rng.choice([0.0, 0.25, 0.9]))
        if case["dir"] == "forward" and rng.random() < 0.6:
            case["top"] = rng.randint(1, 32)
        shrink = ("rows",)
    else:
        case.update(batch=_log(rng, 1, 64), steps=_log(rng, 1, 65536), channels=_log(rng, 32, 4096), ragged=rng.random() < 0.3)
        shrink = ("batch", "steps")
        if op == "convolution":
            case.update(width=rng.randint(2, 6), silu=rng.random() < 0.6, bias=rng.random() < 0.6)
        else:
            case.update(states=rng.choice([16, 16, _log(rng, 1, 64)]), groups=rng.choice([1, 1, 2, 4]), gate=rng.random() < 0.6,
                        softplus=rng.random() < 0.7)
            case["channels"] = max(1, case["channels"] // case["groups"]) * case["groups"]
    most = max(_cost(c) for c in listed() if c["op"] == op)
    while _cost(case) > most:
        key = max(shrink, key=lambda k: case[k])
        case[key] = case[key] // 2 + 1
    return case


# ---- inputs ---------------------------------------------------------------------------------------------

def _gen(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    return gen


def _normal(gen, *shape, scale=1.0, dtype=torch.float32):
    return torch.randn(*shape, generator=gen, device=DEVICE).mul_(scale).to(dtype)


def _uniform(gen, *shape, lo, hi):
    return torch.empty(*shape, device=DEVICE).uniform_(lo, hi, generator=gen)


def _lengths(case, gen):
    if not case["ragged"]:
        return None
    n = (torch.rand(case["batch"], generator=gen, device=DEVICE) * (case["steps"] + 1)).to(torch.int32)
    n[-1] = case["steps"]
    return n


def _empty(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device=DEVICE)


def prepare(case, seed):
    gen, op, forward, kind = _gen(seed), case["op"], case["dir"] == "forward", TYPES[case["type"]]
    s = dict(case=case)
    if op == "logprob":
        rows, vocab = case["rows"], case["vocab"]
        # logits of a trained model: a level per row, most tokens far below the few likely ones; some tokens forbidden
        s["logits"] = (_normal(gen, rows, vocab, scale=2.5) + _normal(gen, rows, 1, scale=3.0)).to(kind)
        if case["masked"]:
            s["logits"].masked_fill_(torch.rand(vocab, generator=gen, device=DEVICE) < case["masked"], -math.inf)
            s["logits"][:, 0] = 0.0
        index = torch.int32 if case["index"] == "i32" else torch.int64
        ids = torch.randint(0, vocab, (rows,), generator=gen, device=DEVICE)
        ids.masked_fill_(torch.isinf(s["logits"].gather(1, ids[:, None])[:, 0]), 0)
        # rows without a token (padding)
        s["targets"] = ids.masked_fill_(torch.rand(rows, generator=gen, device=DEVICE) < 0.05, -100).to(index)
        if forward:
            s["logprob"], s["lse"] = _empty(rows), _empty(rows)
            s["entropy"] = _empty(rows) if case["entropy"] else None
            s["top_logprobs"] = _empty(rows, case["top"]) if case["top"] else None
            s["top_ids"] = _empty(rows, case["top"], dtype=index) if case["top"] else None
        else:
            parts = [_row_statistics(s["logits"][r:r + 256]) for r in range(0, rows, 256)]
            s["lse"], entropy = (torch.cat(p).float() for p in zip(*parts))
            s["grad_logprob"] = _normal(gen, rows, scale=1.0 / rows)
            s["entropy"] = entropy if case["entropy"] else None
            s["grad_entropy"] = _normal(gen, rows, scale=1e-2 / rows) if case["entropy"] else None
            s["grad_logits"] = _empty(rows, vocab, dtype=kind)
        return s
    shape = (case["batch"], case["steps"], case["channels"])
    batch, steps, channels = shape
    # one projection writes the layer's input and its gate side by side
    both = _normal(gen, batch, steps, 2 * channels, dtype=kind)
    s.update(x=both[..., :channels], lengths=_lengths(case, gen))
    if op == "convolution":
        k = case["width"]
        s.update(weight=_uniform(gen, channels, k, lo=-k ** -0.5, hi=k ** -0.5), state=_normal(gen, batch, k - 1, channels),
                 bias=_uniform(gen, channels, lo=-k ** -0.5, hi=k ** -0.5) if case["bias"] else None)
        s["state"] = s["state"].to(kind).float()
        if forward:
            s.update(out=_empty(*shape, dtype=kind), last=_empty(batch, k - 1, channels))
        else:
            s.update(grad_out=_normal(gen, *shape, scale=1e-2, dtype=kind), grad_last=_normal(gen, batch, k - 1, channels, scale=1e-2),
                     grad_x=_empty(*shape, dtype=kind), grad_weight=_empty(channels, k), grad_state=_empty(batch, k - 1, channels),
                     grad_bias=_empty(channels) if case["bias"] else None)
        return s
    n, groups = case["states"], case["groups"]
    # dt spread over [0.001, 0.1] by channel, decays of 1 to `states` by state, b and c two slices of one projection
    dt = torch.exp(_uniform(gen, channels, lo=math.log(1e-3), hi=math.log(1e-1)))
    if case["softplus"]:
        s.update(delta=_normal(gen, *shape, scale=0.5, dtype=kind), delta_bias=dt + torch.log(-torch.expm1(-dt)))
    else:
        s.update(delta=(dt * torch.exp(_normal(gen, *shape, scale=0.3))).to(kind), delta_bias=None)
    wide = _normal(gen, batch, steps, 32 + 2 * groups * n, dtype=kind)
    s.update(a=-torch.arange(1, n + 1, device=DEVICE) * torch.exp(_normal(gen, channels, n, scale=0.2)),
             b=wide[..., 32:32 + groups * n].unflatten(2, (groups, n)), c=wide[..., 32 + groups * n:].unflatten(2, (groups, n)),
             d=_normal(gen, channels), gate=both[..., channels:] if case["gate"] else None, h0=_normal(gen, batch, channels, n, scale=0.1))
    if forward:
        s.update(out=_empty(*shape, dtype=kind), h_last=_empty(batch, channels, n))
    else:
        s.update(grad_out=_normal(gen, *shape, scale=1e-2, dtype=kind), grad_last=_normal(gen, batch, channels, n, scale=1e-2),
                 grad_x=_empty(*shape, dtype=kind), grad_delta=_empty(*shape, dtype=kind), grad_a=_empty(channels, n),
                 grad_b=_empty(batch, steps, groups, n, dtype=kind), grad_c=_empty(batch, steps, groups, n, dtype=kind),
                 grad_d=_empty(channels), grad_gate=_empty(*shape, dtype=kind) if case["gate"] else None,
                 grad_delta_bias=_empty(channels) if case["softplus"] else None, grad_h0=_empty(batch, channels, n))
    return s


def _row_statistics(logits):
    """Log of the sum of exponentials and entropy of every row, in 64 bits."""
    x = logits.double()
    lse = torch.logsumexp(x, 1)
    lp = x - lse[:, None]
    return lse, -torch.where(lp > -math.inf, lp.exp() * lp, 0.0).sum(1)


# ---- the plain forms ------------------------------------------------------------------------------------

def _valid(steps, lengths):
    """[batch, steps]: the steps that belong to a sequence."""
    return torch.arange(steps, device=DEVICE)[None, :] < lengths[:, None]


def _sigmoid(v):
    return 1.0 / (1.0 + torch.exp(-v))


def _windows(s):
    """The inputs of all steps behind the state's, and per sequence the place of its last ones."""
    k, x = s["case"]["width"], s["x"].float()
    if s["lengths"] is not None:
        x = torch.where(_valid(x.shape[1], s["lengths"])[:, :, None], x, 0.0)
    xs = torch.cat([s["state"], x], 1)
    n = torch.full((x.shape[0],), x.shape[1], device=DEVICE) if s["lengths"] is None else s["lengths"].long()
    return xs, (n[:, None] + torch.arange(k - 1, device=DEVICE)[None, :])[:, :, None].expand(-1, -1, x.shape[2])


def _convolution(s):
    case, kind = s["case"], s["x"].dtype
    k, steps = case["width"], case["steps"]
    xs, ends = _windows(s)
    u = sum(s["weight"][:, j] * xs[:, j:j + steps] for j in range(k))
    if s["bias"] is not None:
        u = u + s["bias"]
    on = None if s["lengths"] is None else _valid(steps, s["lengths"])[:, :, None]
    if case["dir"] == "forward":
        out = u * _sigmoid(u) if case["silu"] else u
        if on is not None:
            out = torch.where(on, out, 0.0)
        return {"out": out.to(kind), "last": xs.gather(1, ends)}
    g = s["grad_out"].float()
    if case["silu"]:
        z = _sigmoid(u)
        g = g * (z * (1.0 + u * (1.0 - z)))
    if on is not None:
        g = torch.where(on, g, 0.0)
    total = torch.zeros_like(xs)
    for j in range(k):
        total[:, j:j + steps] += s["weight"][:, j] * g
    total.scatter_add_(1, ends, s["grad_last"])
    weight = torch.stack([(g * xs[:, j:j + steps]).sum((0, 1)) for j in range(k)], 1)
    inputs = total[:, k - 1:]
    if on is not None:
        inputs = torch.where(on, inputs, 0.0)
    return {"x": inputs.to(kind), "weight": weight, "bias": g.sum((0, 1)) if case["bias"] else None, "state": total[:, :k - 1]}


def _recur(a, u, first):
    """h_t = a_t h_{t-1} + u_t along dim 1 from `first`: blocks of about sqrt(steps) side by side, then what each starts from."""
    steps = a.shape[1]
    size = max(1, int(math.sqrt(steps)))
    pad = -steps % size
    if pad:
        a = torch.cat([a, torch.ones_like(a[:, :pad])], 1)
        u = torch.cat([u, torch.zeros_like(u[:, :pad])], 1)
    blocks = (a.shape[1]) // size
    a, u = (t.unflatten(1, (blocks, size)) for t in (a, u))
    h, p = torch.empty_like(u), torch.empty_like(a)
    h[:, :, 0], p[:, :, 0] = u[:, :, 0], a[:, :, 0]
    for i in range(1, size):
        h[:, :, i] = torch.addcmul(u[:, :, i], a[:, :, i], h[:, :, i - 1])
        p[:, :, i] = a[:, :, i] * p[:, :, i - 1]
    starts = torch.empty_like(h[:, :, 0])
    for i in range(blocks):
        starts[:, i] = first
        first = torch.addcmul(h[:, i, -1], p[:, i, -1], first)
    return torch.addcmul(h, p, starts[:, :, None]).flatten(1, 2)[:, :steps]


def _scan(s):
    case, kind = s["case"], s["x"].dtype
    groups = case["groups"]
    per = case["channels"] // groups

    def spread(t):           # [batch, steps, groups, states] to every channel of a group
        return t.float().repeat_interleave(per, 2) if groups > 1 else t.float()

    x, raw = s["x"].float(), s["delta"].float()
    if s["delta_bias"] is not None:
        raw = raw + s["delta_bias"]
    dt = raw.clamp(min=0.0) + torch.log1p(torch.exp(-raw.abs())) if case["softplus"] else raw
    on = None if s["lengths"] is None else _valid(case["steps"], s["lengths"])[:, :, None]
    if on is not None:
        dt = torch.where(on, dt, 0.0)
    b, c = spread(s["b"]), spread(s["c"])
    a = torch.exp(dt[..., None] * s["a"])
    h = _recur(a, (dt * x)[..., None] * b, s["h0"])
    y = (c * h).sum(3) + s["d"] * x
    if case["gate"]:
        gate = s["gate"].float()
        z = _sigmoid(gate)
    if case["dir"] == "forward":
        out = y * gate * z if case["gate"] else y
        if on is not None:
            out = torch.where(on, out, 0.0)
        return {"out": out.to(kind), "h_last": h[:, -1].clone()}
    grad_out = s["grad_out"].float()
    if on is not None:
        grad_out = torch.where(on, grad_out, 0.0)
    dy = grad_out * gate * z if case["gate"] else grad_out
    result = {"gate": (grad_out * y * z * (1.0 + gate * (1.0 - z))).to(kind) if case["gate"] else None, "d": (dy * x).sum((0, 1))}

    def gather(t):           # sums over the channels of a group
        return t.unflatten(2, (groups, per)).sum(3).to(kind)

    result["c"] = gather(dy[..., None] * h)
    h = torch.cat([s["h0"][:, None], h[:, :-1]], 1)
    after = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], 1)
    total = _recur(after.flip(1), (c * dy[..., None]).flip(1), s["grad_last"]).flip(1)
    result["b"] = gather(total * (dt * x)[..., None])
    along = (total * b).sum(3)
    inputs = dt * along + s["d"] * dy
    h *= a
    h *= total
    step = (h * s["a"]).sum(3) + along * x
    if case["softplus"]:
        step = step * _sigmoid(raw)
    if on is not None:
        step = torch.where(on, step, 0.0)
    result.update(x=inputs.to(kind), delta=step.to(kind), a=(h * dt[..., None]).sum((0, 1)), h0=a[:, 0] * total[:, 0],
                  delta_bias=step.sum((0, 1)) if case["softplus"] else None)
    return result


def _logprob(s):
    case = s["case"]
    x, ids = s["logits"].float(), s["targets"].long()
    named = (ids >= 0) & (ids < case["vocab"])
    place = torch.where(named, ids, 0)[:, None]
    if case["dir"] == "backward":
        lp = x - s["lse"][:, None]
        p = torch.exp(lp)
        grad = -p * torch.where(named, s["grad_logprob"], 0.0)[:, None]
        grad.scatter_add_(1, place, torch.where(named, s["grad_logprob"], 0.0)[:, None])
        if case["entropy"]:
            grad -= torch.where(p > 0, p * (lp + s["entropy"][:, None]), 0.0) * s["grad_entropy"][:, None]
        return grad.to(s["logits"].dtype)
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    result = {"logprob": torch.where(named, (x.gather(1, place) - lse)[:, 0], 0.0), "lse": lse[:, 0], "entropy": None,
              "top_logprobs": None, "top_ids": None}
    if case["entropy"]:
        result["entropy"] = (torch.log(total) - torch.where(e > 0, e * (x - top), 0.0).sum(1, keepdim=True) / total)[:, 0]
    if case["top"]:
        values, order = torch.sort(x, dim=1, descending=True, stable=True)
        result["top_logprobs"] = values[:, :case["top"]] - lse
        result["top_ids"] = order[:, :case["top"]].to(s["targets"].dtype)
    return result


# ---- a pass ---------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    op, forward = case["op"], case["dir"] == "forward"
    if not own:
        return {"convolution": _convolution, "scan": _scan, "logprob": _logprob}[op](s)
    from paper_2010_16248_amd import binding as B
    if op == "convolution":
        if forward:
            B.convolution_forward(s["x"], s["weight"], s["out"], bias=s["bias"], state=s["state"], last=s["last"], lengths=s["lengths"],
                                  silu=case["silu"])
            return {"out": s["out"], "last": s["last"]}
        B.convolution_backward(s["x"], s["weight"], s["grad_out"], s["grad_x"], s["grad_weight"], bias=s["bias"],
                               grad_bias=s["grad_bias"], state=s["state"], grad_last=s["grad_last"], grad_state=s["grad_state"],
                               lengths=s["lengths"], silu=case["silu"])
        return {"x": s["grad_x"], "weight": s["grad_weight"], "bias": s["grad_bias"], "state": s["grad_state"]}
    if op == "scan":
        if forward:
            B.scan_forward(s["x"], s["delta"], s["a"], s["b"], s["c"], s["out"], d=s["d"], gate=s["gate"], delta_bias=s["delta_bias"],
                           softplus=case["softplus"], h0=s["h0"], h_last=s["h_last"], lengths=s["lengths"])
            return {"out": s["out"], "h_last": s["h_last"]}
        B.scan_backward(s["x"], s["delta"], s["a"], s["b"], s["c"], s["grad_out"], s["grad_x"], s["grad_delta"], s["grad_a"],
                        s["grad_b"], s["grad_c"], d=s["d"], grad_d=s["grad_d"], gate=s["gate"], grad_gate=s["grad_gate"],
                        delta_bias=s["delta_bias"], grad_delta_bias=s["grad_delta_bias"], softplus=case["softplus"], h0=s["h0"],
                        grad_last=s["grad_last"], grad_h0=s["grad_h0"], lengths=s["lengths"])
        return {"gate": s["grad_gate"], "d": s["grad_d"], "c": s["grad_c"], "b": s["grad_b"], "x": s["grad_x"], "delta": s["grad_delta"],
                "a": s["grad_a"], "h0": s["grad_h0"], "delta_bias": s["grad_delta_bias"]}
    if forward:
        B.logprob_forward(s["logits"], s["targets"], s["logprob"], lse=s["lse"], entropy=s["entropy"], top_logprobs=s["top_logprobs"],
                          top_ids=s["top_ids"])
        return {key: s[key] for key in ("logprob", "lse", "entropy", "top_logprobs", "top_ids")}
    B.logprob_backward(s["logits"], s["targets"], s["lse"], s["grad_logprob"], s["grad_logits"], entropy=s["entropy"],
                       grad_entropy=s["grad_entropy"])
    return s["grad_logits"]


# ---- what a pass cannot do without ----------------------------------------------------------------------

def work(case):
    op, e, forward = case["op"], BYTES[case["type"]], case["dir"] == "forward"
    if op == "logprob":
        r, v = case["rows"], case["vocab"]
        if forward:
            return {"bytes": r * v * e + r * (12 + BYTES[case["index"]] + case["top"] * (4 + BYTES[case["index"]])),
                    "flops": r * v * (6 if case["entropy"] else 4)}
        return {"bytes": 2 * r * v * e + r * (8 + BYTES[case["index"]]), "flops": r * v * (8 if case["entropy"] else 4)}
    ends = case["batch"] * case["channels"]
    tokens = ends * case["steps"]
    if op == "convolution":
        k = case["width"]
        if forward:
            return {"bytes": 2 * tokens * e + 8 * ends * (k - 1) + 4 * case["channels"] * (k + 1), "flops": (2 * k + 4) * tokens}
        return {"bytes": 3 * tokens * e + 12 * ends * (k - 1) + 8 * case["channels"] * (k + 1), "flops": (6 * k + 12) * tokens}
    n, shared = case["states"], case["batch"] * case["steps"] * case["groups"] * case["states"]
    params = case["channels"] * (n + 2)
    if forward:
        return {"bytes": (4 if case["gate"] else 3) * tokens * e + 2 * shared * e + 8 * ends * n + 4 * params, "flops": 7 * n * tokens}
    return {"bytes": (7 if case["gate"] else 5) * tokens * e + 4 * shared * e + 12 * ends * n + 8 * params, "flops": 18 * n * tokens}


# ---- the definitions in 64 bits -------------------------------------------------------------------------

def _wide(s, *names):
    return [None if s[k] is None else s[k].double() for k in names]


def exact(case, seed):
    s = prepare(case, seed)
    forward, steps = case["dir"] == "forward", case["steps"] if "steps" in case else 0
    if case["op"] == "logprob":
        return _logprob_exact(case, s, forward)
    if "lengths" in s and s["lengths"] is not None:
        lengths = s["lengths"].tolist()
    else:
        lengths = [steps] * case["batch"]
    return (_convolution_exact if case["op"] == "convolution" else _scan_exact)(case, s, forward, lengths)


def _logprob_exact(case, s, forward):
    # blocks of rows
    vocab, parts = case["vocab"], []
    for r in range(0, case["rows"], 256):
        rows = slice(r, min(r + 256, case["rows"]))
        x, ids = s["logits"][rows].double(), s["targets"][rows].long()
        hit = (torch.arange(vocab, device=DEVICE)[None, :] == ids[:, None])
        named = hit.any(1)
        if forward:
            lp = torch.log_softmax(x, 1)
            plogp = torch.where(lp > -math.inf, lp.exp() * lp, 0.0)
            part = {"logprob": torch.where(hit, lp, 0.0).sum(1), "lse": torch.logsumexp(x, 1)}
            if case["entropy"]:
                part["entropy"] = -plogp.sum(1)
            if case["top"]:
                # the k-th row of values is the largest of what is left, at its lowest index
                left, seats, best = x.clone(), [], []
                for _ in range(case["top"]):
                    top = left.nan_to_num(nan=-math.inf, neginf=-math.inf).amax(1)
                    at = torch.where(left == top[:, None], torch.arange(vocab, device=DEVICE)[None, :], vocab).amin(1)
                    seats.append(at)
                    best.append(lp.gather(1, at[:, None])[:, 0])
                    left.scatter_(1, at[:, None], math.nan)
                part["top_ids"], part["top_logprobs"] = torch.stack(seats, 1), torch.stack(best, 1)
        else:
            lp = x - s["lse"][rows].double()[:, None]
            grad = torch.where(named, s["grad_logprob"][rows].double(), 0.0)[:, None] * (hit.double() - lp.exp())
            if case["entropy"]:
                inner = torch.where(lp > -math.inf, lp.exp() * (lp + s["entropy"][rows].double()[:, None]), 0.0)
                grad = grad - s["grad_entropy"][rows].double()[:, None] * inner
            part = {"grad": grad}
        parts.append(part)
    whole = {key: torch.cat([p[key] for p in parts]) for key in parts[0]}
    if not forward:
        return whole["grad"]
    ids = whole.get("top_ids")
    return {"logprob": whole["logprob"], "lse": whole["lse"], "entropy": whole.get("entropy"), "top_logprobs": whole.get("top_logprobs"),
            "top_ids": None if ids is None else ids.to(s["targets"].dtype)}


def _convolution_exact(case, s, forward, lengths):
    # one sequence after the other
    k, steps, channels = case["width"], case["steps"], case["channels"]
    weight, bias = _wide(s, "weight", "bias")
    zero = torch.zeros(channels, dtype=torch.float64, device=DEVICE)
    outs, ends = [], []
    grad_w, grad_b = torch.zeros(channels, k, dtype=torch.float64, device=DEVICE), zero.clone()
    for i, n in enumerate(lengths):
        xs = torch.cat([s["state"][i].double(), s["x"][i, :n].double()])
        u = torch.cat([xs, zero[None]]).unfold(0, k, 1)[:n]          # [n, channels, k]
        u = (u * weight).sum(2) + (0.0 if bias is None else bias)
        if forward:
            y = torch.nn.functional.silu(u) if case["silu"] else u
            outs.append(torch.cat([y, zero.expand(steps - n, -1)]))
            ends.append(xs[n:])
            continue
        g = s["grad_out"][i, :n].double()
        if case["silu"]:
            sig = torch.sigmoid(u)
            g = g * sig + g * u * sig * torch.sigmoid(-u)
        total = torch.zeros_like(xs)
        total[n:] = s["grad_last"][i].double()
        for j in range(k):
            total[j:j + n] += g * weight[:, j]
            grad_w[:, j] += (g * xs[j:j + n]).sum(0)
        grad_b += g.sum(0)
        outs.append(torch.cat([total[k - 1:], zero.expand(steps - n, -1)]))
        ends.append(total[:k - 1])
    if forward:
        return {"out": torch.stack(outs), "last": torch.stack(ends)}
    return {"x": torch.stack(outs), "weight": grad_w, "bias": grad_b if case["bias"] else None, "state": torch.stack(ends)}


def _scan_exact(case, s, forward, lengths):
    # one sequence after the other, one step after the other
    steps, channels, n = case["steps"], case["channels"], case["states"]
    if sum(lengths) > 400000:
        return None
    owner = torch.arange(channels, device=DEVICE) // (channels // case["groups"])
    decay, skip, bias = _wide(s, "a", "d", "delta_bias")
    results = []
    for i, length in enumerate(lengths):
        x, raw, gate = (None if s[k] is None else s[k][i, :length].double() for k in ("x", "delta", "gate"))
        b, c = (s[k][i, :length].double() for k in ("b", "c"))
        raw = raw if bias is None else raw + bias
        dt = torch.logaddexp(raw, torch.zeros_like(raw)) if case["softplus"] else raw
        a = torch.exp(dt[:, :, None] * decay)
        states = torch.empty(length + 1, channels, n, dtype=torch.float64, device=DEVICE)
        states[0] = s["h0"][i].double()
        pushed = (dt * x)[:, :, None] * b[:, owner]
        for t in range(length):
            torch.addcmul(pushed[t], a[t], states[t], out=states[t + 1])
        del pushed
        y = skip * x
        for t in range(0, length, 1024):
            y[t:t + 1024] += (c[t:t + 1024][:, owner] * states[t + 1:t + 1025]).sum(2)
        rest = steps - length

        def filled(t):
            return torch.cat([t, t.new_zeros(rest, *t.shape[1:])])

        if forward:
            out = y * torch.nn.functional.silu(gate) if case["gate"] else y
            results.append({"out": filled(out), "h_last": states[-1].clone()})
            continue
        grad = s["grad_out"][i, :length].double()
        r = {}
        if case["gate"]:
            sig = torch.sigmoid(gate)
            r["gate"] = filled(grad * y * (sig + gate * sig * torch.sigmoid(-gate)))
            grad = grad * gate * sig
        r["d"] = (grad * x).sum(0)
        total = s["grad_last"][i].double()
        one_of = torch.nn.functional.one_hot(owner, case["groups"]).double()          # [channels, groups]
        rows = {k: [] for k in ("b", "c", "x", "delta")}
        r["a"] = torch.zeros(channels, n, dtype=torch.float64, device=DEVICE)
        block = 256
        for end in range(length, 0, -block):
            lo = max(0, end - block)
            of = slice(lo, end)
            g = c[of][:, owner] * grad[of][:, :, None]
            for t in range(end - lo - 1, -1, -1):
                g[t] += total
                total = a[lo + t] * g[t]
            carried = g * a[of] * states[lo:end]
            bs = b[of][:, owner]
            rows["b"].append(torch.einsum("tcn,tc,cg->tgn", g, dt[of] * x[of], one_of))
            rows["c"].append(torch.einsum("tcn,tc,cg->tgn", states[lo + 1:end + 1], grad[of], one_of))
            rows["x"].append((g * bs).sum(2) * dt[of] + skip * grad[of])
            rows["delta"].append((carried * decay).sum(2) + (g * bs).sum(2) * x[of])
            r["a"] += (carried * dt[of][:, :, None]).sum(0)
        shape = {"b": (0, case["groups"], n), "c": (0, case["groups"], n), "x": (0, channels), "delta": (0, channels)}
        for k, parts in rows.items():
            r[k] = torch.cat(parts[::-1]) if parts else torch.zeros(shape[k], dtype=torch.float64, device=DEVICE)
        if case["softplus"]:
            r["delta"] = r["delta"] * torch.sigmoid(raw)
            r["delta_bias"] = r["delta"].sum(0)
        for k in ("b", "c", "x", "delta"):
            r[k] = filled(r[k])
        r["h0"] = total
        results.append(r)
    summed = ("a", "d", "delta_bias")
    whole = {k: sum(r[k] for r in results) if k in summed else torch.stack([r[k] for r in results]) for k in results[0]}
    if forward:
        return whole
    return {k: whole.get(k) for k in ("gate", "d", "c", "b", "x", "delta", "a", "h0", "delta_bias")}
