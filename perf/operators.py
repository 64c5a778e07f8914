"""Operators around the compression path of a language model's training step, as cases that can be timed and compared.

One pass is one call of one operator:

  embedding   forward: rows of the table by token, scaled; backward: the table's dense fp32 gradient from the tokens' gradients
  layernorm   forward: normalised rows with their means and reciprocal deviations; backward: gradients of rows, weight and bias
  recurrence  h_t = sigmoid(f_t) h_{t-1} + sigmoid(-f_t) x_t along a sequence; forward with the last state (one step: its serving
              form); backward: gradients of gates, inputs and the first state
  adamw       one step over all tensors of a model in a flat buffer, moments in 32 or 8 bits

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
EPS_NORM = 1e-5
LR, BETA1, BETA2, EPS_ADAM, DECAY = 1e-3, 0.9, 0.95, 1e-8, 0.1
FIRST_STEP = 1000       # optimizer steps behind the state that a pass starts from
BLOCK = 256             # elements that share a scale in 8-bit moments
TOP = 448.0             # largest e4m3 value
LEAST = 2.0 ** -9       # smallest positive e4m3 value
TINY = 2.0 ** -100      # blocks whose largest value is below are held as zeros


def listed():
    return [
        # the tokens of one micro-batch of the language model, 20 sequences of 35: launch and latency
        dict(name="embedding_forward_batch", op="embedding", dir="forward", vocab=32768, dim=672, tokens=700, type="f32",
             index="i64", accumulate=False),
        # the row-sparse gradient that the compressors take: 5 % of the rows touched, the others written as zeros
        dict(name="embedding_backward_lstm", op="embedding", dir="backward", vocab=32768, dim=672, tokens=2800, type="f32",
             index="i64", accumulate=False),
        # long sequences in bf16, odd vocabulary, table shared with a decoder whose gradient is there already
        dict(name="embedding_backward_tied", op="embedding", dir="backward", vocab=65537, dim=2048, tokens=131072,
             type="bf16", index="i32", accumulate=True),
        # the rows of one micro-batch at the language model's width
        dict(name="layernorm_forward_batch", op="layernorm", dir="forward", rows=700, dim=672, type="f32"),
        # odd sizes: rows that start off 16-byte boundaries
        dict(name="layernorm_backward_odd", op="layernorm", dir="backward", rows=5003, dim=1001, type="f32"),
        # a large batch in bf16
        dict(name="layernorm_backward_large", op="layernorm", dir="backward", rows=65536, dim=2048, type="bf16"),
        # serving: one token for each of 64 sequences
        dict(name="recurrence_forward_token", op="recurrence", dir="forward", batch=64, steps=1, channels=672, type="f32",
             ragged=False),
        # one long document: 672 channels, all parallel work has to come from the sequence
        dict(name="recurrence_forward_long", op="recurrence", dir="forward", batch=1, steps=65536, channels=672, type="f32",
             ragged=False),
        # a padded training batch in bf16 with sequences of different lengths
        dict(name="recurrence_backward_large", op="recurrence", dir="backward", batch=8, steps=4096, channels=2048,
             type="bf16", ragged=True),
        # 62 tensors, most of them small vectors
        dict(name="adamw8_resnet18", op="adamw", set="resnet18", bits=8, type="f32", copy=False, clip=False),
        # the language model's six tensors, 51 M parameters, moments in 32 bits
        dict(name="adamw32_lstm", op="adamw", set="lstm", bits=32, type="f32", copy=False, clip=True),
        # the same with moments in 8 bits, gradients and a copy of the weights in bf16
        dict(name="adamw8_lstm_bf16", op="adamw", set="lstm", bits=8, type="bf16", copy=True, clip=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embedding", "layernorm", "recurrence", "adamw"])
    case = dict(op=op, type=rng.choice(["f32", "bf16"]))
    if op == "adamw":
        case.update(set=rng.choice(["resnet18", "vgg19", "lstm", "ragged", "ragged", "ragged"]), bits=rng.choice([8, 32]),
                    copy=rng.random() < 0.5, clip=rng.random() < 0.5)
        if case["set"] == "ragged":
            case.update(tensors=_log(rng, 1, 200), most=_log(rng, 500, 2000000), shape_seed=rng.randint(1, 10 ** 6))
        large = [c for c in listed() if c["op"] == op]
        while work(case)["bytes"] > max(work(c)["bytes"] for c in large):
            if case["set"] == "ragged":
                case["tensors"] = (case["tensors"] + 1) // 2
            else:
                case["bits"], case["copy"] = 8, False
        return case
    case["dir"] = rng.choice(["forward", "backward"])
    if op == "embedding":
        case.update(vocab=_log(rng, 64, 131072), dim=_log(rng, 32, 4096), tokens=_log(rng, 1, 131072),
                    index=rng.choice(["i32", "i64"]), accumulate=case["dir"] == "backward" and rng.random() < 0.3)
        shrink = ("tokens", "vocab")
    elif op == "layernorm":
        case.update(rows=_log(rng, 1, 131072), dim=_log(rng, 16, 16384))
        shrink = ("rows",)
    else:
        case.update(batch=_log(rng, 1, 64), steps=_log(rng, 1, 65536), channels=_log(rng, 32, 4096),
                    ragged=rng.random() < 0.3)
        shrink = ("batch", "steps")
    same = [work(c)["bytes"] for c in listed() if c["op"] == op]
    while work(case)["bytes"] > max(same):
        key = max(shrink, key=lambda k: case[k])
        case[key] = case[key] // 2 + 1
    return case


# ---- the tensors of a model ----------------------------------------------------------------------------

def _sizes(case):
    """[(elements, decayed)] of the tensors: matrices are decayed, vectors are not."""
    kind, s = case["set"], []

    def conv(o, i, k, bias=False):
        s.append((o * i * k * k, True))
        s.extend([(o, False)] * (3 if bias else 2))

    if kind == "resnet18":
        conv(64, 3, 3)
        inp = 64
        for width in (64, 128, 256, 512):
            for block in range(2):
                conv(width, inp, 3)
                conv(width, width, 3)
                if block == 0 and inp != width:
                    conv(width, inp, 1)
                inp = width
        s += [(10 * 512, True), (10, False)]
    elif kind == "vgg19":
        inp = 3
        for width, reps in ((64, 2), (128, 2), (256, 4), (512, 4), (512, 4)):
            for _ in range(reps):
                conv(width, inp, 3, True)
                inp = width
        s += [(512 * 512, True), (512, False), (512 * 512, True), (512, False), (10 * 512, True), (10, False)]
    elif kind == "lstm":
        s += [(32768 * 672, True)] + [(2688 * 672, True)] * 4 + [(32768 * 672, True)]
    else:
        import random
        r = random.Random(case["shape_seed"])
        for _ in range(case["tensors"]):
            s.append((r.randint(1, case["most"]) if r.random() < 0.6 else r.randint(1, min(4096, case["most"])), r.random() < 0.6))
    return s


# ---- inputs ---------------------------------------------------------------------------------------------

def _gen(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    return gen


def _normal(gen, *shape, scale=1.0, dtype=torch.float32):
    return torch.randn(*shape, generator=gen, device=DEVICE).mul_(scale).to(dtype)


def _lengths(case, gen):
    if not case["ragged"]:
        return None
    n = (torch.rand(case["batch"], generator=gen, device=DEVICE) * (case["steps"] + 1)).to(torch.int32)
    n[-1] = case["steps"]
    return n


def _valid(steps, lengths):
    """[batch, steps, 1]: the steps that belong to a sequence."""
    return (torch.arange(steps, device=DEVICE)[None, :] < lengths[:, None])[:, :, None]


def _inputs(case, seed):
    gen, op = _gen(seed), case["op"]
    kind = TYPES[case["type"]]
    if op == "embedding":
        # tokens by rank: the frequency of rank r falls as 1 / r
        u = torch.rand(case["tokens"], generator=gen, device=DEVICE, dtype=torch.float64)
        ids = (torch.exp(u * math.log(case["vocab"] + 1.0)) - 1.0).to(torch.int64).clamp_(0, case["vocab"] - 1)
        s = dict(ids=ids.to(torch.int32 if case["index"] == "i32" else torch.int64), scale=math.sqrt(case["dim"]))
        if case["dir"] == "forward":
            s["table"] = _normal(gen, case["vocab"], case["dim"], scale=case["dim"] ** -0.5, dtype=kind)
            s["out"] = torch.empty(case["tokens"], case["dim"], dtype=kind, device=DEVICE)
        else:
            s["grad_out"] = _normal(gen, case["tokens"], case["dim"], scale=1e-3, dtype=kind)
            s["grad_table"] = _normal(gen, case["vocab"], case["dim"], scale=1e-3)
        return s
    if op == "layernorm":
        rows, dim = case["rows"], case["dim"]
        s = dict(x=(_normal(gen, rows, dim) * _normal(gen, rows, 1).exp_() + _normal(gen, rows, 1)).to(kind),
                 weight=1.0 + _normal(gen, dim, scale=0.1), bias=_normal(gen, dim, scale=0.1),
                 mean=torch.empty(rows, device=DEVICE), rstd=torch.empty(rows, device=DEVICE))
        if case["dir"] == "forward":
            s["y"] = torch.empty(rows, dim, dtype=kind, device=DEVICE)
        else:
            x = s["x"].double()
            s["mean"].copy_(x.mean(1))
            s["rstd"].copy_((x.var(1, unbiased=False) + EPS_NORM).rsqrt())
            s["grad_y"] = _normal(gen, rows, dim, scale=1e-2, dtype=kind)
            s["grad_x"] = torch.empty(rows, dim, dtype=kind, device=DEVICE)
            s["grad_weight"], s["grad_bias"] = torch.empty(dim, device=DEVICE), torch.empty(dim, device=DEVICE)
        return s
    if op == "recurrence":
        shape = (case["batch"], case["steps"], case["channels"])
        # every channel remembers over a time of its own; a document's first token shuts the gate
        gate = _normal(gen, *shape) + torch.empty(shape[2], device=DEVICE).uniform_(-1.0, 6.0, generator=gen)
        gate.masked_fill_(torch.rand(*shape[:2], 1, generator=gen, device=DEVICE) < 1 / 500, -math.inf)
        s = dict(gate=gate.to(kind), input=_normal(gen, *shape, dtype=kind), h0=_normal(gen, shape[0], shape[2]),
                 lengths=_lengths(case, gen))
        if case["dir"] == "forward":
            s["out"] = torch.empty(shape, dtype=kind, device=DEVICE)
            s["h_last"] = torch.empty(shape[0], shape[2], device=DEVICE)
        else:
            s["out"] = _recurrence(s["gate"], s["input"], s["h0"], s["lengths"])[0]
            s["grad_out"] = _normal(gen, *shape, scale=1e-2, dtype=kind)
            s["grad_last"] = _normal(gen, shape[0], shape[2], scale=1e-2)
            s["grad_gate"], s["grad_input"] = (torch.empty(shape, dtype=kind, device=DEVICE) for _ in range(2))
            s["grad_h0"] = torch.empty(shape[0], shape[2], device=DEVICE)
        return s
    sizes = _sizes(case)
    n = sum(k for k, _ in sizes)
    # every tensor's gradients at a scale of their own
    level = torch.exp(torch.empty(len(sizes), device=DEVICE).uniform_(math.log(1e-4), math.log(1e-2), generator=gen))
    level = _per_element(level, torch.tensor([k for k, _ in sizes], device=DEVICE), n)
    s = dict(weights=_normal(gen, n, scale=0.05), grads=(_normal(gen, n) * level).to(kind), step=FIRST_STEP,
             copy=torch.empty(n, dtype=torch.bfloat16, device=DEVICE) if case["copy"] else None,
             clip=torch.full((1,), 0.7, device=DEVICE) if case["clip"] else None)
    m = _normal(gen, n, scale=0.2) * level
    v = (0.25 + torch.rand(n, generator=gen, device=DEVICE)) * level.square()
    if case["bits"] == 32:
        s["state"] = (m, v, None, None)
    else:
        padded, place = _padding(sizes)
        both = torch.zeros(2, padded, device=DEVICE)
        both[0, place], both[1, place] = m, v.sqrt()
        (mc, ms), (rc, rs) = _encode(both[0].view(-1, BLOCK), False), _encode(both[1].view(-1, BLOCK), True)
        s["state"] = (mc.view(-1), rc.view(-1), ms, rs)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "adamw":
        s["sizes"] = _sizes(case)
        counts = [k for k, _ in s["sizes"]]
        s["decay"] = [DECAY if d else 0.0 for _, d in s["sizes"]]
        s["tensors"], s["tensor_grads"] = s["weights"].split(counts), s["grads"].split(counts)
        s["tensor_copies"] = None if s["copy"] is None else s["copy"].split(counts)
    return s


# ---- the plain forms ------------------------------------------------------------------------------------

def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along dim 1 from h = 0, by doubling: after k rounds an element holds 2^k steps."""
    b, reach = b.clone(), 1
    while reach < a.shape[1]:
        b = torch.cat([b[:, :reach], b[:, reach:] + a[:, reach:] * b[:, :-reach]], 1)
        a = torch.cat([a[:, :reach], a[:, reach:] * a[:, :-reach]], 1)
        reach *= 2
    return b


def _gates(gate):
    """sigmoid(f) and sigmoid(-f), neither by a difference from one."""
    e = torch.exp(-gate.abs())
    big = 1.0 / (1.0 + e)
    small = e * big
    return torch.where(gate >= 0, big, small), torch.where(gate >= 0, small, big)


def _recurrence(gate, x, h0, lengths):
    kind = gate.dtype
    a, z = _gates(gate.float())
    b = z * x.float()
    if lengths is not None:
        valid = _valid(gate.shape[1], lengths)
        a, b = torch.where(valid, a, 1.0), torch.where(valid, b, 0.0)
    b[:, 0] += a[:, 0] * h0
    h = _scan(a, b)
    last = h[:, -1].clone()
    return (h if lengths is None else torch.where(valid, h, 0.0)).to(kind), last


def _recurrence_gradients(s):
    kind = s["gate"].dtype
    a, z = _gates(s["gate"].float())
    g = s["grad_out"].float()
    if s["lengths"] is not None:
        valid = _valid(a.shape[1], s["lengths"])
        a, z, g = torch.where(valid, a, 1.0), torch.where(valid, z, 0.0), torch.where(valid, g, 0.0)
    g[:, -1] += s["grad_last"]
    after = torch.cat([a[:, 1:], a[:, :1]], 1)
    total = _scan(after.flip(1), g.flip(1)).flip(1)
    before = torch.cat([s["h0"][:, None], s["out"].float()[:, :-1]], 1)
    return {"gate": (total * (before - s["input"].float()) * a * z).to(kind), "input": (z * total).to(kind),
            "h0": a[:, 0] * total[:, 0]}


def _per_element(values, counts, n):
    """values[i] for each of the counts[i] elements of tensor i."""
    ends = counts.cumsum(0)
    return values[torch.searchsorted(ends, torch.arange(n, device=DEVICE), right=True)]


def _padding(sizes):
    """Elements of a state whose tensors start on whole blocks, and the place of every weight in it."""
    counts = torch.tensor([k for k, _ in sizes], device=DEVICE)
    whole = (counts + BLOCK - 1) // BLOCK * BLOCK
    gap = (whole.cumsum(0) - whole) - (counts.cumsum(0) - counts)
    place = _per_element(gap, counts, sum(k for k, _ in sizes))
    place += torch.arange(len(place), device=DEVICE)
    return sum((k + BLOCK - 1) // BLOCK * BLOCK for k, _ in sizes), place


def _encode(x, root):
    """Blocks of values as e4m3 codes of x * (448 / largest) and the scale largest / 448; a positive root keeps a positive code."""
    top = x.abs().amax(1)
    held = ~(top < TINY)
    up = torch.where(held, torch.full_like(top, TOP) / top, 0.0)
    y = x * up[:, None]
    if root:
        y = torch.where((x > 0) & held[:, None], y.clamp(min=LEAST), y)
    return y.float().to(torch.float8_e4m3fn), torch.where(held, top * (1.0 / TOP), 0.0)


def _adamw(s, kind):
    """Moments, weights and, with 8 bits, codes after a step in the floating type `kind`; nothing is written."""
    sizes, (m, v, m_scale, v_scale) = s["sizes"], s["state"]
    counts = torch.tensor([k for k, _ in sizes], device=DEVICE)
    g, w = s["grads"].to(kind), s["weights"].to(kind)
    if s["clip"] is not None:
        g = g * s["clip"].to(kind)
    if m_scale is not None:
        padded, place = _padding(sizes)
        g = torch.zeros(padded, dtype=kind, device=DEVICE).scatter_(0, place, g)
        m = (m.to(kind).view(-1, BLOCK) * m_scale.to(kind)[:, None]).view(-1)
        v = (v.to(kind).view(-1, BLOCK) * v_scale.to(kind)[:, None]).view(-1)
        v = v * v
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + ((1.0 - BETA2) * g) * g
    root = torch.sqrt(v)
    move = (LR / (1.0 - BETA1 ** s["step"])) * m / (root * (1.0 - BETA2 ** s["step"]) ** -0.5 + EPS_ADAM)
    if m_scale is not None:
        move = move[place]
    decay = torch.tensor([1.0 - LR * d for d in s["decay"]], dtype=kind, device=DEVICE)
    w = w * _per_element(decay, counts, w.numel()) - move
    if m_scale is None:
        return w, (m, v, None, None)
    (mc, ms), (rc, rs) = _encode(m.view(-1, BLOCK), False), _encode(root.view(-1, BLOCK), True)
    return w, (mc.view(-1), rc.view(-1), ms, rs)


def _results(weights, copy, state):
    return {"weights": weights, "copy": copy, "m": state[0], "v": state[1], "m_scale": state[2], "v_scale": state[3]}


def _plain(s):
    case = s["case"]
    op, kind, forward = case["op"], TYPES[case["type"]], case.get("dir") == "forward"
    if op == "embedding":
        if forward:
            return (s["table"][s["ids"]].float() * s["scale"]).to(kind)
        if not case["accumulate"]:
            s["grad_table"].zero_()
        return s["grad_table"].index_add_(0, s["ids"], s["grad_out"].float() * s["scale"])
    if op == "layernorm":
        x = s["x"].float()
        if forward:
            mean = x.mean(1)
            d = x - mean[:, None]
            rstd = 1.0 / torch.sqrt((d * d).mean(1) + EPS_NORM)
            return {"y": (d * rstd[:, None] * s["weight"] + s["bias"]).to(kind), "mean": mean, "rstd": rstd}
        dy = s["grad_y"].float()
        xh = (x - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * s["weight"]
        gx = g * xh
        dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xh * gx.mean(1, keepdim=True))
        return {"x": dx.to(kind), "weight": (dy * xh).sum(0), "bias": dy.sum(0)}
    if op == "recurrence":
        if forward:
            out, last = _recurrence(s["gate"], s["input"], s["h0"], s["lengths"])
            return {"out": out, "last": last}
        return _recurrence_gradients(s)
    s["step"] += 1
    w, state = _adamw(s, torch.float32)
    s["weights"].copy_(w)
    s["state"] = state
    if s["copy"] is not None:
        s["copy"].copy_(w)
    return _results(s["weights"], s["copy"], state)


# ---- a pass ---------------------------------------------------------------------------------------------

def run(s):
    if not own:
        return _plain(s)
    from paper_2010_16248_amd import binding as B
    op, forward = s["case"]["op"], s["case"].get("dir") == "forward"
    if op == "embedding":
        if forward:
            B.embedding_forward(s["ids"], s["table"], s["out"], s["scale"])
            return s["out"]
        B.embedding_backward(s["ids"], s["grad_out"], s["grad_table"], s["scale"], accumulate=s["case"]["accumulate"])
        return s["grad_table"]
    if op == "layernorm":
        if forward:
            B.layernorm_forward(s["x"], s["weight"], s["bias"], s["y"], s["mean"], s["rstd"], eps=EPS_NORM)
            return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
        B.layernorm_backward(s["grad_y"], s["x"], s["weight"], s["mean"], s["rstd"], s["grad_x"], s["grad_weight"],
                             s["grad_bias"])
        return {"x": s["grad_x"], "weight": s["grad_weight"], "bias": s["grad_bias"]}
    if op == "recurrence":
        if forward:
            B.recurrence_forward(s["gate"], s["input"], s["out"], h0=s["h0"], h_last=s["h_last"], lengths=s["lengths"])
            return {"out": s["out"], "last": s["h_last"]}
        B.recurrence_backward(s["gate"], s["input"], s["out"], s["grad_out"], s["grad_gate"], s["grad_input"], h0=s["h0"],
                              grad_last=s["grad_last"], grad_h0=s["grad_h0"], lengths=s["lengths"])
        return {"gate": s["grad_gate"], "input": s["grad_input"], "h0": s["grad_h0"]}
    s["step"] += 1
    B.adamw_step(s["tensors"], s["tensor_grads"], s["state"], LR, s["step"], weight_decay=s["decay"],
                 betas=(BETA1, BETA2), eps=EPS_ADAM, copies=s["tensor_copies"], grad_scale=s["clip"])
    return _results(s["weights"], s["copy"], s["state"])


# ---- what a pass cannot do without ----------------------------------------------------------------------

def _distinct(tokens, vocab):
    """Expected number of different tokens in a batch."""
    top = math.log(vocab + 1.0)
    p = torch.log1p(1.0 / torch.arange(1, vocab + 1, dtype=torch.float64)) / top
    return float((1.0 - (1.0 - p) ** tokens).sum())


def work(case):
    op, e = case["op"], BYTES[case["type"]]
    if op == "embedding":
        t, d, v = case["tokens"], case["dim"], case["vocab"]
        rows = _distinct(t, v)
        if case["dir"] == "forward":
            return {"bytes": t * BYTES[case["index"]] + rows * d * e + t * d * e, "flops": t * d}
        out = 8 * rows * d if case["accumulate"] else 4 * v * d
        return {"bytes": t * (BYTES[case["index"]] + d * e) + out, "flops": 2 * t * d}
    if op == "layernorm":
        r, d = case["rows"], case["dim"]
        if case["dir"] == "forward":
            return {"bytes": 2 * r * d * e + 8 * r + 8 * d, "flops": 8 * r * d}
        return {"bytes": 3 * r * d * e + 8 * r + 12 * d, "flops": 14 * r * d}
    if op == "recurrence":
        n, s = case["batch"] * case["steps"] * case["channels"], case["batch"] * case["channels"]
        if case["dir"] == "forward":
            return {"bytes": 3 * n * e + 8 * s, "flops": 8 * n}
        return {"bytes": 6 * n * e + 12 * s, "flops": 14 * n}
    n = sum(k for k, _ in _sizes(case))
    state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (8 + e + state + (2 if case["copy"] else 0)), "flops": 16 * n}


# ---- the definitions in 64 bits -------------------------------------------------------------------------

def _held(value, root):
    """What 8 bits hold of a tensor in 64 bits: the codes' values and the scales."""
    x = torch.cat([value, value.new_zeros(-len(value) % BLOCK)]).view(-1, BLOCK)
    largest = x.abs().max(1, keepdim=True).values
    codes = torch.where(largest >= TINY, x / largest * TOP, 0.0)
    if root:
        codes = torch.where((codes > 0) & (codes < LEAST), LEAST, codes)
    scale = torch.where(largest >= TINY, largest / TOP, 0.0)
    return codes.float().to(torch.float8_e4m3fn).double().view(-1), scale[:, 0]


def exact(case, seed):
    s = prepare(case, seed)
    op, forward = case["op"], case.get("dir") == "forward"
    if op == "embedding":
        if forward:
            return s["table"].double().index_select(0, s["ids"].long()) * s["scale"]
        # every token's row added to the gradient of its id, one slice of the columns after the other
        total = s["grad_table"].double() if case["accumulate"] else torch.zeros_like(s["grad_table"], dtype=torch.float64)
        ids = s["ids"].long()
        for c in range(0, case["dim"], 256):
            total[:, c:c + 256] += torch.zeros(case["vocab"], min(256, case["dim"] - c), dtype=torch.float64, device=DEVICE) \
                .index_add_(0, ids, s["grad_out"][:, c:c + 256].double()) * s["scale"]
        return total
    if op == "layernorm":
        x, w = s["x"].double(), s["weight"].double()
        if forward:
            var, mean = torch.var_mean(x, 1, correction=0)
            rstd = (var + EPS_NORM) ** -0.5
            return {"y": (x - mean[:, None]) * rstd[:, None] * w + s["bias"].double(), "mean": mean, "rstd": rstd}
        mean, rstd, dy = s["mean"].double()[:, None], s["rstd"].double()[:, None], s["grad_y"].double()
        d, g, n = x - mean, dy * w, case["dim"]
        along = (g * d).sum(1, keepdim=True) * rstd ** 2 / n
        return {"x": rstd * (g - g.sum(1, keepdim=True) / n - d * along), "weight": (dy * d * rstd).sum(0), "bias": dy.sum(0)}
    if op == "recurrence":
        steps = case["steps"]
        f, x, h = s["gate"].double(), s["input"].double(), s["h0"].double()
        a, z = torch.sigmoid(f), torch.sigmoid(-f)
        if s["lengths"] is not None:
            on = _valid(steps, s["lengths"])
            a, z = torch.where(on, a, 1.0), torch.where(on, z, 0.0)
        if forward:
            out = torch.empty_like(f)
            for t in range(steps):
                h = a[:, t] * h + z[:, t] * x[:, t]
                out[:, t] = h
            return {"out": out if s["lengths"] is None else torch.where(on, out, 0.0), "last": h}
        before = torch.cat([h[:, None], s["out"].double()[:, :-1]], 1)
        d = s["grad_out"].double()
        if s["lengths"] is not None:
            d = torch.where(on, d, 0.0)
        total, g = torch.empty_like(f), s["grad_last"].double()
        for t in reversed(range(steps)):
            total[:, t] = g = g + d[:, t]
            g = a[:, t] * g
        return {"gate": total * (before - x) * a * z, "input": total * z, "h0": g}
    # one tensor after the other
    s["step"] += 1
    m, v, m_scale, v_scale = s["state"]
    weights, parts, at, first = [], [], 0, 0
    for (k, _), decay in zip(s["sizes"], s["decay"]):
        g = s["grads"][at:at + k].double()
        if s["clip"] is not None:
            g *= s["clip"].double()
        if m_scale is None:
            pm, pv = m[at:at + k].double(), v[at:at + k].double()
        else:
            blocks = -(-k // BLOCK)
            of = slice(first, first + blocks)
            pm = (m.view(-1, BLOCK)[of].double() * m_scale[of].double()[:, None]).view(-1)[:k]
            pv = (v.view(-1, BLOCK)[of].double() * v_scale[of].double()[:, None]).view(-1)[:k] ** 2
            first += blocks
        pm, pv = BETA1 * pm + (1 - BETA1) * g, BETA2 * pv + (1 - BETA2) * g ** 2
        mh, vh = pm / (1 - BETA1 ** s["step"]), pv / (1 - BETA2 ** s["step"])
        w = s["weights"][at:at + k].double()
        weights.append(w - LR * decay * w - LR * mh / (vh.sqrt() + EPS_ADAM))
        if m_scale is None:
            parts.append((pm, pv))
        else:
            (mc, ms), (rc, rs) = _held(pm, False), _held(pv.sqrt(), True)
            parts.append((mc, rc, ms, rs))
        at += k
    state = [torch.cat(p) for p in zip(*parts)]
    weights = torch.cat(weights)
    return _results(weights, weights if case["copy"] else None, state + [None, None] if len(state) == 2 else state)
