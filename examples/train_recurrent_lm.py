"""A small recurrent language model trained through the library, on one GPU and on synthetic text.

Every step, for each of W simulated data-parallel workers: embedding lookup, layer norm, gated recurrence, layer norm, decoder,
and back, which leaves the worker's gradient in a flat buffer; the W gradients go through Accordion's TopK compression with error
feedback (accordion_step_all), and the averaged gradient it returns, clipped by its norm, is applied by AdamW with moments in 8 bits.
At the end of a window Accordion decides each layer's compression level, and after training the model continues a text token by
token from the recurrent state.  Products with weight matrices and the loss are torch's; everything else above is the library's.

--mixer scan: in the recurrence's place a short convolution and a selective state space scan, gated, and the loss is the library's too (the tokens'
log probabilities).

    python examples/train_recurrent_lm.py --steps 200
    python examples/train_recurrent_lm.py --mixer scan
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2010_16248_amd import binding as B  # noqa: E402


class Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids, scale):
        out = torch.empty(*ids.shape, table.shape[1], device=table.device)
        B.embedding_forward(ids, table, out, scale)
        ctx.save_for_backward(ids)
        ctx.table, ctx.scale = table.shape, scale
        return out

    @staticmethod
    def backward(ctx, grad):
        (ids,) = ctx.saved_tensors
        table = torch.empty(ctx.table, device=grad.device)
        B.embedding_backward(ids, grad.contiguous(), table, ctx.scale)
        return table, None, None


class LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias):
        y, rows = torch.empty_like(x), x.numel() // x.shape[-1]
        mean, rstd = torch.empty(rows, device=x.device), torch.empty(rows, device=x.device)
        B.layernorm_forward(x, weight, bias, y, mean, rstd)
        ctx.save_for_backward(x, weight, mean, rstd)
        return y

    @staticmethod
    def backward(ctx, grad):
        x, weight, mean, rstd = ctx.saved_tensors
        dx, dw, db = torch.empty_like(x), torch.empty_like(weight), torch.empty_like(weight)
        B.layernorm_backward(grad.contiguous(), x, weight, mean, rstd, dx, dw, db)
        return dx, dw, db


class Recurrence(torch.autograd.Function):
    """both: gates and inputs side by side, as one projection writes them."""

    @staticmethod
    def forward(ctx, both, h0):
        c = both.shape[2] // 2
        out, last = torch.empty(*both.shape[:2], c, device=both.device), torch.empty_like(h0)
        B.recurrence_forward(both[..., :c], both[..., c:], out, h0=h0, h_last=last)
        ctx.save_for_backward(both, h0, out)
        ctx.mark_non_differentiable(last)
        return out, last

    @staticmethod
    def backward(ctx, grad, _):
        both, h0, out = ctx.saved_tensors
        c, grads = both.shape[2] // 2, torch.empty_like(both)
        B.recurrence_backward(both[..., :c], both[..., c:], out, grad.contiguous(), grads[..., :c], grads[..., c:], h0=h0)
        return grads, None


class Convolution(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, state):
        out, last = torch.empty_like(x, memory_format=torch.contiguous_format), torch.empty_like(state)
        B.convolution_forward(x, weight, out, bias=bias, state=state, last=last, silu=True)
        ctx.save_for_backward(x, weight, bias, state)
        ctx.mark_non_differentiable(last)
        return out, last

    @staticmethod
    def backward(ctx, grad, _):
        x, weight, bias, state = ctx.saved_tensors
        grad = grad.contiguous()
        dx, dw, db = torch.empty_like(grad), torch.empty_like(weight), torch.empty_like(bias)
        B.convolution_backward(x, weight, grad, dx, dw, bias=bias, grad_bias=db, state=state, silu=True)
        return dx, dw, db, None


class Scan(torch.autograd.Function):
    """shared: b and c side by side."""

    @staticmethod
    def forward(ctx, x, delta, log_a, shared, d, gate, delta_bias, h0):
        a, n = -torch.exp(log_a), log_a.shape[1]
        out, last = torch.empty_like(x), torch.empty_like(h0)
        B.scan_forward(x, delta, a, shared[..., :n], shared[..., n:], out, d=d, gate=gate, delta_bias=delta_bias, softplus=True, h0=h0, h_last=last)
        ctx.save_for_backward(x, delta, a, shared, d, gate, delta_bias, h0)
        ctx.mark_non_differentiable(last)
        return out, last

    @staticmethod
    def backward(ctx, grad, _):
        x, delta, a, shared, d, gate, delta_bias, h0 = ctx.saved_tensors
        n, grads = a.shape[1], [torch.empty_like(t) for t in (x, delta, a, shared, d, x, delta_bias)]
        dx, ddelta, da, dshared, dd, dgate, dbias = grads
        B.scan_backward(x, delta, a, shared[..., :n], shared[..., n:], grad.contiguous(), dx, ddelta, da, dshared[..., :n], dshared[..., n:], d=d,
                        grad_d=dd, gate=gate, grad_gate=dgate, delta_bias=delta_bias, grad_delta_bias=dbias, softplus=True, h0=h0)
        return dx, ddelta, da * a, dshared, dd, dgate, dbias, None


class LogProb(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets):
        logprob, lse = (torch.empty(len(targets), device=logits.device) for _ in range(2))
        B.logprob_forward(logits, targets, logprob, lse=lse)
        ctx.save_for_backward(logits, targets, lse)
        return logprob

    @staticmethod
    def backward(ctx, grad):
        logits, targets, lse = ctx.saved_tensors
        out = torch.empty_like(logits)
        B.logprob_backward(logits, targets, lse, grad.contiguous(), out)
        return out, None


WIDTH, STATES = 4, 16       # of the convolution, of a channel


def loss_of(model, logits, targets):
    if model.mixer == "scan":
        return -LogProb.apply(logits, targets).mean()
    return torch.nn.functional.cross_entropy(logits, targets)


class Model:
    """Parameters as views of one flat buffer; gradients of a worker as views of another one."""

    def __init__(self, vocab: int, dim: int, device: str, seed: int, mixer: str = "recurrence"):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.vocab, self.dim, self.mixer = vocab, dim, mixer
        self.shapes = {"table": (vocab, dim), "norm1.weight": (dim,), "norm1.bias": (dim,), "project": (2 * dim, dim),
                       "project.bias": (2 * dim,), "norm2.weight": (dim,), "norm2.bias": (dim,), "decoder": (vocab, dim)}
        if mixer == "scan":
            self.shapes.update({"conv": (dim, WIDTH), "conv.bias": (dim,), "steps": (dim, dim), "steps.bias": (dim,), "shared": (2 * STATES, dim),
                                "log_a": (dim, STATES), "skip": (dim,)})
        self.sizes = [math.prod(s) for s in self.shapes.values()]
        self.flat = torch.empty(sum(self.sizes), device=device)
        self.p = dict(zip(self.shapes, (v.view(s) for v, s in zip(self.flat.split(self.sizes), self.shapes.values()))))
        for name, p in self.p.items():
            if p.dim() == 2:
                p.normal_(0.0, dim ** -0.5, generator=gen)
            else:
                p.fill_(1.0 if name.endswith("weight") else 0.0)
        if mixer == "scan":
            # states that remember for 1 / n steps of dt, dt from 0.001 to 0.1 by channel
            self.p["log_a"][:] = torch.arange(1, STATES + 1, device=device).float().log()
            self.p["steps.bias"][:] = torch.expm1(torch.linspace(math.log(1e-3), math.log(1e-1), dim, device=device).exp()).log()
            self.p["skip"].fill_(1.0)
        else:
            self.p["project.bias"][:dim] = torch.linspace(-1.0, 4.0, dim, device=device)     # memories of different lengths
        for p in self.p.values():
            p.requires_grad_(True)

    def layers(self):
        """(offset, rows, cols, is_matrix) for the compressor."""
        out, at = [], 0
        for s, n in zip(self.shapes.values(), self.sizes):
            out.append((at, *(s if len(s) == 2 else (1, s[0])), int(len(s) == 2)))
            at += n
        return out

    def gradients_into(self, flat):
        flat.zero_()
        for p, g in zip(self.p.values(), flat.split(self.sizes)):
            p.grad = g.view(p.shape)

    def first_state(self, batch: int, device: str):
        if self.mixer == "scan":
            return torch.zeros(batch, WIDTH - 1, self.dim, device=device), torch.zeros(batch, self.dim, STATES, device=device)
        return torch.zeros(batch, self.dim, device=device)

    def mix(self, both, state):
        """What the mixing layer makes of its projection, and the state behind it."""
        p, c = self.p, self.dim
        if self.mixer != "scan":
            return Recurrence.apply(both, state)
        front, h0 = state
        u, front = Convolution.apply(both[..., :c], p["conv"], p["conv.bias"], front)
        delta, shared = u @ p["steps"].t(), u @ p["shared"].t()
        y, last = Scan.apply(u, delta, p["log_a"], shared, p["skip"], both[..., c:], p["steps.bias"], h0)
        return y, (front, last)

    def __call__(self, ids, h0):
        p = self.p
        x = LayerNorm.apply(Embedding.apply(p["table"], ids, math.sqrt(self.dim)), p["norm1.weight"], p["norm1.bias"])
        both = torch.addmm(p["project.bias"], x.view(-1, self.dim), p["project"].t()).view(*ids.shape, -1)
        h, last = self.mix(both, h0)
        y = LayerNorm.apply(h, p["norm2.weight"], p["norm2.bias"])
        return y.view(-1, self.dim) @ p["decoder"].t(), last


def text(gen, batch: int, steps: int, vocab: int, device: str):
    """Sequences in which a token follows from the one before it, nine times of ten."""
    ids = torch.empty(batch, steps + 1, dtype=torch.int64, device=device)
    ids[:, 0] = torch.randint(0, vocab, (batch,), generator=gen, device=device)
    odd = torch.rand(batch, steps, generator=gen, device=device) < 0.1
    other = torch.randint(0, vocab, (batch, steps), generator=gen, device=device)
    for t in range(steps):
        ids[:, t + 1] = torch.where(odd[:, t], other[:, t], (5 * ids[:, t] + 7) % vocab)
    return ids


def train(steps: int = 200, workers: int = 2, batch: int = 8, length: int = 64, vocab: int = 257, dim: int = 96, lr: float = 4e-3,
          window: int = 20, device: str = "cuda:0", say=print, mixer: str = "recurrence"):
    """Losses of the steps, and how much of a continued text follows the rule."""
    model, gen = Model(vocab, dim, device, 1, mixer), torch.Generator(device=device).manual_seed(2)
    n = model.flat.numel()
    accordion = B.Accordion(B.ACC_TOPK, model.layers(), workers, 20, 5, device=device)
    state = B.adamw_state(model.sizes, 8, device)
    grads, mean = [torch.zeros(n, device=device) for _ in range(workers)], torch.empty(n, device=device)
    decay = [0.01 if len(s) == 2 else 0.0 for s in model.shapes.values()]
    h0, losses = model.first_state(batch, device), []
    for step in range(1, steps + 1):
        total = 0.0
        for w in range(workers):
            ids = text(gen, batch, length, vocab, device)
            model.gradients_into(grads[w])
            logits, _ = model(ids[:, :-1].contiguous(), h0)
            loss = loss_of(model, logits, ids[:, 1:].reshape(-1))
            loss.backward()
            total += loss.item() / workers
        losses.append(total)
        accordion.step_all(grads, mean)
        clip = (1.0 / (mean.norm() + 1e-6)).clamp(max=1.0).reshape(1)
        with torch.no_grad():
            B.adamw_step(list(model.flat.split(model.sizes)), list(mean.split(model.sizes)), state, lr, step, weight_decay=decay,
                         betas=(0.9, 0.99), grad_scale=clip)
        if step % window == 0:
            accordion.detect_regime(lr, lr)
            say(f"step {step}: loss {total:.3f}, layers at the accurate level: {int(accordion.get_levels().sum())} of {len(model.sizes)}")
    # continue a text, one token at a time
    with torch.no_grad():
        token, h = torch.randint(0, vocab, (batch, 1), generator=gen, device=device), h0
        right = 0
        for _ in range(length):
            logits, h = model(token, h)
            follows = logits.argmax(1, keepdim=True)
            right += int((follows == (5 * token + 7) % vocab).sum())
            token = follows
    accordion.destroy()
    return losses, right / (batch * length)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--workers", type=int, default=2)
    ap.add_argument("--mixer", choices=("recurrence", "scan"), default="recurrence")
    a = ap.parse_args()
    losses, right = train(a.steps, a.workers, mixer=a.mixer)
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f}; {100 * right:.0f} % of the continued text follows the rule")


if __name__ == "__main__":
    main()
