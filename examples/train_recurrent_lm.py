"""A small recurrent language model trained through the library, on one GPU and on synthetic text.

Every step, for each of W simulated data-parallel workers: embedding lookup, layer norm, gated recurrence, layer norm, decoder,
and back, which leaves the worker's gradient in a flat buffer; the W gradients go through Accordion's TopK compression with error
feedback (accordion_step_all), and the averaged gradient it returns, clipped by its norm, is applied by AdamW with moments in 8 bits.
At the end of a window Accordion decides each layer's compression level, and after training the model continues a text token by
token from the recurrent state.  Products with weight matrices and the loss are torch's; everything else above is the library's.

    python examples/train_recurrent_lm.py --steps 200
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


class Model:
    """Parameters as views of one flat buffer; gradients of a worker as views of another one."""

    def __init__(self, vocab: int, dim: int, device: str, seed: int):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.vocab, self.dim = vocab, dim
        self.shapes = {"table": (vocab, dim), "norm1.weight": (dim,), "norm1.bias": (dim,), "project": (2 * dim, dim),
                       "project.bias": (2 * dim,), "norm2.weight": (dim,), "norm2.bias": (dim,), "decoder": (vocab, dim)}
        self.sizes = [math.prod(s) for s in self.shapes.values()]
        self.flat = torch.empty(sum(self.sizes), device=device)
        self.p = dict(zip(self.shapes, (v.view(s) for v, s in zip(self.flat.split(self.sizes), self.shapes.values()))))
        for name, p in self.p.items():
            if p.dim() == 2:
                p.normal_(0.0, dim ** -0.5, generator=gen)
            else:
                p.fill_(1.0 if name.endswith("weight") else 0.0)
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

    def __call__(self, ids, h0):
        p = self.p
        x = LayerNorm.apply(Embedding.apply(p["table"], ids, math.sqrt(self.dim)), p["norm1.weight"], p["norm1.bias"])
        both = torch.addmm(p["project.bias"], x.view(-1, self.dim), p["project"].t()).view(*ids.shape, -1)
        h, last = Recurrence.apply(both, h0)
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
          window: int = 20, device: str = "cuda:0", say=print):
    """Losses of the steps, and how much of a continued text follows the rule."""
    model, gen = Model(vocab, dim, device, 1), torch.Generator(device=device).manual_seed(2)
    n = model.flat.numel()
    accordion = B.Accordion(B.ACC_TOPK, model.layers(), workers, 20, 5, device=device)
    state = B.adamw_state(model.sizes, 8, device)
    grads, mean = [torch.zeros(n, device=device) for _ in range(workers)], torch.empty(n, device=device)
    decay = [0.01 if len(s) == 2 else 0.0 for s in model.shapes.values()]
    h0, losses = torch.zeros(batch, dim, device=device), []
    for step in range(1, steps + 1):
        total = 0.0
        for w in range(workers):
            ids = text(gen, batch, length, vocab, device)
            model.gradients_into(grads[w])
            logits, _ = model(ids[:, :-1].contiguous(), h0)
            loss = torch.nn.functional.cross_entropy(logits, ids[:, 1:].reshape(-1))
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
        token, h = torch.randint(0, vocab, (batch, 1), generator=gen, device=device), h0.clone()
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
    a = ap.parse_args()
    losses, right = train(a.steps, a.workers)
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f}; {100 * right:.0f} % of the continued text follows the rule")


if __name__ == "__main__":
    main()
