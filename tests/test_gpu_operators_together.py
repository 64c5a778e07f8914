"""The language-model operators as a program uses them: on other streams, in captured graphs, with workspaces of the caller's, and
together in a training run whose gradients go through the compressor."""
import os
import sys

import numpy as np
import pytest
import torch

from paper_2010_16248_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Step:
    """One forward and backward pass through the three layers and an AdamW step, on buffers of its own."""

    def __init__(self, tokens, seed):
        gen = torch.Generator().manual_seed(seed)
        batch, steps, dim, vocab = 2, tokens // 2, 40, 300
        r = lambda *s: torch.randn(*s, generator=gen).to(DEV)
        self.ids = torch.randint(0, vocab, (tokens,), generator=gen).to(DEV)
        self.table, self.weight, self.bias, self.gate = r(vocab, dim), r(dim), r(dim), r(batch, steps, dim)
        self.h0, self.dh = r(batch, dim), r(batch, steps, dim)
        e = lambda *s: torch.zeros(*s, device=DEV)
        self.x, self.y, self.mean, self.rstd = e(tokens, dim), e(tokens, dim), e(tokens), e(tokens)
        self.h, self.last, self.dgate, self.dy, self.dh0 = e(batch, steps, dim), e(batch, dim), e(batch, steps, dim), e(batch, steps, dim), e(batch, dim)
        self.dx, self.dw, self.db, self.dtable = e(tokens, dim), e(dim), e(dim), e(vocab, dim)
        self.params = [self.table, self.weight, self.bias]
        self.state = B.adamw_state([p.numel() for p in self.params], 8, DEV)
        self.shape = (batch, steps, dim)

    def run(self, workspace=None):
        ws = dict(workspace=workspace) if workspace is not None else {}
        B.embedding_forward(self.ids, self.table, self.x, 2.0)
        B.layernorm_forward(self.x, self.weight, self.bias, self.y, self.mean, self.rstd)
        B.recurrence_forward(self.gate, self.y.view(self.shape), self.h, h0=self.h0, h_last=self.last, **ws)
        B.recurrence_backward(self.gate, self.y.view(self.shape), self.h, self.dh, self.dgate, self.dy, h0=self.h0, grad_last=self.last,
                              grad_h0=self.dh0, **ws)
        B.layernorm_backward(self.dy.view(self.x.shape), self.x, self.weight, self.mean, self.rstd, self.dx, self.dw, self.db, **ws)
        B.embedding_backward(self.ids, self.dx, self.dtable, 2.0, **ws)
        B.adamw_step(self.params, [self.dtable, self.dw, self.db], self.state, 1e-3, 1)

    def results(self):
        return [t.clone() for t in (self.x, self.y, self.h, self.last, self.dgate, self.dy, self.dh0, self.dx, self.dw, self.db, self.dtable,
                                    self.table, self.weight, self.bias, self.state[0].view(torch.uint8), self.state[1].view(torch.uint8),
                                    self.state[2], self.state[3])]


def _same(a, b, what):
    for i, (x, y) in enumerate(zip(a, b)):
        assert torch.equal(x, y), f"{what}: result {i}"


@pytest.mark.parametrize("tokens", [2, 600, 20000])
def test_other_streams_and_dirty_workspaces_give_the_same_bits(tokens):
    print(f"case streams {tokens}", flush=True)
    plain = Step(tokens, 1)
    plain.run()
    ref = plain.results()
    side = torch.cuda.Stream()
    other = Step(tokens, 1)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        other.run()
    side.synchronize()
    _same(ref, other.results(), "side stream")
    third = Step(tokens, 1)
    dirty = torch.full((64 << 20,), 0xff, dtype=torch.uint8, device=DEV)
    third.run(workspace=dirty)
    _same(ref, third.results(), "workspace of the caller's")


@pytest.mark.parametrize("tokens", [2, 600, 20000])
def test_a_captured_step_replays_like_eager(tokens):
    print(f"case graph {tokens}", flush=True)
    graphed, eager = Step(tokens, 2), Step(tokens, 2)
    graphed.run()
    eager.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            graphed.run()
    gen = torch.Generator().manual_seed(9)
    for replay in range(4):
        ids = torch.randint(0, 300, (tokens,), generator=gen).to(DEV)
        gate = (torch.randn(*graphed.shape, generator=gen) + replay).to(DEV)
        for s in (graphed, eager):
            s.ids.copy_(ids), s.gate.copy_(gate)
        torch.cuda.synchronize()
        graph.replay()
        eager.run()
        torch.cuda.synchronize()
        _same(graphed.results(), eager.results(), f"replay {replay}")
        torch.zeros(1 << 20, device=DEV).sum().item()          # the program's own work in between


def test_workspaces_that_are_too_small_or_elsewhere_are_refused():
    s = Step(2000, 3)
    with pytest.raises(B.AccordionError) as err:
        B.embedding_backward(s.ids, s.dx, s.dtable, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    assert err.value.status == B.ACC_ENOSPACE
    with pytest.raises(ValueError):
        B.embedding_backward(s.ids, s.dx, s.dtable, workspace=torch.empty(1 << 24, dtype=torch.uint8))
    with pytest.raises(B.AccordionError) as err:
        B.embedding_backward(s.ids, s.dx, s.dx)
    assert err.value.status == B.ACC_EINVAL


def test_a_language_model_learns_through_the_compressor():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import train_recurrent_lm as example
    losses, right = example.train(steps=150, say=lambda *_: None)
    print(f"losses {losses[0]:.3f} {losses[49]:.3f} {losses[-1]:.3f}, right {right:.2f}", flush=True)
    assert all(np.isfinite(losses))
    # ln(257) = 5.55 at the start; the text's own entropy is 0.1 ln(257) + 0.33 = 0.88
    assert losses[0] > 5.0 and losses[-1] < 2.0 and right > 0.8
