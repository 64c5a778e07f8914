"""The convolution, the scan and the log probabilities as a program uses them: one behind the other, on other streams, in captured graphs, with
workspaces of the caller's, and in a training run through the compressor."""
import os
import sys

import numpy as np
import pytest
import torch

from paper_2010_16248_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Layer:
    """A mixing layer and its tokens' log probabilities, forward and backward, on buffers of its own: convolution, scan, and logits that are a
    product with a matrix."""

    def __init__(self, batch, steps, seed, kind=torch.float32, channels=72, states=16, vocab=2100):
        gen = torch.Generator().manual_seed(seed)
        r = lambda *s, k=torch.float32: torch.randn(*s, generator=gen).to(k).to(DEV)
        e = lambda *s, k=torch.float32: torch.zeros(*s, dtype=k, device=DEV)
        shape, k = (batch, steps, channels), kind
        self.both, self.delta, self.shared = r(batch, steps, 2 * channels, k=k), r(*shape, k=k), r(batch, steps, 2 * states, k=k)
        self.weight, self.bias, self.state = r(channels, 4), r(channels), r(batch, 3, channels)
        self.a, self.d, self.dbias, self.h0 = -r(channels, states).exp(), r(channels), r(channels) - 2, r(batch, channels, states)
        self.decoder, self.targets = r(vocab, channels, k=k) * 0.1, torch.randint(-1, vocab, (batch * steps,), generator=gen).to(DEV)
        self.lengths = torch.randint(0, steps + 1, (batch,), generator=gen).to(torch.int32).to(DEV)
        rows = batch * steps
        self.u, self.last, self.y, self.h_last = e(*shape, k=k), e(batch, 3, channels), e(*shape, k=k), e(batch, channels, states)
        self.logits, self.lp, self.lse, self.entropy = e(rows, vocab, k=k), e(rows), e(rows), e(rows)
        self.values, self.ids = e(rows, 5), e(rows, 5, k=torch.int64)
        self.g, self.ge = r(rows), r(rows)
        self.dlogits, self.dy = e(rows, vocab, k=k), e(*shape, k=k)
        self.dboth, self.ddelta, self.dshared, self.du = e(batch, steps, 2 * channels, k=k), e(*shape, k=k), e(batch, steps, 2 * states, k=k), e(*shape, k=k)
        self.da, self.dd, self.ddbias, self.dh0 = e(channels, states), e(channels), e(channels), e(batch, channels, states)
        self.dweight, self.dconvbias, self.dstate = e(channels, 4), e(channels), e(batch, 3, channels)
        self.c, self.n = channels, states

    def run(self, workspace=None):
        ws = dict(workspace=workspace) if workspace is not None else {}
        c, n = self.c, self.n
        x, z, dx, dz = self.both[..., :c], self.both[..., c:], self.dboth[..., :c], self.dboth[..., c:]
        b, cc, db, dc = self.shared[..., :n], self.shared[..., n:], self.dshared[..., :n], self.dshared[..., n:]
        options = dict(d=self.d, gate=z, delta_bias=self.dbias, softplus=True, h0=self.h0, lengths=self.lengths)
        B.convolution_forward(x, self.weight, self.u, bias=self.bias, state=self.state, last=self.last, lengths=self.lengths, silu=True)
        B.scan_forward(self.u, self.delta, self.a, b, cc, self.y, h_last=self.h_last, **options, **ws)
        torch.mm(self.y.view(-1, c), self.decoder.t(), out=self.logits)
        B.logprob_forward(self.logits, self.targets, self.lp, self.lse, self.entropy, self.values, self.ids, **ws)
        B.logprob_backward(self.logits, self.targets, self.lse, self.g, self.dlogits, entropy=self.entropy, grad_entropy=self.ge)
        torch.mm(self.dlogits, self.decoder, out=self.dy.view(-1, c))
        B.scan_backward(self.u, self.delta, self.a, b, cc, self.dy, self.du, self.ddelta, self.da, db, dc, grad_d=self.dd, grad_gate=dz,
                        grad_delta_bias=self.ddbias, grad_last=self.h_last, grad_h0=self.dh0, **options, **ws)
        B.convolution_backward(x, self.weight, self.du, dx, self.dweight, bias=self.bias, grad_bias=self.dconvbias, state=self.state,
                               grad_last=self.last, grad_state=self.dstate, lengths=self.lengths, silu=True, **ws)

    def results(self):
        return [t.clone() for t in (self.u, self.last, self.y, self.h_last, self.lp, self.lse, self.entropy, self.values, self.ids, self.dlogits,
                                    self.dboth, self.ddelta, self.dshared, self.du, self.da, self.dd, self.ddbias, self.dh0, self.dweight,
                                    self.dconvbias, self.dstate)]


def _same(a, b, what):
    for i, (x, y) in enumerate(zip(a, b)):
        assert torch.equal(x, y), f"{what}: result {i}"


SHAPES = [(2, 1), (3, 50), (2, 700)]
KINDS = [torch.float32, torch.bfloat16]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", SHAPES)
def test_other_streams_and_dirty_workspaces_give_the_same_bits(shape, kind):
    print(f"case streams {shape} {kind}", flush=True)
    plain = Layer(*shape, 1, kind)
    plain.run()
    ref = plain.results()
    side = torch.cuda.Stream()
    other = Layer(*shape, 1, kind)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        other.run()
    side.synchronize()
    _same(ref, other.results(), "side stream")
    third = Layer(*shape, 1, kind)
    dirty = torch.full((64 << 20,), 0xff, dtype=torch.uint8, device=DEV)
    third.run(workspace=dirty)
    _same(ref, third.results(), "workspace of the caller's")


@pytest.mark.parametrize("shape", SHAPES)
def test_two_calls_at_once(shape):
    """Two streams, each with a layer and a workspace of its own."""
    print(f"case two streams {shape}", flush=True)
    refs = []
    for seed in (1, 2):
        layer = Layer(*shape, seed)
        layer.run()
        refs.append(layer.results())
    layers, streams = [Layer(*shape, seed) for seed in (1, 2)], [torch.cuda.Stream() for _ in range(2)]
    spaces = [torch.empty(64 << 20, dtype=torch.uint8, device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for layer, stream, space in zip(layers, streams, spaces):
            with torch.cuda.stream(stream):
                layer.run(workspace=space)
    torch.cuda.synchronize()
    for layer, ref in zip(layers, refs):
        _same(ref, layer.results(), "beside another")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape", SHAPES)
def test_captured_layers_replay_like_eager(shape, kind):
    """Two graphs with one workspace, replayed one behind the other, with eager work between."""
    print(f"case graphs {shape} {kind}", flush=True)
    space = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)
    graphed, eager, graphs = [Layer(*shape, s, kind) for s in (2, 3)], [Layer(*shape, s, kind) for s in (2, 3)], []
    for layer in (*graphed, *eager):
        layer.run(space)
    for layer in graphed:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.stream(side):
            with torch.cuda.graph(graphs[-1], stream=side):
                layer.run(space)
    gen = torch.Generator().manual_seed(9)
    for replay in range(4):
        for a, b in zip(graphed, eager):
            both = torch.randn(*a.both.shape, generator=gen).to(DEV)
            lengths = torch.randint(0, shape[1] + 1, (shape[0],), generator=gen).to(torch.int32).to(DEV)
            for layer in (a, b):
                layer.both.copy_(both), layer.lengths.copy_(lengths)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        for layer in eager:
            layer.run()
        torch.cuda.synchronize()
        for a, b in zip(graphed, eager):
            _same(a.results(), b.results(), f"replay {replay}")
        torch.zeros(1 << 20, device=DEV).sum().item()          # the program's own work in between


def test_workspaces_that_are_too_small_or_elsewhere_are_refused():
    s = Layer(3, 50, 3)
    small, far = torch.empty(256, dtype=torch.uint8, device=DEV), torch.empty(1 << 26, dtype=torch.uint8)
    for space, error in ((small, B.AccordionError), (far, ValueError)):
        with pytest.raises(error):
            B.scan_forward(s.u, s.delta, s.a, s.shared[..., :16], s.shared[..., 16:], s.y, workspace=space)
        with pytest.raises(error):
            B.convolution_backward(s.u, s.weight, s.y, s.du, s.dweight, workspace=space)
    with pytest.raises(B.AccordionError) as err:
        B.scan_forward(s.u, s.delta, s.a, s.shared[..., :16], s.shared[..., 16:], s.u)
    assert err.value.status == B.ACC_EINVAL


def test_a_language_model_with_scans_runs_through_the_compressor():
    """It runs, its gradients are finite, and those of its parameters follow the loss (differences along a random direction)."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import train_recurrent_lm as example
    losses, right = example.train(steps=20, mixer="scan", say=lambda *_: None)
    assert all(np.isfinite(losses)) and 0 <= right <= 1
    model = example.Model(101, 32, DEV, 5, mixer="scan")
    gen = torch.Generator(device=DEV).manual_seed(6)
    ids = torch.randint(0, 101, (3, 41), generator=gen, device=DEV)
    start = model.first_state(3, DEV)

    def loss():
        return example.loss_of(model, model(ids[:, :-1].contiguous(), start)[0], ids[:, 1:].reshape(-1))

    grads = torch.zeros_like(model.flat)
    model.gradients_into(grads)
    loss().backward()
    assert torch.isfinite(grads).all()
    with torch.no_grad():
        keep, step = model.flat.clone(), 1e-2
        way = grads / grads.norm()                       # along it the loss changes by the gradient's norm
        model.flat.copy_(keep + step * way)
        up = loss().item()
        model.flat.copy_(keep - step * way)
        down = loss().item()
        model.flat.copy_(keep)
    # the loss, about 5, holds 24 bits: 120 losses of 2^-22 each at most over 2 steps of 0.01; the third derivative times step^2 / 6
    norm = grads.norm().item()
    assert abs((up - down) / (2 * step) - norm) <= 2 * 5 * 2.0 ** -20 / step + 0.05 * norm
