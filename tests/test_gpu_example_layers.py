"""The example's layers under gradients that are not laid out as their outputs: transposed, and one number for all."""
import os
import sys

import pytest
import torch

from tests import more_operators_plain as M
from tests.operators_plain import assert_within
from tests.test_gpu_operators_convolution import make as convolution
from tests.test_gpu_operators_scan import make as scan

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def gradients(out):
    """(loss, the gradient of out) of a loss that reads out transposed, and of a sum."""
    weight = torch.randn(out.shape[0], out.shape[2], out.shape[1], generator=torch.Generator().manual_seed(8)).to(out.device)
    yield (out.transpose(1, 2) * weight).sum(), weight.transpose(1, 2)
    yield out.sum(), torch.ones_like(out)


def test_convolution():
    import train_recurrent_lm as example
    s = convolution(3, 20, 10, 4, torch.float32)
    leaves = [s[k].requires_grad_(True) for k in ("x", "weight", "bias")]
    for i in range(2):
        out, _ = example.Convolution.apply(*leaves, s["state"])
        loss, grad = list(gradients(out))[i]
        got = torch.autograd.grad(loss, leaves)
        refs, offs = M.convolution_gradients(*leaves, s["state"], None, True, grad, None)
        for name, g, ref, off in zip(("x", "weight", "bias"), got, refs, offs):
            assert_within(g, ref, off, name)


def test_scan():
    import train_recurrent_lm as example
    s = scan(3, 20, 10, 16)
    n, log_a = 16, (-s["a"]).log()
    shared = torch.cat([s["b"], s["c"]], -1).squeeze(2)
    leaves = [t.requires_grad_(True) for t in (s["x"], s["delta"], shared, s["d"], s["gate"], s["delta_bias"])]
    x, delta, shared, d, gate, bias = leaves
    for i in range(2):
        out, _ = example.Scan.apply(x, delta, log_a, shared, d, gate, bias, s["h0"])
        loss, grad = list(gradients(out))[i]
        got = torch.autograd.grad(loss, leaves)
        ref = M.Scan(x, delta, -torch.exp(log_a), shared[..., :n], shared[..., n:], d, gate, bias, True, s["h0"])
        refs, offs = ref.gradients(grad)
        for name, g in zip(("x", "delta", None, "d", "gate", "delta_bias"), got):
            if name is None:
                for k, part in (("b", g[..., :n]), ("c", g[..., n:])):
                    assert_within(part.contiguous(), refs[k].reshape(part.shape), offs[k].reshape(part.shape), k)
            else:
                assert_within(g, refs[name].reshape(g.shape), offs[name].reshape(g.shape), name)
