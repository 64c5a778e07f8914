"""The selective scan over sequences whose states are carried over hundreds of chunks, and with bounds that know how the steps are cut."""
import numpy as np
import pytest
import torch

from tests import more_operators_plain as M
from tests.test_gpu_operators_scan import BF16, DEV, F32, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("steps,channels,states", [(8192, 8, 16), (9001, 5, 3), (20000, 3, 5)])
def test_states_are_carried_over_many_chunks(steps, channels, states, kind, monkeypatch):
    """Decays by which a state lasts for one to some thousand steps.  The sums of dt that the carry takes are those of a chunk, up to 256 steps, added over a
    wave's run of chunks: at most the sequence's number of chunks of 16 over 16 waves."""
    print(f"case carry {steps} {channels} {states} {kind}", flush=True)
    s = make(1, steps, channels, states, kind)
    s["a"] = -torch.logspace(-3, 0.5, channels * states).view(channels, states).to(DEV)
    monkeypatch.setattr(M, "CHUNK", 256 + steps // 256 + 16)
    check(s)


@pytest.mark.parametrize("growth", [0.05, 0.18])
@pytest.mark.parametrize("channels,states", [(8, 16), (64, 16), (3, 5)])
def test_growing_states_behind_zeros(channels, states, growth, monkeypatch):
    """States that grow, but that are zero until shortly before the end, and gradients that are until shortly after the start: numbers throughout, though a factor over
    the steps between is beyond fp32."""
    print(f"case growing {channels} {states} {growth}", flush=True)
    steps, live = 8192, 192
    s = make(1, steps, channels, states, softplus=False, bias=False, h0=False)
    s["a"] = torch.full_like(s["a"], growth)
    s["delta"] = torch.full_like(s["delta"], 1.0)
    s["x"][:, :steps - live] = 0
    s["dout"][:, live:] = 0
    monkeypatch.setattr(M, "CHUNK", 256 + steps // 256 + 16)
    check(s, dlast=False)
    # a small state that grows over many chunks, and a gradient that does
    s = make(1, 2000, channels, states, softplus=False, bias=False)
    s["a"] = torch.full_like(s["a"], 0.06)
    s["delta"] = torch.full_like(s["delta"], 1.0)
    s["h0"], s["dlast"] = s["h0"] * 1e-30, s["dlast"] * 1e-30
    s["x"].zero_(), s["dout"].zero_()
    check(s)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("states", [1, 4, 6, 16, 24, 64])
@pytest.mark.parametrize("steps", [1, 9, 16, 17, 40, 64])
def test_steps_of_one_walk_take_no_sums_of_steps(steps, states, kind, monkeypatch):
    """Up to 64 steps of the forward pass are one walk: no sum of dt is among the roundings of a decay."""
    print(f"case one walk {steps} {states} {kind}", flush=True)
    monkeypatch.setattr(M, "CHUNK", 0)
    check(make(3, steps, 70, states, kind, seed=steps), back=False)
    s = make(3, steps, 70, states, kind, softplus=False, seed=steps)
    s["a"] = 8 * s["a"]
    check(s, back=False)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("steps", [100, 700])
def test_sums_of_a_chunk_are_its_steps(steps, kind, monkeypatch):
    """A few sequences: chunks of 32 steps forward, of 16 backward."""
    print(f"case chunks {steps} {kind}", flush=True)
    monkeypatch.setattr(M, "CHUNK", 32 + steps // 16)
    check(make(2, steps, 70, 16, kind, seed=steps), back=False)
