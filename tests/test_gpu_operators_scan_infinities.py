"""Infinite inputs, states and gradients of the selective scan: what the definition gives, however the steps and the states are cut."""
import numpy as np
import pytest
import torch

from paper_2010_16248_amd import binding as B
from tests import more_operators_plain as M
from tests.operators_plain import assert_within
from tests.test_gpu_operators_scan import ARGS, BF16, DEV, F32, OPTIONS, backward, forward, make

pytestmark = pytest.mark.gpu
INF = float("inf")


def positive(batch, steps, channels, states, kind=F32, fall=1.0, **kw):
    """Inputs above zero: a sum over states, channels or steps with an infinite term is infinite, never a difference of infinities.  A state falls to
    exp(-fall / 2) to exp(-fall) of itself each step."""
    s = make(batch, steps, channels, states, kind, softplus=False, bias=False, **kw)
    for k in ("x", "b", "c", "gate", "dout", "dlast", "h0", "d"):
        if s[k] is not None:
            s[k] = s[k].abs() + 0.1
    gen = torch.Generator().manual_seed(steps + states)
    s["a"] = -fall * (0.5 + 0.5 * torch.rand(channels, states, generator=gen)).to(DEV)
    s["delta"] = torch.full_like(s["delta"], 1.0)
    return s


def within(got, ref, bound, what):
    """Where an infinity has made a bound of nothing, finite is all that is asked of a finite result."""
    assert_within(got, ref, np.where(np.isnan(bound), INF, bound), what)


def check(s, back=True):
    with np.errstate(all="ignore"):
        ref = M.Scan(*(s[k] for k in ARGS), **{k: s[k] for k in OPTIONS})
        refs, offs = ref.gradients(s["dout"], s["dlast"])
        out, last = forward(s)
        within(out, ref.out, ref.out_off, "out")
        within(last, ref.last, ref.last_off, "h_last")
        if back:
            for name, got in backward(s).items():
                if got is not None:
                    within(got, refs[name].reshape(got.shape), offs[name].reshape(got.shape), f"gradient of {name}")
    return ref, refs


STATES = [(1, F32), (3, BF16), (5, F32), (16, F32), (16, BF16), (20, BF16), (40, F32)]
SHAPES = [(1, 70), (5, 70), (8, 64), (16, 64), (40, 64), (8, 70), (40, 70), (700, 70)]      # steps, channels


@pytest.mark.parametrize("states,kind", STATES)
@pytest.mark.parametrize("steps,channels", SHAPES)
def test_infinite_inputs(steps, channels, states, kind):
    """An infinite x makes an infinite state, and so does an infinite step."""
    print(f"case inputs {steps} {channels} {states} {kind}", flush=True)
    far = channels - 1
    s = positive(3, steps, channels, states, kind, fall=0.05)
    s["x"][0, steps // 2, 3] = INF
    s["x"][0, steps - 1, far] = -INF
    ref, refs = check(s)
    assert np.isposinf(ref.out[0, steps // 2:, 3]).all() and np.isneginf(ref.last[0, far]).all() and np.isposinf(refs["a"][3]).all() == (steps > 1)
    s = positive(3, steps, channels, states, kind, fall=0.05)
    s["delta"][1, steps // 3, far] = INF
    ref, refs = check(s)
    assert np.isposinf(ref.out[1, steps // 3:, far]).all() and np.isposinf(refs["x"][1, steps // 3, far]) and np.isfinite(refs["x"]).sum() == refs["x"].size - 1


# fall: a chunk's steps take a state below what fp32 holds, one step does not
@pytest.mark.parametrize("states,kind", STATES)
@pytest.mark.parametrize("steps,fall", [(1, 5.0), (16, 20.0), (40, 0.5), (40, 20.0), (100, 20.0), (700, 0.5), (700, 20.0)])
def test_infinite_states_stay_infinite(steps, fall, states, kind):
    print(f"case states {steps} {fall} {states} {kind}", flush=True)
    s = positive(3, steps, 70, states, kind, fall=fall)
    s["h0"][0, 5] = INF
    s["h0"][1, 69, states - 1] = INF
    ref, refs = check(s)
    assert np.isposinf(ref.out[0, :, 5]).all() and np.isposinf(ref.out[1, :, 69]).all() and np.isposinf(refs["a"][69, states - 1])


@pytest.mark.parametrize("states,kind", STATES)
@pytest.mark.parametrize("steps,fall", [(1, 5.0), (8, 20.0), (16, 20.0), (40, 0.5), (40, 20.0), (700, 0.5), (700, 20.0)])
def test_infinite_gradients_stay_infinite(steps, fall, states, kind):
    print(f"case gradients {steps} {fall} {states} {kind}", flush=True)
    s = positive(3, steps, 70, states, kind, fall=fall)
    s["dlast"][0, 69] = INF
    s["dout"][1, steps // 2, 4] = INF
    s["dout"][2, steps - 1, 69] = INF
    _, refs = check(s)
    assert np.isposinf(refs["h0"][0, 69]).all() and np.isposinf(refs["x"][1, :steps // 2 + 1, 4]).all() and np.isposinf(refs["x"][2, :, 69]).all()


@pytest.mark.parametrize("states", [5, 16])
def test_channels_beside_an_infinite_one_keep_their_bits(states):
    s = positive(2, 700, 70, states, fall=2.0)
    before = (*forward(s), *(v for k, v in backward(s).items() if k not in ("b", "c")))
    s["x"][0, 100, 7], s["h0"][0, 7], s["dout"][0, 600, 7], s["dlast"][1, 7] = INF, INF, INF, INF
    after = (*forward(s), *(v for k, v in backward(s).items() if k not in ("b", "c")))
    for a, b in zip(before, after):
        if a is None:
            continue
        axis = list(a.shape).index(70)
        others = torch.tensor([c for c in range(70) if c != 7], device=a.device)
        assert torch.equal(a.index_select(axis, others), b.index_select(axis, others))
        assert not torch.isfinite(b.select(axis, 7)).all()


def test_infinite_states_by_many_waves_and_by_lengths():
    """Chunks of the longest kind, and beside the infinite sequences some that end before them.  (The infinite ones are whole: the definition's sums have zeros behind
    a sequence's end, and 64 bits make NaN of these and infinity too.)"""
    print("case many", flush=True)
    s = positive(400, 523, 66, 3, fall=1.0, lengths=[523 - i % 2 * i for i in range(400)])
    s["x"][4, 100, 65] = INF
    s["h0"][6, 2] = INF
    s["dout"][8, 300, 5] = INF
    s["dlast"][10, 65, 1] = INF
    check(s)


@pytest.mark.parametrize("states", [1, 5, 16, 20])
@pytest.mark.parametrize("steps", [16, 40])
def test_token_by_token_is_the_whole(steps, states):
    s = positive(2, steps, 37, states, fall=0.05)
    s["x"][0, steps // 2, 3], s["delta"][1, steps // 3, 36], s["h0"][0, 5] = INF, INF, INF
    with np.errstate(all="ignore"):
        ref = M.Scan(*(s[k] for k in ARGS), **{k: s[k] for k in OPTIONS})
    state = s["h0"].clone()
    for t in range(steps):
        of = lambda k: s[k][:, t:t + 1]
        out = torch.empty_like(of("x")).contiguous()
        B.scan_forward(of("x"), of("delta"), s["a"], of("b"), of("c"), out, d=s["d"], gate=of("gate"), h0=state, h_last=state)
        within(out, ref.out[:, t:t + 1], ref.out_off[:, t:t + 1], f"out {t}")
    within(state, ref.last, ref.last_off, "state")
