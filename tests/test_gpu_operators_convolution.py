"""The short causal convolution against its definition in 64 bits."""
import pytest
import torch

from paper_2010_16248_amd import binding as B
from tests import more_operators_plain as M
from tests.operators_plain import assert_within, f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def make(batch, steps, channels, width, kind, seed=0, bias=True, state=True, lengths=None):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)
    s = dict(x=r(batch, steps, channels).to(kind).to(DEV), weight=r(channels, width).to(DEV), bias=r(channels).to(DEV) if bias else None,
             state=r(batch, width - 1, channels).to(DEV) if state else None, dout=r(batch, steps, channels).to(kind).to(DEV),
             dlast=r(batch, width - 1, channels).to(DEV))
    s["lengths"] = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    return s


def forward(s, silu, out=None, last=None):
    out = torch.full_like(s["x"], 7.0) if out is None else out
    last = torch.full_like(s["dlast"], 7.0) if last is None else last
    B.convolution_forward(s["x"], s["weight"], out, bias=s["bias"], state=s["state"], last=last, lengths=s["lengths"], silu=silu)
    return out, last


def backward(s, silu, dlast=True, **kw):
    dx, dw = torch.full_like(s["x"], 7.0), torch.full_like(s["weight"], 7.0)
    db = torch.full_like(dw[:, 0], 7.0).contiguous()
    ds = torch.full_like(s["dlast"], 7.0)
    B.convolution_backward(s["x"], s["weight"], s["dout"], dx, dw, bias=s["bias"], grad_bias=db, state=s["state"],
                           grad_last=s["dlast"] if dlast else None, grad_state=ds, lengths=s["lengths"], silu=silu, **kw)
    return dx, dw, db, ds


def check(s, silu, dlast=True):
    (out, last), off = M.convolution(s["x"], s["weight"], s["bias"], s["state"], s["lengths"], silu)
    got, got_last = forward(s, silu)
    assert_within(got, out, off, "out")
    assert (f64(got_last) == last).all(), "last"
    refs, offs = M.convolution_gradients(s["x"], s["weight"], s["bias"], s["state"], s["lengths"], silu, s["dout"], s["dlast"] if dlast else None)
    for name, g, ref, bound in zip(("dx", "dw", "db", "dstate"), backward(s, silu, dlast), refs, offs):
        assert_within(g, ref, bound, name)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("width", [1, 2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("shape", [(1, 1, 1), (2, 3, 5), (3, 17, 8), (2, 130, 33)])
def test_widths_and_shapes(shape, width, kind):
    print(f"case {shape} {width} {kind}", flush=True)
    check(make(*shape, width, kind, bias=width % 2 == 0, state=width % 3 != 0), silu=width % 2 == 1)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("shape", [(1, 1500, 520), (5, 8, 1001), (70, 2, 64), (1, 9, 4100), (40, 300, 16), (3, 64, 257)])
def test_many_runs_and_blocks(shape, kind):
    print(f"case {shape} {kind}", flush=True)
    check(make(*shape, 4, kind), silu=True)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("width", [2, 4, 8])
def test_lengths_leave_what_lies_behind_alone(width, silu, kind):
    """Lengths of zero, below zero, shorter than the window and beyond the steps; what padded places hold plays no role."""
    lengths = [0, -3, 1, 2, 5, 40, 77, 99]
    s = make(8, 77, 19, width, kind, lengths=lengths)
    for i, n in enumerate(lengths):
        s["x"][i, max(n, 0):] = float("nan")
        s["dout"][i, max(n, 0):] = float("inf")
    print(f"case lengths {width} {silu} {kind}", flush=True)
    check(s, silu)


@pytest.mark.parametrize("kind", [F32, BF16])
def test_rows_apart(kind):
    """Inputs and outputs as columns of wider tensors, sequences interleaved."""
    print(f"case strides {kind}", flush=True)
    s = make(3, 41, 21, 4, kind)
    plain = (*forward(s, True), *backward(s, True))
    wide = torch.zeros(41, 3, 50, dtype=kind, device=DEV)
    x = wide.transpose(0, 1)[..., 3:24]
    x.copy_(s["x"])
    dout = torch.zeros(3, 41, 23, dtype=kind, device=DEV)[..., 1:22]
    dout.copy_(s["dout"])
    s.update(x=x, dout=dout)
    outs = torch.full((41, 3, 60), 9.0, dtype=kind, device=DEV)
    out, dx = outs.transpose(0, 1)[..., 5:26], outs.transpose(0, 1)[..., 30:51]
    last = torch.empty_like(s["dlast"])
    B.convolution_forward(x, s["weight"], out, bias=s["bias"], state=s["state"], last=last, silu=True)
    dw, db, ds = torch.empty_like(s["weight"]), torch.empty(21, device=DEV), torch.empty_like(last)
    B.convolution_backward(x, s["weight"], dout, dx, dw, bias=s["bias"], grad_bias=db, state=s["state"], grad_last=s["dlast"], grad_state=ds, silu=True)
    for a, b in zip(plain, (out, last, dx, dw, db, ds)):
        assert torch.equal(a, b)
    rest = torch.ones(60, dtype=torch.bool)
    rest[5:26] = rest[30:51] = False
    assert (outs[..., rest.to(DEV)] == 9.0).all()


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("width", [1, 3, 4])
def test_token_by_token_is_the_whole(width, kind):
    """The serving form, the state in one buffer, gives the bits of one call; so do pieces of any length."""
    s = make(3, 23, 37, width, kind)
    whole, last = forward(s, True)
    for pieces in ([1] * 23, [2, 1, 9, 11], [5, 18]):
        state, at = s["state"].clone(), 0
        for n in pieces:
            out = torch.empty_like(s["x"][:, at:at + n]).contiguous()
            B.convolution_forward(s["x"][:, at:at + n], s["weight"], out, bias=s["bias"], state=state, last=state, silu=True)
            assert torch.equal(out, whole[:, at:at + n])
            at += n
        assert torch.equal(state, last)


def test_states_in_place_of_sequences_shorter_than_the_window():
    s = make(4, 6, 5, 8, F32, lengths=[0, 2, 6, 3])
    _, last = forward(s, False)
    state = s["state"].clone()
    B.convolution_forward(s["x"], s["weight"], torch.empty_like(s["x"]), state=state, last=state, lengths=s["lengths"])
    assert torch.equal(state, last)


@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("channels", [3, 9, 35, 129, 257, 258, 513, 515, 1001, 2049])
def test_rows_that_end_in_a_part_of_a_pack(channels, kind):
    """The last channels alone, in a wave of their own and beside others; a state replaced and one left as it is."""
    print(f"case ends {channels} {kind}", flush=True)
    for steps in (1, 2, 40):
        s = make(3, steps, channels, 4, kind, seed=steps, lengths=[steps, 0, steps // 2])
        last, out = torch.full_like(s["state"], 7.0), torch.full_like(s["x"], 7.0)
        kw = dict(bias=s["bias"], lengths=s["lengths"], silu=True)
        B.convolution_forward(s["x"], s["weight"], out, state=s["state"], last=last, **kw)
        state, again = s["state"].clone(), torch.full_like(s["x"], 7.0)
        B.convolution_forward(s["x"], s["weight"], again, state=state, last=state, **kw)
        assert torch.equal(out, again) and torch.equal(last, state)
        one = channels - 1                    # the last channel for itself
        cut = lambda t: t[..., one:].contiguous()
        alone, end = torch.full_like(cut(out), 7.0), torch.full_like(cut(last), 7.0)
        B.convolution_forward(cut(s["x"]), s["weight"][one:].contiguous(), alone, state=cut(s["state"]), last=end, bias=s["bias"][one:].contiguous(),
                              lengths=s["lengths"], silu=True)
        assert torch.equal(alone, cut(out)) and torch.equal(end, cut(last))


def test_what_may_be_left_out():
    s = make(2, 9, 6, 4, F32, bias=False, state=False)
    check(s, True, dlast=False)
    dx, dw = torch.empty_like(s["x"]), torch.empty_like(s["weight"])
    B.convolution_forward(s["x"], s["weight"], torch.empty_like(s["x"]))
    B.convolution_backward(s["x"], s["weight"], s["dout"], dx, dw)
    refs, offs = M.convolution_gradients(s["x"], s["weight"], None, None, None, False, s["dout"], None)
    assert_within(dx, refs[0], offs[0], "dx")
    assert_within(dw, refs[1], offs[1], "dw")


def test_gradients_are_added():
    s = make(2, 50, 70, 3, F32)
    dx, dw, db, ds = backward(s, True)
    more_w, more_b = torch.randn_like(dw), torch.randn_like(db)
    w, b = more_w.clone(), more_b.clone()
    B.convolution_backward(s["x"], s["weight"], s["dout"], dx, w, bias=s["bias"], grad_bias=b, state=s["state"], grad_last=s["dlast"],
                           grad_state=ds, silu=True, accumulate=True)
    assert torch.equal(w, more_w + dw) and torch.equal(b, more_b + db)


@pytest.mark.parametrize("shape", [(0, 5, 3), (2, 0, 3), (0, 0, 3)])
def test_nothing_to_do(shape):
    s = make(*shape, 4, F32)
    out, last = forward(s, True)
    assert torch.equal(last, s["state"])
    dx, dw, db, ds = backward(s, True)
    assert not dw.any() and not db.any() and torch.equal(ds, s["dlast"])
    dw.fill_(3.0)
    B.convolution_backward(s["x"], s["weight"], s["dout"], dx, dw, accumulate=True)
    assert (dw == 3.0).all()


def test_the_same_bits_every_time():
    s = make(7, 900, 130, 4, BF16)
    first = (*forward(s, True), *backward(s, True))
    for _ in range(3):
        for a, b in zip(first, (*forward(s, True), *backward(s, True))):
            assert torch.equal(a, b)


@pytest.mark.parametrize("value", [-200.0, -90.0, -30.0, 30.0, 200.0])
def test_far_values(value):
    """SiLU where its exponential leaves the range of fp32."""
    s = make(1, 8, 4, 1, F32, state=False)
    s["x"].fill_(value)
    s["weight"].fill_(1.0)
    s["bias"].zero_()
    check(s, True)


def test_places_beyond_2_to_the_31():
    step = (1 << 30) + 8
    big = torch.zeros(2 * step + 64, dtype=BF16, device=DEV)
    s = make(1, 3, 40, 4, BF16)
    plain = (*forward(s, True), *backward(s, True))
    print("case large", flush=True)
    x = big.as_strided((1, 3, 40), (0, step, 1))
    x.copy_(s["x"])
    s["x"] = x
    out, last = forward(s, True, out=torch.empty(1, 3, 40, dtype=BF16, device=DEV))
    dx, dw = torch.empty(1, 3, 40, dtype=BF16, device=DEV), torch.empty_like(s["weight"])
    db, ds = torch.empty_like(s["bias"]), torch.empty_like(last)
    B.convolution_backward(x, s["weight"], s["dout"], dx, dw, bias=s["bias"], grad_bias=db, state=s["state"], grad_last=s["dlast"],
                           grad_state=ds, silu=True)
    for a, b in zip(plain, (out, last, dx, dw, db, ds)):
        assert torch.equal(a, b)
