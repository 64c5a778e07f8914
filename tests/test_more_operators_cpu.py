"""What the convolution, the scan and the log probabilities refuse, before anything is launched (CPU only: the pointers are never
followed), and the gradients' formulas in 64 bits against differences."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

from paper_2010_16248_amd import binding as B
from tests import more_operators_plain as M


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2010_16248_amd import build
        build.build(verbose=False)
    return B.load_library()


def at(i, off=0):
    return C.c_void_p(((i + 1) << 40) + off)


def refused(lib, rc, word, status=B.ACC_EINVAL):
    assert rc == status
    assert word in lib.accordion_operator_error().decode()


LARGE = 1 << 60


def pointers(n, **changes):
    """n pointers, some of them changed: to None, or by some bytes."""
    out = [at(i) for i in range(n)]
    for k, v in changes.items():
        i = int(k[1:])
        out[i] = v if v is None or isinstance(v, C.c_void_p) else at(i, v)
    return out


# ---- convolution ----------------------------------------------------------------------------------------

def convolution(**kw):
    args = dict(batch=2, steps=3, channels=4, width=4, type=0, silu=0, accumulate=0)
    args.update({f"{k}_{d}": v for k in ("x", "out", "grad_x") for d, v in (("batch", 12), ("step", 4))})
    args.update(kw)
    return B.acc_convolution(**args)


@pytest.mark.parametrize("change,word", [
    (dict(batch=-1), "batch"), (dict(batch=65536), "batch"), (dict(steps=-1), "steps"), (dict(steps=2 ** 31), "steps"),
    (dict(channels=0), "channels"), (dict(channels=2 ** 23 + 1), "channels"), (dict(width=0), "width"), (dict(width=9), "width"),
    (dict(type=2), "type"), (dict(silu=2), "silu"), (dict(accumulate=-1), "accumulate"), (dict(x_step=-4), "stride"), (dict(x_batch=2 ** 41), "stride"),
])
def test_convolution_configurations(lib, change, word):
    cfg, n = convolution(**change), C.c_size_t(0)
    refused(lib, lib.accordion_convolution_forward(C.byref(cfg), *pointers(7), None), word)
    refused(lib, lib.accordion_convolution_backward(C.byref(cfg), *pointers(12), LARGE, None), word)
    refused(lib, lib.accordion_convolution_workspace_bytes(C.byref(cfg), C.byref(n)), word)


def test_convolution_rows_that_are_written(lib):
    for change in (dict(out_step=3), dict(out_batch=11)):
        refused(lib, lib.accordion_convolution_forward(C.byref(convolution(**change)), *pointers(7), None), "overlap")
    for change in (dict(grad_x_step=3), dict(grad_x_batch=0)):
        refused(lib, lib.accordion_convolution_backward(C.byref(convolution(**change)), *pointers(12), LARGE, None), "overlap")


def test_convolution_pointers(lib):
    cfg, n = convolution(), C.c_size_t(0)
    fwd = lambda **k: lib.accordion_convolution_forward(C.byref(cfg), *pointers(7, **k), None)
    refused(lib, lib.accordion_convolution_forward(None, *pointers(7), None), "NULL")
    refused(lib, lib.accordion_convolution_workspace_bytes(C.byref(cfg), None), "NULL")
    for i in (0, 1, 5):
        refused(lib, fwd(**{f"p{i}": None}), "NULL")
    for i in range(7):
        refused(lib, fwd(**{f"p{i}": 1}), "aligned")
    refused(lib, fwd(p5=at(0)), "overlaps")
    refused(lib, fwd(p6=at(1)), "overlaps")
    refused(lib, fwd(p6=at(3, 16)), "overlaps")                  # a state that is last in part
    assert lib.accordion_convolution_workspace_bytes(C.byref(cfg), C.byref(n)) == B.ACC_OK and n.value > 0
    bwd = lambda size=n.value, **k: lib.accordion_convolution_backward(C.byref(cfg), *pointers(12, **k), size, None)
    for i in (0, 1, 5, 7, 8):
        refused(lib, bwd(**{f"p{i}": None}), "NULL")
    refused(lib, bwd(p11=None), "workspace")
    for i in range(11):
        refused(lib, bwd(**{f"p{i}": 1}), "aligned")
    refused(lib, bwd(p11=128), "aligned")
    refused(lib, bwd(size=n.value - 1), "workspace", B.ACC_ENOSPACE)
    for i in (7, 8, 9, 10, 11):
        refused(lib, bwd(**{f"p{i}": at(5)}), "overlaps")
    refused(lib, bwd(p9=at(8)), "overlaps")


# ---- scan -----------------------------------------------------------------------------------------------

def scan(**kw):
    args = dict(batch=2, steps=30, channels=4, states=3, groups=2, type=0, softplus=0, accumulate=0)
    args.update({f"{k}_{d}": v for k in ("x", "delta", "gate", "out", "grad_x", "grad_delta", "grad_gate") for d, v in (("batch", 120), ("step", 4))})
    args.update({f"{k}_{d}": v for k in ("b", "c", "grad_b", "grad_c") for d, v in (("batch", 180), ("step", 6))})
    args.update(kw)
    return B.acc_scan(**args)


@pytest.mark.parametrize("change,word", [
    (dict(batch=-1), "batch"), (dict(batch=65536), "batch"), (dict(steps=-1), "steps"), (dict(steps=2 ** 31), "steps"),
    (dict(channels=0), "channels"), (dict(channels=2 ** 24 + 2), "channels"), (dict(states=0), "states"), (dict(states=65), "states"),
    (dict(groups=0), "groups"), (dict(groups=3), "groups"), (dict(type=-1), "type"), (dict(softplus=2), "softplus"), (dict(accumulate=2), "accumulate"),
    (dict(delta_step=-4), "stride"), (dict(b_batch=2 ** 41), "stride"), (dict(c_step=-1), "stride"), (dict(gate_step=-1), "stride"),
])
def test_scan_configurations(lib, change, word):
    cfg, n = scan(**change), C.c_size_t(0)
    refused(lib, lib.accordion_scan_forward(C.byref(cfg), *pointers(13), LARGE, None), word)
    refused(lib, lib.accordion_scan_backward(C.byref(cfg), *pointers(22), LARGE, None), word)
    for backward in (0, 1):
        refused(lib, lib.accordion_scan_workspace_bytes(C.byref(cfg), backward, C.byref(n)), word)


def test_scan_rows_that_are_written(lib):
    for change in (dict(out_step=3), dict(out_batch=100)):
        refused(lib, lib.accordion_scan_forward(C.byref(scan(**change)), *pointers(13), LARGE, None), "overlap")
    for change in (dict(grad_x_step=3), dict(grad_delta_batch=0), dict(grad_b_step=5), dict(grad_c_batch=1), dict(grad_gate_step=0)):
        refused(lib, lib.accordion_scan_backward(C.byref(scan(**change)), *pointers(22), LARGE, None), "overlap")
    refused(lib, lib.accordion_scan_backward(C.byref(scan(grad_b_step=-1)), *pointers(22), LARGE, None), "stride")


def test_scan_sizes(lib):
    n = C.c_size_t(0)
    refused(lib, lib.accordion_scan_workspace_bytes(C.byref(scan()), 2, C.byref(n)), "backward")
    refused(lib, lib.accordion_scan_workspace_bytes(C.byref(scan()), 0, None), "NULL")
    long = scan(steps=2 ** 21 + 1, batch=1)
    assert lib.accordion_scan_workspace_bytes(C.byref(long), 0, C.byref(n)) == B.ACC_OK
    refused(lib, lib.accordion_scan_workspace_bytes(C.byref(long), 1, C.byref(n)), "steps")
    many = scan(steps=2 ** 21, batch=60000, x_batch=2 ** 30, delta_batch=2 ** 30, gate_batch=2 ** 30, out_batch=2 ** 30)
    refused(lib, lib.accordion_scan_workspace_bytes(C.byref(many), 0, C.byref(n)), "out of range")
    most = scan(batch=65535, steps=2 ** 21, channels=2 ** 20, groups=2 ** 20, states=64)        # products beyond 63 bits
    for backward in (0, 1):
        refused(lib, lib.accordion_scan_workspace_bytes(C.byref(most), backward, C.byref(n)), "out of range")


def test_scan_pointers(lib):
    cfg, n = scan(), C.c_size_t(0)
    refused(lib, lib.accordion_scan_forward(None, *pointers(13), LARGE, None), "NULL")
    assert lib.accordion_scan_workspace_bytes(C.byref(cfg), 0, C.byref(n)) == B.ACC_OK and n.value > 0
    fwd = lambda size=n.value, **k: lib.accordion_scan_forward(C.byref(cfg), *pointers(13, **k), size, None)
    for i in (0, 1, 2, 3, 4, 10):
        refused(lib, fwd(**{f"p{i}": None}), "NULL")
    for i in range(12):
        refused(lib, fwd(**{f"p{i}": 1}), "aligned")
    refused(lib, fwd(p12=None), "workspace")
    refused(lib, fwd(p12=128), "aligned")
    refused(lib, fwd(size=n.value - 1), "workspace", B.ACC_ENOSPACE)
    for i in (10, 11, 12):
        refused(lib, fwd(**{f"p{i}": at(3)}), "overlaps")
    refused(lib, fwd(p11=at(8, 16)), "overlaps")                 # a state that is last in part
    assert lib.accordion_scan_workspace_bytes(C.byref(cfg), 1, C.byref(n)) == B.ACC_OK and n.value > 0
    bwd = lambda size=n.value, **k: lib.accordion_scan_backward(C.byref(cfg), *pointers(22, **k), size, None)
    for i in (0, 1, 2, 3, 4, 10, 12, 13, 14, 15, 16):
        refused(lib, bwd(**{f"p{i}": None}), "NULL")
    refused(lib, bwd(p6=None), "together")
    refused(lib, bwd(p18=None), "together")
    refused(lib, bwd(p5=None), "needs d_dev")
    refused(lib, bwd(p7=None), "needs delta_bias_dev")
    for i in range(21):
        refused(lib, bwd(**{f"p{i}": 1}), "aligned")
    refused(lib, bwd(size=n.value - 1), "workspace", B.ACC_ENOSPACE)
    for i in (12, 13, 14, 15, 16, 17, 18, 19, 20, 21):
        refused(lib, bwd(**{f"p{i}": at(10)}), "overlaps")
    refused(lib, bwd(p16=at(15)), "overlaps")


def test_scan_backward_asks_for_no_workspace_without_sequences(lib):
    n = C.c_size_t(7)
    assert lib.accordion_scan_workspace_bytes(C.byref(scan(batch=0)), 1, C.byref(n)) == B.ACC_OK and n.value == 0


# ---- log probabilities ----------------------------------------------------------------------------------

def logprob(**kw):
    args = dict(rows=3, vocab=100, logits_stride=100, grad_stride=100, index_bits=64, type=0, top=2)
    args.update(kw)
    return B.acc_logprob(**args)


@pytest.mark.parametrize("change,word", [
    (dict(rows=-1), "rows"), (dict(rows=2 ** 28 + 1), "rows"), (dict(vocab=0), "vocab"), (dict(vocab=2 ** 22 + 1), "vocab"), (dict(index_bits=8), "index_bits"),
    (dict(type=2), "type"), (dict(top=-1), "top"), (dict(top=65), "top"), (dict(vocab=1), "top"), (dict(logits_stride=99), "logits_stride"),
])
def test_logprob_configurations(lib, change, word):
    cfg, n = logprob(**change), C.c_size_t(0)
    refused(lib, lib.accordion_logprob_forward(C.byref(cfg), *pointers(8), LARGE, None), word)
    refused(lib, lib.accordion_logprob_backward(C.byref(cfg), *pointers(7), None), word)
    refused(lib, lib.accordion_logprob_workspace_bytes(C.byref(cfg), C.byref(n)), word)


def test_logprob_pointers(lib):
    cfg, n = logprob(vocab=100000, logits_stride=100000, grad_stride=100000), C.c_size_t(0)
    refused(lib, lib.accordion_logprob_forward(None, *pointers(8), LARGE, None), "NULL")
    refused(lib, lib.accordion_logprob_workspace_bytes(C.byref(cfg), None), "NULL")
    assert lib.accordion_logprob_workspace_bytes(C.byref(cfg), C.byref(n)) == B.ACC_OK and n.value > 0
    fwd = lambda size=n.value, **k: lib.accordion_logprob_forward(C.byref(cfg), *pointers(8, **k), size, None)
    for i in (0, 1, 5, 6):
        refused(lib, fwd(**{f"p{i}": None}), "NULL" if i != 1 else "needs targets_dev")
    for i in range(7):
        refused(lib, fwd(**{f"p{i}": 1}), "aligned")
    refused(lib, fwd(p7=128), "aligned")
    refused(lib, fwd(size=n.value - 1), "workspace", B.ACC_ENOSPACE)
    for i in (2, 3, 4, 5, 6, 7):
        refused(lib, fwd(**{f"p{i}": at(1)}), "overlaps")
    bwd = lambda **k: lib.accordion_logprob_backward(C.byref(cfg), *pointers(7, **k), None)
    for i in (0, 2, 6):
        refused(lib, bwd(**{f"p{i}": None}), "NULL")
    refused(lib, bwd(p1=None), "needs targets_dev")
    refused(lib, bwd(p4=None), "needs entropy_dev")
    for i in range(7):
        refused(lib, bwd(**{f"p{i}": 1}), "aligned")
    refused(lib, bwd(p6=at(0, 4)), "overlaps")
    refused(lib, bwd(p6=at(3)), "overlaps")
    other = logprob(grad_stride=101)                             # in place needs one stride
    refused(lib, lib.accordion_logprob_backward(C.byref(other), *pointers(7, p6=at(0)), None), "overlaps")
    refused(lib, lib.accordion_logprob_backward(C.byref(logprob(grad_stride=99)), *pointers(7), None), "grad_stride")


# ---- what the binding sees ------------------------------------------------------------------------------

def test_tensors_that_do_not_fit_are_refused():
    z = lambda *s, k=torch.float32: torch.zeros(*s, dtype=k)
    x, w = z(2, 5, 4), z(4, 3)
    with pytest.raises(ValueError, match="batch x steps"):
        B.convolution_forward(z(5, 4), w, z(5, 4))
    with pytest.raises(ValueError, match="width"):
        B.convolution_forward(x, z(3), z(2, 5, 4))
    with pytest.raises(ValueError, match="weight"):
        B.convolution_forward(x, z(5, 3), z(2, 5, 4))
    with pytest.raises(ValueError, match="out must be"):
        B.convolution_forward(x, w, z(2, 5, 4, k=torch.bfloat16))
    with pytest.raises(ValueError, match="contiguous"):
        B.convolution_forward(x, w, z(2, 4, 5).transpose(1, 2))
    with pytest.raises(ValueError, match="state"):
        B.convolution_forward(x, w, z(2, 5, 4), state=z(2, 3, 4))
    with pytest.raises(ValueError, match="lengths"):
        B.convolution_forward(x, w, z(2, 5, 4), lengths=z(2, k=torch.int64))
    with pytest.raises(ValueError, match="grad_x"):
        B.convolution_backward(x, w, x, z(2, 5, 5), z(4, 3))
    with pytest.raises(ValueError, match="grad_bias"):
        B.convolution_backward(x, w, x, z(2, 5, 4), z(4, 3), grad_bias=z(3))
    with pytest.raises(ValueError, match="one GPU"):
        B.convolution_forward(x, w, z(2, 5, 4))
    a, b = z(4, 6), z(2, 5, 1, 6)
    with pytest.raises(ValueError, match="channels x states"):
        B.scan_forward(x, x, z(4), b, b, z(2, 5, 4))
    with pytest.raises(ValueError, match="groups"):
        B.scan_forward(x, x, a, z(2, 6), b, z(2, 5, 4))
    with pytest.raises(ValueError, match="b must be"):
        B.scan_forward(x, x, a, z(2, 5, 1, 5), b, z(2, 5, 4))
    with pytest.raises(ValueError, match="c must be"):
        B.scan_forward(x, x, a, b, z(2, 5, 6), z(2, 5, 4))
    with pytest.raises(ValueError, match="c: the elements"):
        B.scan_forward(x, x, a, b, z(2, 5, 1, 12)[..., ::2], z(2, 5, 4))
    with pytest.raises(ValueError, match="gate must be"):
        B.scan_forward(x, x, a, b, b, z(2, 5, 4), gate=z(2, 5, 4, k=torch.bfloat16))
    with pytest.raises(ValueError, match="delta must be"):
        B.scan_forward(x, z(2, 5, 3), a, b, b, z(2, 5, 4))
    with pytest.raises(ValueError, match="h0"):
        B.scan_forward(x, x, a, b, b, z(2, 5, 4), h0=z(2, 4, 5))
    with pytest.raises(ValueError, match="go together"):
        B.scan_backward(x, x, a, b, b, x, z(2, 5, 4), z(2, 5, 4), z(4, 6), z(2, 5, 1, 6), z(2, 5, 1, 6), gate=x)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        h = x.half()
        B.scan_forward(h, h, a, b.half(), b.half(), h.clone())
    logits, ids = z(3, 10), z(3, k=torch.int64)
    with pytest.raises(ValueError, match="go together"):
        B.logprob_forward(logits, ids, z(3), top_ids=z(3, 2, k=torch.int64))
    with pytest.raises(ValueError, match="needs targets"):
        B.logprob_forward(logits, None, z(3))
    with pytest.raises(ValueError, match="int32 or int64"):
        B.logprob_forward(logits, z(3), z(3))
    with pytest.raises(ValueError, match="one per row"):
        B.logprob_forward(logits, z(4, k=torch.int64), z(3))
    with pytest.raises(ValueError, match="of targets' type"):
        B.logprob_forward(logits, ids, z(3), top_logprobs=z(3, 2), top_ids=z(3, 2, k=torch.int32))
    with pytest.raises(ValueError, match="lse"):
        B.logprob_forward(logits, ids, z(3), lse=z(2))
    with pytest.raises(ValueError, match="fit together"):
        B.logprob_backward(logits, ids, z(3), z(3), z(3, 11))


# ---- the gradients' formulas against differences --------------------------------------------------------

def _differences(value, tensor, grad, seed):
    """value's central difference along a random direction of tensor, against the gradient's part along it: the third derivative's term
    is of the step's square, 1e-10, and the rounding 1e-16 / 1e-5."""
    step = 1e-5
    way = np.random.default_rng(seed).standard_normal(tensor.shape)
    keep = tensor.clone()
    tensor += torch.from_numpy(step * way)
    up = value()
    tensor.copy_(keep - torch.from_numpy(step * way))
    down = value()
    tensor.copy_(keep)
    ref, got = (up - down) / (2 * step), (grad * way).sum()
    assert abs(ref - got) <= 1e-7 * (1 + abs(ref)), (ref, got)


@pytest.mark.parametrize("silu", [False, True])
def test_convolution_gradients_follow_differences(silu):
    gen = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    x, w, b, state, dout, dlast = r(3, 6, 4), r(4, 3), r(4), r(3, 2, 4), r(3, 6, 4), r(3, 2, 4)
    lengths = torch.tensor([6, 1, 4])

    def value():
        (out, last), _ = M.convolution(x, w, b, state, lengths, silu)
        return (out * dout.numpy()).sum() + (last * dlast.numpy()).sum()

    grads, _ = M.convolution_gradients(x, w, b, state, lengths, silu, dout, dlast)
    for i, (t, g) in enumerate(zip((x, w, b, state), grads)):
        _differences(value, t, g, i)


@pytest.mark.parametrize("soft,gated", [(True, True), (False, True), (True, False)])
def test_scan_gradients_follow_differences(soft, gated):
    gen = torch.Generator().manual_seed(4)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    t = dict(x=r(2, 7, 4), delta=0.3 * r(2, 7, 4), a=-r(4, 3).exp(), b=r(2, 7, 2, 3), c=r(2, 7, 2, 3), d=r(4), gate=r(2, 7, 4) if gated else None,
             delta_bias=0.1 * r(4), h0=r(2, 4, 3))
    dout, dlast, lengths = r(2, 7, 4), r(2, 4, 3), torch.tensor([7, 3])

    def value():
        s = M.Scan(softplus=soft, lengths=lengths, **t)
        return (s.out * dout.numpy()).sum() + (s.last * dlast.numpy()).sum()

    grads, _ = M.Scan(softplus=soft, lengths=lengths, **t).gradients(dout, dlast)
    for i, (k, v) in enumerate(t.items()):
        if v is not None:
            _differences(value, v, grads[k].reshape(v.shape), i)


def test_logprob_gradients_follow_differences():
    gen = torch.Generator().manual_seed(5)
    logits, g, ge = (torch.randn(*s, generator=gen, dtype=torch.float64) for s in ((4, 9), (4,), (4,)))
    ids = torch.tensor([0, 8, -1, 3])

    def value():
        _, lp, entropy, *_ = M.logprob(logits)
        chosen = np.where(ids.numpy() >= 0, np.take_along_axis(lp, np.maximum(ids.numpy(), 0)[:, None], 1)[:, 0], 0)
        return (g.numpy() * chosen).sum() + (ge.numpy() * entropy).sum()

    lse, _, entropy, *_ = M.logprob(logits)
    grad, _ = M.logprob_gradient(logits, ids, torch.from_numpy(lse), g, torch.from_numpy(entropy), ge)
    _differences(value, logits, grad, 0)
