"""Operators on slices of one buffer that lie in one another's range without sharing an element."""
import pytest
import torch

from paper_2010_16248_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("time_first", [False, True])
@pytest.mark.parametrize("steps", [1, 5, 300])
def test_steps_of_one_buffer(steps, time_first):
    """Inputs and results lie behind one another along the time of one buffer (or, time first, along its batch)."""
    print(f"case slices {steps} {time_first}", flush=True)
    batch, channels = 3, 70
    gen = torch.Generator().manual_seed(steps)
    r = lambda *s: torch.randn(*s, generator=gen).to(DEV)
    gate, x, dout, h0 = r(batch, steps, channels), r(batch, steps, channels), r(batch, steps, channels), r(batch, channels)
    if time_first:
        whole = torch.full((steps, 4 * batch, channels), 4.0, device=DEV)
        parts = [whole[:, k * batch:(k + 1) * batch].transpose(0, 1) for k in range(4)]
    else:
        whole = torch.full((batch, 4 * steps, channels), 4.0, device=DEV)
        parts = [whole[:, k * steps:(k + 1) * steps] for k in range(4)]
    v, out, dgate, dinput = parts
    v.copy_(x)
    plain, d1, d2 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    B.recurrence_forward(gate, x, plain, h0=h0)
    B.recurrence_forward(gate, v, out, h0=h0)
    assert torch.equal(out, plain) and torch.equal(v, x) and dgate.eq(4).all()
    B.recurrence_backward(gate, x, plain, dout, d1, d2, h0=h0)
    B.recurrence_backward(gate, v, out, dout, dgate, dinput, h0=h0)
    assert torch.equal(dgate, d1) and torch.equal(dinput, d2) and torch.equal(v, x) and torch.equal(out, plain)


def test_steps_that_are_shared_are_refused():
    whole = torch.zeros(3, 11, 70, device=DEV)
    gate = torch.zeros(3, 5, 70, device=DEV)
    for out in (whole[:, 4:9], whole[:, :5], whole.as_strided((3, 5, 70), (770, 70, 1), 4 * 70 + 35)):
        with pytest.raises(B.AccordionError) as err:
            B.recurrence_forward(gate, whole[:, :5], out)
        assert err.value.status == B.ACC_EINVAL
    # the last sequence's results end beyond the next one's inputs
    with pytest.raises(B.AccordionError) as err:
        B.recurrence_forward(gate[:2], whole[:2, :5], whole[:2, 7:11].as_strided((2, 5, 70), (770, 70, 1), 7 * 70))
    assert err.value.status == B.ACC_EINVAL


def test_adamw_tensors_between_one_another():
    """Weights, gradients and copies that take turns in one buffer, in any order, gradients that share memory, tensors without elements."""
    sizes = [100, 0, 7, 256, 1, 1000]
    gen = torch.Generator().manual_seed(1)
    apart = [torch.randn(n, generator=gen).to(DEV) for n in sizes]
    shared = torch.randn(1200, generator=gen).to(DEV)
    grads = [shared[3 * i:3 * i + n] for i, n in enumerate(sizes)]
    whole = torch.full((sum(sizes) * 3 + 64,), 4.0, device=DEV)
    weights, own, copies, at = [None] * 6, [None] * 6, [None] * 6, 0
    for i in (3, 0, 5, 1, 4, 2):
        n = sizes[i]
        copies[i] = whole[at:at + (n + 1) // 2].view(torch.bfloat16)[:n]
        at += (n + 1) // 2
        own[i], at = whole[at:at + n], at + n
        weights[i], at = whole[at:at + n], at + n
        own[i].copy_(grads[i]), weights[i].copy_(apart[i])
    B.adamw_step(apart, grads, B.adamw_state(sizes, 32, DEV), 0.1, 1, weight_decay=0.1)
    B.adamw_step(weights, own, B.adamw_state(sizes, 32, DEV), 0.1, 1, weight_decay=0.1, copies=copies)
    for i in range(6):
        assert torch.equal(weights[i], apart[i]) and torch.equal(copies[i], apart[i].bfloat16()) and torch.equal(own[i], grads[i])
    with pytest.raises(B.AccordionError) as err:
        B.adamw_step([apart[5], apart[5]], [grads[5], grads[5]], B.adamw_state([1000, 1000], 32, DEV), 0.1, 1)
    assert err.value.status == B.ACC_EINVAL
