"""AdamW over many tensors: bit for bit against the step in fp32, and against the textbook step in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2010_16248_amd import binding as B
from tests import operators_plain as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF = torch.float32, torch.bfloat16
ARGS = dict(betas=(0.9, 0.95), eps=1e-8)

# one element, parts of blocks, whole blocks, tiles, an empty tensor among others
SIZES = [[1], [255], [256], [257], [2048], [2049], [3, 0, 1000, 256, 5, 4097, 1, 30001], [7] * 150 + [5000]]


def _data(sizes, w_type, g_type, seed):
    gen = torch.Generator().manual_seed(seed)
    weights = [torch.randn(n, generator=gen).to(w_type).to(DEV) for n in sizes]
    grads = [(torch.randn(n, generator=gen) * math.exp(float(torch.randn(1, generator=gen)) * 2 - 6)).to(g_type).to(DEV) for n in sizes]
    decay = [0.1 * (i % 3) for i in range(len(sizes))]
    return weights, grads, decay


def _offsets(sizes, bits):
    at, out = 0, []
    for n in sizes:
        out.append(at)
        at += n if bits == 32 else -(-n // 256) * 256
    return out


@pytest.mark.parametrize("g_type", [F32, BF])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", SIZES)
def test_steps_are_those_of_fp32_bit_for_bit(sizes, bits, g_type):
    print(f"case adamw {len(sizes)} tensors {sum(sizes)} {bits} {g_type}", flush=True)
    weights, _, decay = _data(sizes, F32, g_type, 1)
    copies = [None if i % 4 == 3 else torch.full((n,), 9.0, dtype=BF, device=DEV) for i, n in enumerate(sizes)]
    scale = torch.tensor([0.37], device=DEV)
    state = B.adamw_state(sizes, bits)
    ref_w = [w.cpu().numpy().copy() for w in weights]
    ref_m, ref_v = [np.zeros(n, np.float32) for n in sizes], [np.zeros(n, np.float32) for n in sizes]
    for step in range(1, 4):
        _, grads, _ = _data(sizes, F32, g_type, 10 + step)
        B.adamw_step(weights, grads, state, 0.01 * step, step, weight_decay=decay, copies=copies, grad_scale=scale if step > 1 else None,
                     **ARGS)
        for i, at in enumerate(_offsets(sizes, bits)):
            n = sizes[i]
            w, m, v, root = P.adamw32(ref_w[i], grads[i].float().cpu().numpy(), ref_m[i], ref_v[i], 0.01 * step, step, ARGS["betas"],
                                      ARGS["eps"], decay[i], None if step == 1 else 0.37)
            ref_w[i] = w
            assert np.array_equal(weights[i].cpu().numpy().view(np.uint32), w.view(np.uint32)), f"step {step} tensor {i}: weights"
            if copies[i] is not None:
                assert torch.equal(copies[i].cpu(), torch.from_numpy(w).to(BF)), f"step {step} tensor {i}: copy"
            if bits == 32:
                ref_m[i], ref_v[i] = m, v
                assert np.array_equal(state[0][at:at + n].cpu().numpy().view(np.uint32), m.view(np.uint32)), f"step {step} tensor {i}: m"
                assert np.array_equal(state[1][at:at + n].cpu().numpy().view(np.uint32), v.view(np.uint32)), f"step {step} tensor {i}: v"
            else:
                blocks = -(-n // 256)
                for k, (value, root_) in enumerate(((m, False), (root, True))):
                    codes, scales = P.encode(value, root_)
                    got = state[k].view(torch.uint8)[at:at + 256 * blocks].cpu().numpy()
                    got_scale = state[2 + k][at // 256:at // 256 + blocks].cpu().numpy()
                    assert np.array_equal(got, codes), f"step {step} tensor {i}: codes {k}"
                    assert np.array_equal(got_scale.view(np.uint32), scales.view(np.uint32)), f"step {step} tensor {i}: scales {k}"
                    held = P.decode(codes, scales)[:n]
                    if k == 0:
                        ref_m[i] = held
                    else:
                        ref_v[i] = held * held


@pytest.mark.parametrize("bits", [32, 8])
def test_against_the_textbook_in_64_bits(bits):
    sizes, lr = [5000, 700], 3e-3
    weights, _, _ = _data(sizes, F32, F32, 3)
    state = B.adamw_state(sizes, bits)
    ref = [(w.double().cpu().numpy(), np.zeros(n), np.zeros(n)) for w, n in zip(weights, sizes)]
    for step in range(1, 6):
        _, grads, _ = _data(sizes, F32, F32, 20 + step)
        if bits == 8:        # the moments as the state holds them
            for i, at in enumerate(_offsets(sizes, 8)):
                n, blocks = sizes[i], -(-sizes[i] // 256)
                held = [P.decode(state[k].view(torch.uint8)[at:at + 256 * blocks].cpu().numpy(),
                                 state[2 + k][at // 256:at // 256 + blocks].cpu().numpy())[:n].astype(np.float64) for k in (0, 1)]
                ref[i] = (ref[i][0], held[0], held[1] ** 2)
        before = [r[0].copy() for r in ref]
        B.adamw_step(weights, grads, state, lr, step, weight_decay=0.1, **ARGS)
        for i in range(2):
            ref[i] = P.adamw64(ref[i][0], grads[i].cpu().numpy(), ref[i][1], ref[i][2], lr, step, ARGS["betas"], ARGS["eps"], 0.1)
            # m carries five roundings a step, v as many, the quotient six more; w two of its own; five steps of that
            move = np.abs(ref[i][0] - before[i])
            bound = 5 * P.U * (4 * np.abs(ref[i][0]) + 40 * (move + lr * 0.1 * np.abs(before[i])) + 40 * lr)
            P.assert_within(weights[i], ref[i][0], bound, f"step {step}: weights")


def test_bf16_weights():
    sizes = [300, 4096, 33]
    weights, grads, decay = _data(sizes, BF, BF, 4)
    start = [w.float().cpu().numpy() for w in weights]
    state = B.adamw_state(sizes, 32)
    B.adamw_step(weights, grads, state, 0.1, 1, weight_decay=decay, **ARGS)
    for w, w0, g, d in zip(weights, start, grads, decay):
        zero = np.zeros(len(w0), np.float32)
        ref = P.adamw32(w0, g.float().cpu().numpy(), zero, zero, 0.1, 1, ARGS["betas"], ARGS["eps"], d)[0]
        assert torch.equal(w.cpu(), torch.from_numpy(ref).to(BF))


def test_layers_of_a_flat_buffer_leave_the_gaps():
    flat, grad = torch.randn(5000, device=DEV), torch.randn(5000, device=DEV)
    spans = [(3, 1000), (1005, 17), (1500, 3001)]
    before = flat.clone()
    state = B.adamw_state([n for _, n in spans], 8)
    B.adamw_step([flat[a:a + n] for a, n in spans], [grad[a:a + n] for a, n in spans], state, 0.1, 1)
    inside = torch.zeros(5000, dtype=torch.bool, device=DEV)
    for a, n in spans:
        inside[a:a + n] = True
    assert torch.equal(flat[~inside], before[~inside]) and (flat[inside] != before[inside]).all()


def test_small_second_moments_keep_a_code_and_tiny_blocks_are_zero():
    n = 512
    g = torch.full((n,), 1.0, device=DEV)
    g[1:256] = 1e-6                     # sqrt(v) a millionth of the block's largest: below half the smallest code
    g[5] = 0.0
    g[256:] = 1e-36                     # a block below 2^-100
    w = [torch.zeros(n, device=DEV)]
    state = B.adamw_state([n], 8)
    B.adamw_step(w, [g], state, 1e-3, 1, **ARGS)
    codes = state[1].view(torch.uint8)
    assert codes[0] == 0x7e and (codes[1:5] == 1).all() and codes[5] == 0 and (codes[6:256] == 1).all() and (codes[256:] == 0).all()
    assert state[2][1] == 0 and state[3][1] == 0
    B.adamw_step(w, [g], state, 1e-3, 2, **ARGS)
    assert w[0].isfinite().all() and w[0].abs().max() <= 2.1e-3


@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_what_is_not_finite_spoils_its_element_or_its_block(value):
    n = 700
    for bits, spoiled in ((32, slice(300, 301)), (8, slice(256, 512))):
        w, g = [torch.ones(n, device=DEV)], torch.full((n,), 0.5, device=DEV)
        g[300] = value
        state = B.adamw_state([n], bits)
        B.adamw_step(w, [g], state, 0.1, 1)
        B.adamw_step(w, [torch.full((n,), 0.5, device=DEV)], state, 0.1, 2)
        bad = torch.zeros(n, dtype=torch.bool, device=DEV)
        bad[spoiled] = True
        assert torch.equal(w[0].isnan(), bad)


def test_nothing_to_do():
    state = B.adamw_state([], 8)
    B.adamw_step([], [], state, 0.1, 1)
    empty = [torch.empty(0, device=DEV)]
    B.adamw_step(empty, empty, B.adamw_state([0], 32), 0.1, 1)
