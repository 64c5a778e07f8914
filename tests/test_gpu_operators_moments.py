"""AdamW's moments in 8 bits over thousands of steps: they follow the averages that they hold, where the gradients' sizes change too."""
import numpy as np
import pytest
import torch

from paper_2010_16248_amd import binding as B
from tests import operators_plain as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
N = 256 * 16
KEY = {"m": 0x6A09E667, "v": 0xBB67AE85}


def _held(state):
    """m and sqrt(v) as the state holds them."""
    return [(state[k].float().view(-1, 256) * state[2 + k][:, None]).view(-1) for k in (0, 1)]


def _follow(gradients, betas, steps, dither=False):
    """(held m, held sqrt(v), and both in 64 bits without any rounding) after the steps."""
    state = B.adamw_state([N], 8, DEV)
    weights = [torch.zeros(N, device=DEV)]
    m, v = (torch.zeros(N, dtype=torch.float64, device=DEV) for _ in range(2))
    for step in range(1, steps + 1):
        g = gradients(step)
        B.adamw_step(weights, [g], state, 1e-3, step, betas=betas, **(dict(dither=True) if dither else {}))
        g = g.double()
        m.mul_(betas[0]).add_(g, alpha=1 - betas[0])
        v.mul_(betas[1]).add_(g * g, alpha=1 - betas[1])
    assert weights[0].isfinite().all()
    return (*_held(state), m, v.sqrt())


# Neighbouring codes are up to an eighth of their value apart.  Whatever the rounding, single elements are off by about that, by
# a few of them where an average remembers hundreds of roundings; the median over 2048 elements has to be right to one spacing.
SPACING = 1 / 8


def _assert_follows(held, true, what):
    ratio = (held.double() / true).sort().values
    low, mid, high = (float(ratio[int(len(ratio) * q)]) for q in (0.05, 0.5, 0.95))
    print(f"{what}: {low:.3f} {mid:.3f} {high:.3f}", flush=True)
    assert abs(mid - 1) <= SPACING, what
    assert low >= 0.5 and high <= 2.0, what


@pytest.mark.parametrize("beta2", [0.95, 0.98, 0.999])
@pytest.mark.parametrize("change", [1.0, 0.1, 3.0])
def test_second_moments_follow_gradients_that_change(beta2, change):
    print(f"case moments v {beta2} {change}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(5)
    half = torch.arange(N, device=DEV) % 256 < 128
    now, late = torch.ones(N, device=DEV), torch.where(half, change, 1.0)

    def gradients(step):
        return torch.randn(N, generator=gen, device=DEV) * (now if step <= 1000 else late)

    _, root, _, true = _follow(gradients, (0.9, beta2), 5000)
    _assert_follows(root[half], true[half], "changed half")
    _assert_follows(root[~half], true[~half], "unchanged half")


@pytest.mark.parametrize("beta1", [0.9, 0.95, 0.99])
def test_first_moments_follow_steady_gradients_that_fall(beta1):
    print(f"case moments m {beta1}", flush=True)
    gen = torch.Generator(device=DEV).manual_seed(6)
    half = torch.arange(N, device=DEV) % 256 < 128
    now, late = torch.ones(N, device=DEV), torch.where(half, 0.1, 1.0)

    def gradients(step):
        return (1 + 0.1 * torch.randn(N, generator=gen, device=DEV)) * (now if step <= 500 else late)

    m, _, true, _ = _follow(gradients, (beta1, 0.95), 2500)
    _assert_follows(m[half], true[half], "fallen half")
    _assert_follows(m[~half], true[~half], "other half")


def test_gradients_without_any_variation_need_thresholds():
    """Half of each block has the same gradient in every step, the other half none any more: its sqrt(v) falls below a 64th (exactly: to
    0.05 % of what it was in 300 steps of 2.5 %)."""
    half = torch.arange(N, device=DEV) % 256 < 128
    gone = torch.where(half, 0.0, 1.0)
    _, root, _, true = _follow(lambda step: torch.ones(N, device=DEV) if step <= 200 else gone, (0.9, 0.95), 500, dither=True)
    assert root[half].max() <= 1 / 64 and (root[~half] / true[~half] - 1).abs().max() <= 1e-5


def _dithered(x, root, place, step, key):
    """(codes, scales) by the header's statement, in fp32."""
    f = np.float32
    x = np.concatenate([x, np.zeros(-len(x) % 256, f)]).reshape(-1, 256)
    top = np.max(np.abs(x), axis=1, keepdims=True)
    held = ~(top < f(2.0 ** -100))
    y = x * np.where(held, f(448) / np.where(held, top, f(1)), f(0))
    e = (place + np.arange(x.size, dtype=np.uint64)) * np.uint64(key) + np.uint64(step * 0x9E3779B9)
    u = ((e & np.uint64(0xffffffff)) >> np.uint64(12)).astype(f).reshape(-1, 256) * f(2.0 ** -20)
    a = np.abs(y)
    q = np.where(a < f(2.0 ** -6), f(2.0 ** -9), np.exp2(np.floor(np.log2(np.maximum(a, f(2.0 ** -6)).astype(np.float64)))) / 8).astype(f)
    y = np.copysign(np.minimum(np.floor(a / q + u) * q, f(448)), y)
    if root:
        y = np.where(held & (x > 0) & (y < f(2.0 ** -9)), f(2.0 ** -9), y)
    codes = torch.from_numpy(np.ascontiguousarray(y, f)).to(torch.float8_e4m3fn).view(torch.uint8).numpy().reshape(-1)
    return codes, np.where(held, top * f(1 / 448), f(0))[:, 0]


@pytest.mark.parametrize("betas,dither", [((0.9, 0.999), False), ((0.95, 0.95), False), ((0.9, 0.95), True), ((0.99, 0.999), False)])
@pytest.mark.parametrize("g_type", [torch.float32, torch.bfloat16])
def test_thresholds_are_those_of_the_statement_bit_for_bit(betas, dither, g_type):
    print(f"case thresholds {betas} {dither} {g_type}", flush=True)
    sizes = [3, 0, 1000, 256, 4097]
    gen = torch.Generator().manual_seed(8)
    weights = [torch.randn(n, generator=gen).to(DEV) for n in sizes]
    state = B.adamw_state(sizes, 8, DEV)
    ref = [[w.cpu().numpy().copy(), np.zeros(n, np.float32), np.zeros(n, np.float32)] for w, n in zip(weights, sizes)]
    by_step = {"m": dither or betas[0] > 0.9, "v": dither or betas[1] > 0.95}
    for step in range(1, 6):
        grads = [(torch.randn(n, generator=gen) * torch.exp(3 * torch.randn(n, generator=gen))).to(g_type).to(DEV) for n in sizes]
        B.adamw_step(weights, grads, state, 0.01, step, betas=betas, **(dict(dither=True) if dither else {}))
        at = 0
        for i, n in enumerate(sizes):
            w, m, v, root = P.adamw32(ref[i][0], grads[i].float().cpu().numpy(), ref[i][1], ref[i][2], 0.01, step, betas, 1e-8, 0.0)
            assert np.array_equal(weights[i].cpu().numpy().view(np.uint32), w.view(np.uint32)), f"step {step} tensor {i}: weights"
            whole, held = -(-n // 256) * 256, []
            for k, (value, is_root, name) in enumerate(((m, False, "m"), (root, True, "v"))):
                if n == 0:
                    held.append(value)
                    continue
                codes, scales = _dithered(value, is_root, at, step, KEY[name]) if by_step[name] else P.encode(value, is_root)
                got = state[k].view(torch.uint8)[at:at + whole].cpu().numpy()
                assert np.array_equal(got, codes), f"step {step} tensor {i}: codes of {name}"
                assert np.array_equal(state[2 + k][at // 256:(at + whole) // 256].cpu().numpy().view(np.uint32), scales.view(np.uint32))
                held.append(P.decode(codes, scales)[:n])
            ref[i] = [w, held[0], held[1] * held[1]]
            at += whole


def test_infinities_and_nan_pass_the_thresholds():
    for value in (float("inf"), float("nan")):
        w, g = [torch.ones(700, device=DEV)], torch.full((700,), 0.5, device=DEV)
        g[300] = value
        state = B.adamw_state([700], 8, DEV)
        B.adamw_step(w, [g], state, 0.1, 1, dither=True)
        B.adamw_step(w, [torch.full((700,), 0.5, device=DEV)], state, 0.1, 2, dither=True)
        bad = torch.zeros(700, dtype=torch.bool, device=DEV)
        bad[256:512] = True
        assert torch.equal(w[0].isnan(), bad)


@pytest.mark.parametrize("dither", [False, True])
def test_a_second_moment_that_overflows_spoils_its_block(dither):
    """A gradient of 1e25 is finite, and so is m; its square is not.  The block must not go on with infinite sqrt(v), which would hold all
    of its weights still without a sign."""
    n = 700
    w, g, half = [torch.ones(n, device=DEV)], torch.full((n,), 0.5, device=DEV), torch.full((n,), 0.5, device=DEV)
    g[300] = 1e25
    state = B.adamw_state([n], 8, DEV)
    B.adamw_step(w, [g], state, 0.1, 1, dither=dither)
    m, root = _held(state)
    bad = torch.zeros(n, dtype=torch.bool, device=DEV)
    bad[256:512] = True
    assert m.isfinite().all() and torch.equal(root[:n].isnan(), bad) and root[~root.isnan()].isfinite().all()
    B.adamw_step(w, [half], state, 0.1, 2, dither=dither)
    assert torch.equal(w[0].isnan(), bad)
