"""What the language-model operators refuse, before anything is launched (CPU only: the pointers are never followed)."""
import ctypes as C
import os

import pytest
import torch

from paper_2010_16248_amd import binding as B



@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2010_16248_amd import build
        build.build(verbose=False)
    return B.load_library()


def at(i):
    return C.c_void_p((i + 1) << 40)


def refused(lib, rc, word, status=B.ACC_EINVAL):
    assert rc == status
    assert word in lib.accordion_operator_error().decode()


def embedding(**kw):
    args = dict(vocab=10, dim=8, tokens=5, table_stride=8, out_stride=8, index_bits=64, table_type=0, out_type=0, accumulate=0, scale=1.0)
    args.update(kw)
    return B.acc_embedding(**args)


@pytest.mark.parametrize("change,word", [
    (dict(vocab=0), "vocab"), (dict(vocab=2 ** 31 - 1), "vocab"), (dict(dim=0), "dim"), (dict(dim=2 ** 24 + 1), "dim"),
    (dict(tokens=-1), "tokens"), (dict(tokens=2 ** 28 + 1), "tokens"), (dict(index_bits=16), "index_bits"), (dict(table_type=2), "type"),
    (dict(out_type=-1), "type"), (dict(accumulate=2), "accumulate"), (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"),
    (dict(table_stride=7), "table_stride"), (dict(out_stride=7), "out_stride"), (dict(table_stride=2 ** 41), "table_stride"),
])
def test_embedding_configurations(lib, change, word):
    cfg, n = embedding(**change), C.c_size_t(0)
    refused(lib, lib.accordion_embedding_forward(C.byref(cfg), at(0), at(1), at(2), None), word)
    refused(lib, lib.accordion_embedding_backward(C.byref(cfg), at(0), at(1), at(2), at(3), 1 << 40, None), word)
    refused(lib, lib.accordion_embedding_workspace_bytes(C.byref(cfg), C.byref(n)), word)


def test_embedding_pointers(lib):
    cfg, n = embedding(), C.c_size_t(0)
    fwd, bwd = lib.accordion_embedding_forward, lib.accordion_embedding_backward
    refused(lib, lib.accordion_embedding_workspace_bytes(C.byref(cfg), None), "NULL")
    refused(lib, fwd(None, at(0), at(1), at(2), None), "NULL")
    for k in range(3):
        ptrs = [at(0), at(1), at(2)]
        ptrs[k] = None
        refused(lib, fwd(C.byref(cfg), *ptrs, None), "NULL")
        refused(lib, bwd(C.byref(cfg), *ptrs, at(3), 1 << 40, None), "NULL")
        ptrs[k] = C.c_void_p(at(k).value + 2)
        refused(lib, fwd(C.byref(cfg), *ptrs, None), "aligned")
        refused(lib, bwd(C.byref(cfg), *ptrs, at(3), 1 << 40, None), "aligned")
    refused(lib, fwd(C.byref(cfg), at(0), at(1), C.c_void_p(at(1).value + 32), None), "overlaps")
    cfg = embedding(tokens=600)          # enough for a workspace
    assert lib.accordion_embedding_workspace_bytes(C.byref(cfg), C.byref(n)) == B.ACC_OK and n.value > 0
    refused(lib, bwd(C.byref(cfg), at(0), at(1), at(2), None, n.value, None), "workspace")
    refused(lib, bwd(C.byref(cfg), at(0), at(1), at(2), C.c_void_p(at(3).value + 128), n.value, None), "aligned")
    refused(lib, bwd(C.byref(cfg), at(0), at(1), at(2), at(3), n.value - 1, None), "workspace", B.ACC_ENOSPACE)
    refused(lib, bwd(C.byref(cfg), at(0), at(1), at(2), at(1), n.value, None), "overlaps")
    refused(lib, bwd(C.byref(cfg), at(0), at(1), at(1), at(3), n.value, None), "overlaps")


def layernorm(**kw):
    args = dict(rows=4, dim=8, x_stride=8, y_stride=8, grad_x_stride=8, type=0, accumulate=0, eps=1e-5)
    args.update(kw)
    return B.acc_layernorm(**args)


@pytest.mark.parametrize("change,word", [
    (dict(rows=-1), "rows"), (dict(rows=2 ** 31), "rows"), (dict(dim=0), "dim"), (dict(dim=2 ** 24 + 1), "dim"), (dict(type=3), "type"),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(x_stride=7), "x_stride"), (dict(y_stride=7), "y_stride"),
    (dict(accumulate=-1), "accumulate"),
])
def test_layernorm_configurations(lib, change, word):
    cfg, n = layernorm(**change), C.c_size_t(0)
    refused(lib, lib.accordion_layernorm_forward(C.byref(cfg), *[at(i) for i in range(6)], None), word)
    refused(lib, lib.accordion_layernorm_backward(C.byref(cfg), *[at(i) for i in range(9)], 1 << 40, None), word)
    refused(lib, lib.accordion_layernorm_workspace_bytes(C.byref(cfg), C.byref(n)), word)


def test_layernorm_pointers(lib):
    cfg, n = layernorm(), C.c_size_t(0)
    fwd, bwd = lib.accordion_layernorm_forward, lib.accordion_layernorm_backward
    refused(lib, fwd(None, *[at(i) for i in range(6)], None), "NULL")
    refused(lib, lib.accordion_layernorm_workspace_bytes(C.byref(cfg), None), "NULL")
    for k in (0, 1, 3):
        ptrs = [at(i) for i in range(6)]
        ptrs[k] = None
        refused(lib, fwd(C.byref(cfg), *ptrs, None), "NULL")
    for k in range(6):
        ptrs = [at(i) for i in range(6)]
        ptrs[k] = C.c_void_p(at(k).value + 1)
        refused(lib, fwd(C.byref(cfg), *ptrs, None), "aligned")
    refused(lib, fwd(C.byref(cfg), at(0), at(1), at(2), at(3), at(4), None, None), "together")
    refused(lib, fwd(C.byref(cfg), at(0), at(1), at(2), at(0), at(4), at(5), None), "overlaps")
    refused(lib, fwd(C.byref(cfg), at(0), at(1), at(2), at(3), at(4), at(4), None), "overlaps")
    assert lib.accordion_layernorm_workspace_bytes(C.byref(cfg), C.byref(n)) == B.ACC_OK
    for k in (0, 1, 2, 3, 4, 5, 6):
        ptrs = [at(i) for i in range(9)]
        ptrs[k] = None
        refused(lib, bwd(C.byref(cfg), *ptrs, n.value, None), "NULL")
    for k in range(8):
        ptrs = [at(i) for i in range(9)]
        ptrs[k] = C.c_void_p(at(k).value + 1)
        refused(lib, bwd(C.byref(cfg), *ptrs, n.value, None), "aligned")
    ptrs = [at(i) for i in range(9)]
    refused(lib, bwd(C.byref(cfg), *ptrs, n.value - 1, None), "workspace", B.ACC_ENOSPACE)
    ptrs[7] = ptrs[6]
    refused(lib, bwd(C.byref(cfg), *ptrs, n.value, None), "overlaps")
    bad = layernorm(grad_x_stride=3)
    refused(lib, bwd(C.byref(bad), *[at(i) for i in range(9)], n.value, None), "grad_x_stride")


def recurrence(**kw):
    args = dict(batch=2, steps=3, channels=4, type=0)
    args.update({f"{k}_{d}": v for k in ("gate", "input", "out", "grad_gate", "grad_input", "grad_out") for d, v in (("batch", 12), ("step", 4))})
    args.update(kw)
    return B.acc_recurrence(**args)


@pytest.mark.parametrize("change,word", [
    (dict(batch=-1), "batch"), (dict(batch=65536), "batch"), (dict(steps=-1), "steps"), (dict(steps=2 ** 31), "steps"),
    (dict(channels=0), "channels"), (dict(channels=2 ** 24 + 1), "channels"), (dict(type=2), "type"), (dict(gate_step=-4), "stride"),
    (dict(input_batch=-1), "stride"), (dict(out_step=3), "overlap"), (dict(out_batch=11), "overlap"), (dict(out_batch=0), "overlap"),
    (dict(out_batch=4, out_step=7), "overlap"), (dict(gate_batch=2 ** 41), "stride"),
])
def test_recurrence_configurations(lib, change, word):
    cfg = recurrence(**change)
    refused(lib, lib.accordion_recurrence_forward(C.byref(cfg), *[at(i) for i in range(7)], 1 << 40, None), word)
    if not any(k.startswith("out") for k in change):
        refused(lib, lib.accordion_recurrence_backward(C.byref(cfg), *[at(i) for i in range(11)], 1 << 40, None), word)


@pytest.mark.parametrize("change,word", [(dict(grad_gate_step=3), "overlap"), (dict(grad_input_batch=11), "overlap"), (dict(grad_out_step=-1), "stride")])
def test_recurrence_gradient_strides(lib, change, word):
    cfg = recurrence(**change)
    refused(lib, lib.accordion_recurrence_backward(C.byref(cfg), *[at(i) for i in range(11)], 1 << 40, None), word)


def test_recurrence_pointers(lib):
    cfg = recurrence()
    fwd, bwd = lib.accordion_recurrence_forward, lib.accordion_recurrence_backward
    refused(lib, fwd(None, *[at(i) for i in range(7)], 1 << 40, None), "NULL")
    refused(lib, lib.accordion_recurrence_workspace_bytes(C.byref(cfg), None), "NULL")
    for k in (0, 1, 4):
        ptrs = [at(i) for i in range(7)]
        ptrs[k] = None
        refused(lib, fwd(C.byref(cfg), *ptrs, 1 << 40, None), "NULL")
    for k in (0, 1, 2, 5, 7, 8):
        ptrs = [at(i) for i in range(11)]
        ptrs[k] = None
        refused(lib, bwd(C.byref(cfg), *ptrs, 1 << 40, None), "NULL")
    for k in range(6):
        ptrs = [at(i) for i in range(7)]
        ptrs[k] = C.c_void_p(at(k).value + 1)
        refused(lib, fwd(C.byref(cfg), *ptrs, 1 << 40, None), "aligned")
    for k in range(10):
        ptrs = [at(i) for i in range(11)]
        ptrs[k] = C.c_void_p(at(k).value + 1)
        refused(lib, bwd(C.byref(cfg), *ptrs, 1 << 40, None), "aligned")
    ptrs = [at(i) for i in range(7)]
    ptrs[4] = ptrs[0]
    refused(lib, fwd(C.byref(cfg), *ptrs, 1 << 40, None), "overlaps")
    ptrs = [at(i) for i in range(11)]
    ptrs[8] = ptrs[7]
    refused(lib, bwd(C.byref(cfg), *ptrs, 1 << 40, None), "overlaps")


def adamw(sizes=(5, 600), decay=None, **kw):
    arr = (C.c_int64 * len(sizes))(*sizes)
    wd = None if decay is None else (C.c_float * len(sizes))(*decay)
    args = dict(n_tensors=len(sizes), weight_type=0, grad_type=0, state_bits=32, sizes_host=arr, weight_decay_host=wd, lr=0.1, beta1=0.9,
                beta2=0.99, eps=1e-8, step=1)
    args.update(kw)
    return B.acc_adamw(**args)


def step(lib, cfg, w=(0, 1), g=(2, 3), c=None, m=4, v=5, ms=None, vs=None, gs=None):
    arr = lambda ks: None if ks is None else (C.c_void_p * 2)(*[None if k is None else at(k).value for k in ks])
    one = lambda k: None if k is None else at(k)
    return lib.accordion_adamw_step(None if cfg is None else C.byref(cfg), arr(w), arr(g), arr(c), one(m), one(v), one(ms), one(vs), one(gs), None)


@pytest.mark.parametrize("change,word", [
    (dict(n_tensors=-1), "n_tensors"), (dict(n_tensors=2 ** 20 + 1), "n_tensors"), (dict(sizes_host=None), "sizes_host"),
    (dict(sizes=(5, -1)), "size"), (dict(sizes=(2 ** 36 + 1, 1)), "size"), (dict(weight_type=2), "type"), (dict(grad_type=-1), "type"),
    (dict(state_bits=16), "state_bits"), (dict(lr=-1.0), "lr"), (dict(lr=float("inf")), "lr"), (dict(eps=-1e-9), "eps"),
    (dict(beta1=1.0), "betas"), (dict(beta2=-0.1), "betas"), (dict(beta1=float("nan")), "betas"), (dict(step=0), "step"),
    (dict(decay=(0.1, -0.1)), "decay"), (dict(decay=(float("nan"), 0.0)), "decay"),
])
def test_adamw_configurations(lib, change, word):
    refused(lib, step(lib, adamw(**change)), word)


def test_adamw_pointers(lib):
    refused(lib, step(lib, None), "NULL")
    refused(lib, lib.accordion_adamw_state_elements(C.byref(adamw()), None), "NULL")
    for bad in (dict(w=None), dict(g=None), dict(m=None), dict(v=None), dict(w=(0, None)), dict(g=(None, 3))):
        refused(lib, step(lib, adamw(), **bad), "NULL")
    refused(lib, step(lib, adamw(state_bits=8)), "m_scale")
    refused(lib, step(lib, adamw(), ms=6, vs=7), "no scales")
    for bad in (dict(m=0), dict(v=4), dict(c=(0, None)), dict(g=(2, 1)), dict(c=(4, 9)), dict(g=(4, 3))):
        assert step(lib, adamw(), **bad) == B.ACC_EINVAL
        assert "overlap" in lib.accordion_operator_error().decode()


def test_adamw_state_elements(lib):
    assert B.adamw_state_elements([], 8) == 0
    assert B.adamw_state_elements([1, 256, 257, 0], 8) == 256 + 256 + 512
    assert B.adamw_state_elements([1, 256, 257, 0], 32) == 514


def test_the_binding_refuses_what_the_c_abi_cannot_see():
    cpu = torch.ones
    ids = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="one GPU"):
        B.embedding_forward(ids, cpu(4, 5), cpu(3, 5))
    with pytest.raises(ValueError, match="ids"):
        B.embedding_forward(ids.float(), cpu(4, 5), cpu(3, 5))
    with pytest.raises(ValueError, match="fit"):
        B.embedding_forward(ids, cpu(4, 5), cpu(3, 6))
    with pytest.raises(ValueError, match="fit"):
        B.embedding_forward(ids, cpu(4, 5), cpu(2, 5))
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        B.embedding_forward(ids, cpu(4, 5).double(), cpu(3, 5))
    with pytest.raises(ValueError, match="float32"):
        B.embedding_backward(ids, cpu(3, 5), cpu(4, 5).bfloat16())
    with pytest.raises(ValueError, match="contiguous"):
        B.embedding_forward(ids, cpu(5, 4).t(), cpu(3, 5))
    with pytest.raises(ValueError, match="fit"):
        B.layernorm_forward(cpu(3, 4), cpu(4), None, cpu(3, 4).bfloat16())
    with pytest.raises(ValueError, match="weight"):
        B.layernorm_forward(cpu(3, 4), cpu(5), None, cpu(3, 4))
    with pytest.raises(ValueError, match="mean"):
        B.layernorm_forward(cpu(3, 4), cpu(4), None, cpu(3, 4), cpu(4), cpu(3))
    with pytest.raises(ValueError, match="grad_x"):
        B.layernorm_backward(cpu(3, 4), cpu(3, 4), cpu(4), cpu(3), cpu(3), cpu(3, 5), cpu(4))
    with pytest.raises(ValueError, match="gate"):
        B.recurrence_forward(cpu(3, 4), cpu(3, 4), cpu(3, 4))
    with pytest.raises(ValueError, match="input"):
        B.recurrence_forward(cpu(1, 3, 4), cpu(1, 3, 5), cpu(1, 3, 4))
    with pytest.raises(ValueError, match="contiguous"):
        B.recurrence_forward(cpu(1, 3, 4), cpu(1, 4, 3).transpose(1, 2), cpu(1, 3, 4))
    with pytest.raises(ValueError, match="h0"):
        B.recurrence_forward(cpu(1, 3, 4), cpu(1, 3, 4), cpu(1, 3, 4), h0=cpu(1, 5))
    with pytest.raises(ValueError, match="lengths"):
        B.recurrence_forward(cpu(1, 3, 4), cpu(1, 3, 4), cpu(1, 3, 4), lengths=ids[:1])
    state = B.adamw_state([6], 32, "cpu")
    with pytest.raises(ValueError, match="length"):
        B.adamw_step([cpu(6)], [], state, 0.1, 1)
    with pytest.raises(ValueError, match="fit"):
        B.adamw_step([cpu(6)], [cpu(7)], state, 0.1, 1)
    with pytest.raises(ValueError, match="m must"):
        B.adamw_step([cpu(7)], [cpu(7)], state, 0.1, 1)
    with pytest.raises(ValueError, match="m must"):
        B.adamw_step([cpu(6)], [cpu(6)], (*state[:2], cpu(1), cpu(1)), 0.1, 1)
    with pytest.raises(ValueError, match="decay"):
        B.adamw_step([cpu(6)], [cpu(6)], state, 0.1, 1, weight_decay=[0.1, 0.1])
    with pytest.raises(ValueError, match="copy"):
        B.adamw_step([cpu(6)], [cpu(6)], state, 0.1, 1, copies=[cpu(6)])
    with pytest.raises(ValueError, match="grad_scale"):
        B.adamw_step([cpu(6)], [cpu(6)], state, 0.1, 1, grad_scale=cpu(2))
    with pytest.raises(ValueError, match="one GPU"):
        B.adamw_step([cpu(6)], [cpu(6)], state, 0.1, 1)


def test_sizes_beyond_a_launch_are_refused(lib):
    n = C.c_size_t(0)
    cfg = embedding(tokens=2 ** 28, dim=2 ** 20, out_stride=2 ** 20, table_stride=2 ** 20)
    refused(lib, lib.accordion_embedding_workspace_bytes(C.byref(cfg), C.byref(n)), "tokens x dim")
    refused(lib, lib.accordion_embedding_backward(C.byref(cfg), at(0), at(1 << 10), at(2 << 10), at(3 << 10), 1 << 40, None), "tokens x dim")
    cfg = recurrence(batch=65535, steps=2 ** 20, channels=64, out_batch=2 ** 26, out_step=64, gate_batch=2 ** 26, gate_step=64,
                     input_batch=2 ** 26, input_step=64)
    refused(lib, lib.accordion_recurrence_workspace_bytes(C.byref(cfg), C.byref(n)), "too many steps")
    refused(lib, lib.accordion_recurrence_forward(C.byref(cfg), *[at(i << 12) for i in range(7)], 1 << 40, None), "too many steps")


@pytest.mark.parametrize("dither", [-1, 2])
def test_adamw_thresholds_are_on_or_off(lib, dither):
    refused(lib, step(lib, adamw(state_bits=8, dither=dither)), "dither")


@pytest.mark.parametrize("case", ["a weight twice", "a weight in another's gradient", "a copy in another's weight", "a copy twice", "partly"])
def test_adamw_tensors_must_be_apart_from_one_another(lib, case):
    w, g, c = [at(0), at(1)], [at(2), at(3)], None
    if case == "a weight twice":
        w[1] = w[0]
    elif case == "a weight in another's gradient":
        g[0] = C.c_void_p(at(1).value + 64)
    elif case == "a copy in another's weight":
        c = [at(1), None]
    elif case == "a copy twice":
        c = [at(9), C.c_void_p(at(9).value + 8)]
    else:
        w[0] = C.c_void_p(at(1).value + 2396)        # the last of the second one's 600 elements
    arr = lambda ks: None if ks is None else (C.c_void_p * 2)(*[None if k is None else k.value for k in ks])
    cfg = adamw()
    refused(lib, lib.accordion_adamw_step(C.byref(cfg), arr(w), arr(g), arr(c), at(4), at(5), None, None, None, None), "another tensor")
