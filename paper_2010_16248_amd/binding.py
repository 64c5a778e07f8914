"""ctypes binding of libaccordion.so: argument marshalling only.

Every step of the path runs in the HIP kernels behind the C ABI declared in
include/accordion.h; this module converts Python arguments to C ones and checks
status codes.  PyTorch is used for device memory and the stream handle, nothing
else.  There is no CPU fallback: if the shared library is missing or fails to
load, every call raises.
"""
from __future__ import annotations

import array
import ctypes as C
import os
from typing import List, Optional, Sequence, Tuple

import numpy as np

ACC_OK, ACC_EINVAL, ACC_ESTATE, ACC_ENOSPACE, ACC_EHIP = 0, 1, 2, 3, 4
ACC_POWERSGD, ACC_TOPK, ACC_BATCH = 0, 1, 2
ACC_MAX_WORKERS = 32
ACC_MAX_RANK = 4

_STATUS = {0: "ACC_OK", 1: "ACC_EINVAL", 2: "ACC_ESTATE", 3: "ACC_ENOSPACE", 4: "ACC_EHIP"}

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libaccordion.so")


class acc_layer(C.Structure):
    _fields_ = [("offset", C.c_int64), ("rows", C.c_int32), ("cols", C.c_int32),
                ("is_matrix", C.c_int32)]


class acc_config(C.Structure):
    _fields_ = [("method", C.c_int32), ("n_layers", C.c_int32),
                ("layers", C.POINTER(acc_layer)), ("n_params", C.c_int64),
                ("n_workers", C.c_int32), ("rank_crit", C.c_int32), ("rank_noncrit", C.c_int32),
                ("k_num_crit", C.c_int32), ("k_num_noncrit", C.c_int32), ("k_den", C.c_int32),
                ("eta", C.c_float), ("initial_level", C.c_int32),
                ("batch_multiplier", C.c_int32), ("batch_monotone", C.c_int32),
                ("detector", C.c_int32)]


class acc_embedding(C.Structure):
    _fields_ = [("vocab", C.c_int64), ("dim", C.c_int64), ("tokens", C.c_int64), ("table_stride", C.c_int64),
                ("out_stride", C.c_int64), ("index_bits", C.c_int32), ("table_type", C.c_int32),
                ("out_type", C.c_int32), ("accumulate", C.c_int32), ("scale", C.c_float)]


class acc_layernorm(C.Structure):
    _fields_ = [("rows", C.c_int64), ("dim", C.c_int64), ("x_stride", C.c_int64), ("y_stride", C.c_int64),
                ("grad_x_stride", C.c_int64), ("type", C.c_int32), ("accumulate", C.c_int32), ("eps", C.c_float)]


class acc_recurrence(C.Structure):
    _fields_ = [("batch", C.c_int64), ("steps", C.c_int64), ("channels", C.c_int64),
                ("gate_batch", C.c_int64), ("gate_step", C.c_int64), ("input_batch", C.c_int64),
                ("input_step", C.c_int64), ("out_batch", C.c_int64), ("out_step", C.c_int64),
                ("grad_gate_batch", C.c_int64), ("grad_gate_step", C.c_int64), ("grad_input_batch", C.c_int64),
                ("grad_input_step", C.c_int64), ("grad_out_batch", C.c_int64), ("grad_out_step", C.c_int64),
                ("type", C.c_int32)]


class acc_convolution(C.Structure):
    _fields_ = [(k, C.c_int64) for k in ("batch", "steps", "channels", "x_batch", "x_step", "out_batch", "out_step", "grad_x_batch",
                                         "grad_x_step")] + \
               [(k, C.c_int32) for k in ("width", "type", "silu", "accumulate")]


class acc_scan(C.Structure):
    _fields_ = [(k, C.c_int64) for k in ("batch", "steps", "channels")] + \
               [(f"{k}_{d}", C.c_int64) for k in ("x", "delta", "b", "c", "gate", "out", "grad_x", "grad_delta", "grad_b", "grad_c",
                                                  "grad_gate") for d in ("batch", "step")] + \
               [(k, C.c_int32) for k in ("states", "groups", "type", "softplus", "accumulate")]


class acc_logprob(C.Structure):
    _fields_ = [(k, C.c_int64) for k in ("rows", "vocab", "logits_stride", "grad_stride")] + \
               [(k, C.c_int32) for k in ("index_bits", "type", "top")]


class acc_adamw(C.Structure):
    _fields_ = [("n_tensors", C.c_int32), ("weight_type", C.c_int32), ("grad_type", C.c_int32),
                ("state_bits", C.c_int32), ("sizes_host", C.POINTER(C.c_int64)),
                ("weight_decay_host", C.POINTER(C.c_float)), ("lr", C.c_double), ("beta1", C.c_double),
                ("beta2", C.c_double), ("eps", C.c_double), ("step", C.c_int64), ("dither", C.c_int32)]


class AccordionError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status


_lib = None

EXPORTS = [
    "accordion_workspace_bytes", "accordion_init", "accordion_init_static", "accordion_destroy", "accordion_last_error",
    "accordion_compress_step", "accordion_aggregate", "accordion_decompress", "accordion_step_all",
    "accordion_decompress_update", "accordion_step_all_update", "accordion_batch_status", "accordion_set_stream", "accordion_topk_overlap", "accordion_payload_format",
    "accordion_detect_regime", "accordion_reset_accumulator", "accordion_get_levels",
    "accordion_get_norms", "accordion_get_payload", "accordion_get_factors",
    "accordion_payload_words", "accordion_state_bytes", "accordion_get_state", "accordion_set_state",
    "accordion_set_profiling", "accordion_get_profile", "accordion_stage_name",
    "accordion_probe_copy", "accordion_topk_stats", "accordion_topk_short_lists", "accordion_flush",
    "accordion_operator_error", "accordion_embedding_forward", "accordion_embedding_workspace_bytes",
    "accordion_embedding_backward", "accordion_layernorm_forward", "accordion_layernorm_workspace_bytes",
    "accordion_layernorm_backward", "accordion_recurrence_workspace_bytes", "accordion_recurrence_forward",
    "accordion_recurrence_backward", "accordion_convolution_forward", "accordion_convolution_workspace_bytes",
    "accordion_convolution_backward", "accordion_scan_workspace_bytes", "accordion_scan_forward", "accordion_scan_backward",
    "accordion_logprob_workspace_bytes", "accordion_logprob_forward", "accordion_logprob_backward", "accordion_adamw_state_elements", "accordion_adamw_step",
]
ACC_N_STAGES = 48     # upper bound of the stage numbers; accordion_stage_name is NULL beyond the last


def load_library() -> C.CDLL:
    """Load libaccordion.so (built in-tree by paper_2010_16248_amd/build.py)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           "`python -m paper_2010_16248_amd.build` (there is no fallback path)")
    # The caller's device memory and streams come from PyTorch, which ships its own HIP runtime:
    # that runtime has to be the one already in the process when the library is loaded, or the
    # library binds to a second copy that sees no device.
    import torch
    _TYPES.update({torch.float32: ACC_FLOAT, torch.bfloat16: ACC_BF16})
    _INDEX_BITS.update({torch.int32: 32, torch.int64: 64})
    global _FLOAT32, _INT32
    _FLOAT32, _INT32 = torch.float32, torch.int32
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
    sig = {
        "accordion_workspace_bytes": [C.POINTER(acc_config), C.POINTER(C.c_size_t)],
        "accordion_init": [C.POINTER(acc_config), vp, C.c_size_t, vp, vp, C.POINTER(vp)],
        "accordion_init_static": [C.POINTER(acc_config), vp, vp, C.POINTER(vp)],
        "accordion_destroy": [vp],
        "accordion_compress_step": [vp, i32, vp, i32],
        "accordion_aggregate": [vp, i32],
        "accordion_decompress": [vp, vp],
        "accordion_step_all": [vp, C.POINTER(vp), vp],
        "accordion_decompress_update": [vp, vp, vp, f32, f32, f32],
        "accordion_payload_format": [C.POINTER(acc_config), C.c_int32, C.c_int32, C.POINTER(C.c_int32),
                                     C.POINTER(C.c_int64), C.POINTER(C.c_int64)],
        "accordion_topk_overlap": [vp, C.c_int32, C.c_int32, C.POINTER(C.c_int64), C.POINTER(C.c_int64)],
        "accordion_set_stream": [vp, vp],
        "accordion_batch_status": [vp, C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.POINTER(C.c_int32),
                                   C.POINTER(C.c_int64), C.POINTER(C.c_int64)],
        "accordion_step_all_update": [vp, C.POINTER(vp), vp, vp, f32, f32, f32],
        "accordion_detect_regime": [vp, f32, f32],
        "accordion_reset_accumulator": [vp],
        "accordion_flush": [vp],
        "accordion_get_levels": [vp, vp],
        "accordion_get_norms": [vp, vp, vp],
        "accordion_get_payload": [vp, i32, i32, vp, vp, i64, C.POINTER(i64)],
        "accordion_get_factors": [vp, i32, vp, vp, C.POINTER(i32)],
        "accordion_payload_words": [vp, C.POINTER(i64), C.POINTER(i64)],
        "accordion_state_bytes": [vp, C.POINTER(C.c_size_t)],
        "accordion_get_state": [vp, vp, C.c_size_t],
        "accordion_set_state": [vp, vp, C.c_size_t],
        "accordion_set_profiling": [vp, i32],
        "accordion_get_profile": [vp, i32, C.POINTER(C.c_double), C.POINTER(i64)],
        "accordion_probe_copy": [vp, vp, i64, vp],
        "accordion_topk_stats": [vp, C.POINTER(i64), C.POINTER(i64)],
        "accordion_topk_short_lists": [vp, C.POINTER(i64)],
        "accordion_embedding_forward": [C.POINTER(acc_embedding), vp, vp, vp, vp],
        "accordion_embedding_workspace_bytes": [C.POINTER(acc_embedding), C.POINTER(C.c_size_t)],
        "accordion_embedding_backward": [C.POINTER(acc_embedding), vp, vp, vp, vp, C.c_size_t, vp],
        "accordion_layernorm_forward": [C.POINTER(acc_layernorm), vp, vp, vp, vp, vp, vp, vp],
        "accordion_layernorm_workspace_bytes": [C.POINTER(acc_layernorm), C.POINTER(C.c_size_t)],
        "accordion_layernorm_backward": [C.POINTER(acc_layernorm)] + [vp] * 9 + [C.c_size_t, vp],
        "accordion_recurrence_workspace_bytes": [C.POINTER(acc_recurrence), C.POINTER(C.c_size_t)],
        "accordion_recurrence_forward": [C.POINTER(acc_recurrence)] + [vp] * 7 + [C.c_size_t, vp],
        "accordion_recurrence_backward": [C.POINTER(acc_recurrence)] + [vp] * 11 + [C.c_size_t, vp],
        "accordion_convolution_forward": [C.POINTER(acc_convolution)] + [vp] * 8,
        "accordion_convolution_workspace_bytes": [C.POINTER(acc_convolution), C.POINTER(C.c_size_t)],
        "accordion_convolution_backward": [C.POINTER(acc_convolution)] + [vp] * 12 + [C.c_size_t, vp],
        "accordion_scan_workspace_bytes": [C.POINTER(acc_scan), i32, C.POINTER(C.c_size_t)],
        "accordion_scan_forward": [C.POINTER(acc_scan)] + [vp] * 13 + [C.c_size_t, vp],
        "accordion_scan_backward": [C.POINTER(acc_scan)] + [vp] * 22 + [C.c_size_t, vp],
        "accordion_logprob_workspace_bytes": [C.POINTER(acc_logprob), C.POINTER(C.c_size_t)],
        "accordion_logprob_forward": [C.POINTER(acc_logprob)] + [vp] * 8 + [C.c_size_t, vp],
        "accordion_logprob_backward": [C.POINTER(acc_logprob)] + [vp] * 8,
        "accordion_adamw_state_elements": [C.POINTER(acc_adamw), C.POINTER(i64)],
        "accordion_adamw_step": [C.POINTER(acc_adamw), C.POINTER(vp), C.POINTER(vp), C.POINTER(vp)] + [vp] * 6,
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = i32
    lib.accordion_last_error.argtypes = [vp]
    lib.accordion_last_error.restype = C.c_char_p
    lib.accordion_operator_error.argtypes = []
    lib.accordion_operator_error.restype = C.c_char_p
    lib.accordion_stage_name.argtypes = [i32]
    lib.accordion_stage_name.restype = C.c_char_p
    _lib = lib
    return lib


def make_config(method: int, layers: Sequence, n_workers: int, level_crit: int, level_noncrit: int,
                k_den: int = 100, eta: float = 0.5, initial_level: int = 1,
                n_params: Optional[int] = None, batch_multiplier: int = 1,
                batch_monotone: int = 1, detector: int = 0) -> Tuple[acc_config, object]:
    """Build an acc_config; returns (config, keep_alive) -- the layer array must outlive the
    calls that read it.  layers: objects with offset/rows/cols/is_matrix or 4-tuples."""
    arr = (acc_layer * max(1, len(layers)))()
    end = 0
    for i, l in enumerate(layers):
        off, r, c, m = (l.offset, l.rows, l.cols, l.is_matrix) if hasattr(l, "offset") else l
        arr[i] = acc_layer(int(off), int(r), int(c), int(m))
        end = max(end, int(off) + int(r) * int(c))
    cfg = acc_config()
    cfg.method = method
    cfg.n_layers = len(layers)
    cfg.layers = C.cast(arr, C.POINTER(acc_layer))
    cfg.n_params = end if n_params is None else n_params
    cfg.n_workers = n_workers
    cfg.batch_multiplier, cfg.batch_monotone = batch_multiplier, batch_monotone
    cfg.detector = detector
    if method == ACC_POWERSGD:
        cfg.rank_crit, cfg.rank_noncrit = level_crit, level_noncrit
        cfg.k_num_crit = cfg.k_num_noncrit = cfg.k_den = 1
    elif method == ACC_BATCH:
        cfg.rank_crit = cfg.rank_noncrit = cfg.k_num_crit = cfg.k_num_noncrit = cfg.k_den = 1
    else:
        cfg.rank_crit = cfg.rank_noncrit = 1
        cfg.k_num_crit, cfg.k_num_noncrit, cfg.k_den = level_crit, level_noncrit, k_den
    cfg.eta = eta
    cfg.initial_level = initial_level
    return cfg, arr


def _check(lib, ctx, rc: int) -> None:
    if rc != ACC_OK:
        msg = lib.accordion_last_error(ctx)
        raise AccordionError(rc, msg.decode() if msg else "")


def accordion_workspace_bytes(cfg: acc_config) -> int:
    lib = load_library()
    out = C.c_size_t(0)
    _check(lib, None, lib.accordion_workspace_bytes(C.byref(cfg), C.byref(out)))
    return int(out.value)


def payload_format(cfg: acc_config, layer: int, level: int) -> Tuple[int, int, int]:
    """(format, kept, words) of a TopK layer at a level; host arithmetic only."""
    lib = load_library()
    fmt, kept, words = C.c_int32(0), C.c_int64(0), C.c_int64(0)
    _check(lib, None, lib.accordion_payload_format(C.byref(cfg), layer, level, C.byref(fmt), C.byref(kept),
                                                   C.byref(words)))
    return fmt.value, kept.value, words.value


ACC_PAYLOAD_INDEX_VALUE, ACC_PAYLOAD_VALUES_HOLES = 0, 1
ACC_DETECT_NORM, ACC_DETECT_MSDR = 0, 1


def probe_copy(dst, src) -> None:
    """accordion_probe_copy on two device tensors of equal size, on torch's current stream."""
    import torch
    lib = load_library()
    stream = torch.cuda.current_stream().cuda_stream
    _check(lib, None, lib.accordion_probe_copy(C.c_void_p(dst.data_ptr()), C.c_void_p(src.data_ptr()),
                                               src.numel(), C.c_void_p(stream)))


# ---- operators of a language model's training step (no context) ----------------------------------
# Tensors are torch tensors on one GPU; the work goes to torch's current stream of that GPU.  What the
# C ABI cannot see (shapes, element types, devices, strides inside a row) is checked here and raises
# ValueError; what it refuses raises AccordionError.  A workspace is taken from torch's allocator for the
# call unless one is given (uint8, 256-byte aligned, of at least the bytes that the C ABI asks for).

ACC_FLOAT, ACC_BF16 = 0, 1
ACC_ADAMW_BLOCK = 256


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


_TYPES, _INDEX_BITS = {}, {}      # by torch's types, filled once torch is loaded
_FLOAT32 = _INT32 = None          # torch's types, likewise


def _type_of(t, name: str) -> int:
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    return kind


def _rows_of(t, name: str) -> Tuple[int, int, int]:
    """(rows, elements per row, elements between rows) of a tensor whose last dimension is a row."""
    if t.dim() == 2:
        rows, dim = t.shape
        stride, inner = t.stride()
        if inner == 1 or dim <= 1:
            return rows, dim, stride
    elif t.dim() >= 1 and t.is_contiguous():
        dim = t.shape[-1]
        return (t.numel() // dim if dim else 0), dim, dim
    raise ValueError(f"{name}: rows must be contiguous, and lie in one or two dimensions")


def _plain(t, name: str, shape: Tuple[int, ...], dtype) -> Optional[int]:
    """Pointer of an optional contiguous tensor of this shape and type."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous, {dtype}, of shape {tuple(shape)}")
    return t.data_ptr()


def _gpu_of(*tensors) -> int:
    """Index of the GPU that all the tensors are on."""
    index = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ValueError("all tensors must be on one GPU")
    if index < 0:
        raise ValueError("all tensors must be on one GPU")
    return index


def _launch(gpu: int, fn, *args) -> None:
    """fn(*args, torch's current stream of the GPU), with that GPU current."""
    import torch
    if torch.cuda.current_device() != gpu:
        with torch.cuda.device(gpu):
            return _launch(gpu, fn, *args)
    # (the stream's handle alone: torch.cuda.current_stream makes an object around it, 2.7 us of a call's 7)
    rc = fn(*args, torch._C._cuda_getCurrentRawStream(gpu))
    if rc != ACC_OK:
        raise AccordionError(rc, _lib.accordion_operator_error().decode())


def _workspace(gpu: int, fn, cfg, given, *which):
    """(tensor or None, pointer, bytes) of the workspace of a call: as given, or from torch's allocator for the current stream."""
    n = C.c_size_t(0)
    rc = fn(C.byref(cfg), *which, C.byref(n))
    if rc != ACC_OK:
        raise AccordionError(rc, _lib.accordion_operator_error().decode())
    if given is None:
        if n.value == 0:
            return None, None, 0
        import torch
        given = torch.empty(n.value, dtype=torch.uint8, device=f"cuda:{gpu}")
    elif given.get_device() != gpu or not given.is_contiguous():
        raise ValueError("workspace must be contiguous and on the tensors' GPU")
    return given, given.data_ptr(), given.numel() * given.element_size()


def _embedding(ids, table, out, scale: float, accumulate: bool) -> acc_embedding:
    bits = _INDEX_BITS.get(ids.dtype)
    if bits is None or not ids.is_contiguous():
        raise ValueError("ids must be contiguous int32 or int64")
    vocab, dim, table_stride = _rows_of(table, "table")
    tokens, width, out_stride = _rows_of(out, "out")
    if width != dim or tokens != ids.numel() or table.dim() != 2:
        raise ValueError("ids, table and out do not fit together")
    return acc_embedding(vocab, dim, tokens, table_stride, out_stride, bits, _type_of(table, "table"), _type_of(out, "out"),
                         accumulate, scale)


def embedding_forward(ids, table, out, scale: float = 1.0) -> None:
    """out[t, :] = scale * table[ids[t], :]; ids outside the table give zeros."""
    lib = load_library()
    cfg = _embedding(ids, table, out, scale, False)
    _launch(_gpu_of(ids, table, out), lib.accordion_embedding_forward, C.byref(cfg), ids.data_ptr(), table.data_ptr(), out.data_ptr())


def embedding_backward(ids, grad_out, grad_table, scale: float = 1.0, accumulate: bool = False, workspace=None) -> None:
    """grad_table[v, :] (+)= scale * sum of grad_out[t, :] over the t with ids[t] == v; grad_table is float32."""
    lib = load_library()
    cfg = _embedding(ids, grad_table, grad_out, scale, accumulate)
    _need(cfg.table_type == ACC_FLOAT, "grad_table must be float32")
    gpu = _gpu_of(ids, grad_out, grad_table)
    held, ws, n = _workspace(gpu, lib.accordion_embedding_workspace_bytes, cfg, workspace)
    _launch(gpu, lib.accordion_embedding_backward, C.byref(cfg), ids.data_ptr(), grad_out.data_ptr(), grad_table.data_ptr(), ws, n)


def layernorm_forward(x, weight, bias, y, mean=None, rstd=None, eps: float = 1e-5) -> None:
    """y = (x - mean) rstd weight + bias over the last dimension; bias may be None; mean and rstd are written if given."""
    import torch
    lib = load_library()
    rows, dim, x_stride = _rows_of(x, "x")
    y_rows, y_dim, y_stride = _rows_of(y, "y")
    _need(y_rows == rows and y_dim == dim and y.dtype == x.dtype, "x and y do not fit together")
    f = torch.float32
    w, b = _plain(weight, "weight", (dim,), f), _plain(bias, "bias", (dim,), f)
    m, r = _plain(mean, "mean", (rows,), f), _plain(rstd, "rstd", (rows,), f)
    cfg = acc_layernorm(rows, dim, x_stride, y_stride, 0, _type_of(x, "x"), 0, eps)
    _launch(_gpu_of(x, weight, bias, y, mean, rstd), lib.accordion_layernorm_forward, C.byref(cfg), x.data_ptr(), w, b, y.data_ptr(),
            m, r)


def layernorm_backward(grad_y, x, weight, mean, rstd, grad_x, grad_weight, grad_bias=None, accumulate: bool = False,
                       workspace=None) -> None:
    """Gradients of layernorm_forward; grad_bias may be None; accumulate adds to grad_weight and grad_bias."""
    import torch
    lib = load_library()
    rows, dim, x_stride = _rows_of(x, "x")
    g_rows, g_dim, g_stride = _rows_of(grad_y, "grad_y")
    d_rows, d_dim, d_stride = _rows_of(grad_x, "grad_x")
    _need(g_rows == d_rows == rows and g_dim == d_dim == dim and grad_y.dtype == grad_x.dtype == x.dtype,
          "x, grad_y and grad_x do not fit together")
    f = torch.float32
    w, m, r = _plain(weight, "weight", (dim,), f), _plain(mean, "mean", (rows,), f), _plain(rstd, "rstd", (rows,), f)
    dw, db = _plain(grad_weight, "grad_weight", (dim,), f), _plain(grad_bias, "grad_bias", (dim,), f)
    cfg = acc_layernorm(rows, dim, x_stride, g_stride, d_stride, _type_of(x, "x"), accumulate, 0.0)
    gpu = _gpu_of(x, grad_y, weight, mean, rstd, grad_x, grad_weight, grad_bias)
    held, ws, n = _workspace(gpu, lib.accordion_layernorm_workspace_bytes, cfg, workspace)
    _launch(gpu, lib.accordion_layernorm_backward, C.byref(cfg), grad_y.data_ptr(), x.data_ptr(), w, m, r, grad_x.data_ptr(), dw, db,
            ws, n)


def _steps_of(t, name: str, like) -> Tuple[int, int]:
    """(elements between sequences, between steps) of a batch x steps x channels tensor."""
    if t.shape != like.shape or t.dtype != like.dtype:
        raise ValueError(f"{name} must have gate's shape and type")
    batch, step, channel = t.stride()
    if channel != 1 and t.shape[2] > 1:
        raise ValueError(f"{name}: the channels of a step must be contiguous")
    return batch, step


def recurrence_forward(gate, input, out, h0=None, h_last=None, lengths=None, workspace=None) -> None:
    """h_t = sigmoid(gate_t) h_{t-1} + sigmoid(-gate_t) input_t along dimension 1 of batch x steps x channels tensors;
    out gets every h, h_last (batch x channels, float32) the last one.  steps = 1 with h0 and h_last: one token."""
    import torch
    lib = load_library()
    _need(gate.dim() == 3, "gate must be batch x steps x channels")
    batch, steps, channels = gate.shape
    cfg = acc_recurrence(batch, steps, channels, *_steps_of(gate, "gate", gate), *_steps_of(input, "input", gate),
                         *_steps_of(out, "out", gate), 0, 0, 0, 0, 0, 0, _type_of(gate, "gate"))
    ends, f = (batch, channels), torch.float32
    first, last = _plain(h0, "h0", ends, f), _plain(h_last, "h_last", ends, f)
    n_steps = _plain(lengths, "lengths", (batch,), torch.int32)
    gpu = _gpu_of(gate, input, out, h0, h_last, lengths)
    held, ws, n = _workspace(gpu, lib.accordion_recurrence_workspace_bytes, cfg, workspace)
    _launch(gpu, lib.accordion_recurrence_forward, C.byref(cfg), gate.data_ptr(), input.data_ptr(), first, n_steps, out.data_ptr(),
            last, ws, n)


def recurrence_backward(gate, input, out, grad_out, grad_gate, grad_input, h0=None, grad_last=None, grad_h0=None,
                        lengths=None, workspace=None) -> None:
    """Gradients of recurrence_forward; out is what it wrote, grad_last the gradient of h_last (None: zeros)."""
    import torch
    lib = load_library()
    _need(gate.dim() == 3, "gate must be batch x steps x channels")
    batch, steps, channels = gate.shape
    cfg = acc_recurrence(batch, steps, channels, *_steps_of(gate, "gate", gate), *_steps_of(input, "input", gate),
                         *_steps_of(out, "out", gate), *_steps_of(grad_gate, "grad_gate", gate),
                         *_steps_of(grad_input, "grad_input", gate), *_steps_of(grad_out, "grad_out", gate),
                         _type_of(gate, "gate"))
    ends, f = (batch, channels), torch.float32
    first, last, dh0 = _plain(h0, "h0", ends, f), _plain(grad_last, "grad_last", ends, f), _plain(grad_h0, "grad_h0", ends, f)
    n_steps = _plain(lengths, "lengths", (batch,), torch.int32)
    gpu = _gpu_of(gate, input, out, grad_out, grad_gate, grad_input, h0, grad_last, grad_h0, lengths)
    held, ws, n = _workspace(gpu, lib.accordion_recurrence_workspace_bytes, cfg, workspace)
    _launch(gpu, lib.accordion_recurrence_backward, C.byref(cfg), gate.data_ptr(), input.data_ptr(), out.data_ptr(), first, n_steps,
            grad_out.data_ptr(), last, grad_gate.data_ptr(), grad_input.data_ptr(), dh0, ws, n)


def _parts_of(t, name: str, shape, dtype, whole) -> Tuple[int, int]:
    """(elements between sequences, between steps) of a batch x steps x ... tensor whose steps' elements are contiguous; whole: of one that
    is contiguous throughout."""
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype}, of shape {tuple(shape)}")
    if t.is_contiguous():
        return whole
    stride = t.stride()
    if len(stride) == 3:
        apart = stride[2] != 1 and shape[2] > 1
    else:
        apart = (stride[3] != 1 and shape[3] > 1) or (stride[2] != shape[3] and shape[2] > 1)
    if apart:
        raise ValueError(f"{name}: the elements of a step must be contiguous")
    return stride[:2]


def _convolution(x, weight, out, name: str, silu: bool, accumulate: bool, grad_x=None):
    """(config, shapes of weight, of a channels' vector, of a state)."""
    shape, kind = x.shape, x.dtype
    _need(len(shape) == 3, "x must be batch x steps x channels")
    _need(weight.dim() == 2, "weight must be channels x width")
    batch, steps, channels = shape
    width, whole = weight.shape[1], (max(steps, 1) * channels, channels)
    last = (0, 0) if grad_x is None else _parts_of(grad_x, "grad_x", shape, kind, whole)
    cfg = acc_convolution(batch, steps, channels, *_parts_of(x, "x", shape, kind, whole), *_parts_of(out, name, shape, kind, whole), *last,
                          width, _type_of(x, "x"), silu, accumulate)
    return cfg, (channels, width), (channels,), (batch, width - 1, channels)


def convolution_forward(x, weight, out, bias=None, state=None, last=None, lengths=None, silu: bool = False) -> None:
    """out_t = act(bias + sum_j weight[:, j] x_{t - width + 1 + j}) along dimension 1 of batch x steps x channels tensors, act the
    identity or SiLU; state (batch x (width - 1) x channels, float32): the inputs in front (None: zeros); last gets those of a call that
    continues.  steps = 1 with state and last: one token."""
    lib = load_library()
    cfg, wide, flat, ends = _convolution(x, weight, out, "out", silu, False)
    f = _FLOAT32
    w, b = _plain(weight, "weight", wide, f), _plain(bias, "bias", flat, f)
    first, end, n_steps = _plain(state, "state", ends, f), _plain(last, "last", ends, f), _plain(lengths, "lengths", ends[:1], _INT32)
    _launch(_gpu_of(x, weight, out, bias, state, last, lengths), lib.accordion_convolution_forward, C.byref(cfg), x.data_ptr(), w, b, first,
            n_steps, out.data_ptr(), end)


def convolution_backward(x, weight, grad_out, grad_x, grad_weight, bias=None, grad_bias=None, state=None, grad_last=None, grad_state=None,
                         lengths=None, silu: bool = False, accumulate: bool = False, workspace=None) -> None:
    """Gradients of convolution_forward; grad_last is the gradient of last (None: zeros); accumulate adds to grad_weight and grad_bias."""
    lib = load_library()
    cfg, wide, flat, ends = _convolution(x, weight, grad_out, "grad_out", silu, accumulate, grad_x)
    f = _FLOAT32
    w, b, first = _plain(weight, "weight", wide, f), _plain(bias, "bias", flat, f), _plain(state, "state", ends, f)
    dw, db = _plain(grad_weight, "grad_weight", wide, f), _plain(grad_bias, "grad_bias", flat, f)
    dl, ds = _plain(grad_last, "grad_last", ends, f), _plain(grad_state, "grad_state", ends, f)
    n_steps = _plain(lengths, "lengths", ends[:1], _INT32)
    gpu = _gpu_of(x, weight, grad_out, grad_x, grad_weight, bias, grad_bias, state, grad_last, grad_state, lengths)
    held, ws, n = _workspace(gpu, lib.accordion_convolution_workspace_bytes, cfg, workspace)
    _launch(gpu, lib.accordion_convolution_backward, C.byref(cfg), x.data_ptr(), w, b, first, n_steps, grad_out.data_ptr(), dl,
            grad_x.data_ptr(), dw, db, ds, ws, n)


def _scan(x, delta, a, b, c, out, name: str, gate, softplus: bool, accumulate: bool, grads=None):
    """(config, shapes of a, of a channels' vector, of a state); grads: of x, delta, b, c and gate."""
    shape, kind, shared = x.shape, x.dtype, b.shape
    _need(len(shape) == 3, "x must be batch x steps x channels")
    _need(a.dim() == 2, "a must be channels x states")
    _need(len(shared) == 3 or len(shared) == 4, "b must be batch x steps x groups x states")
    batch, steps, channels = shape
    states, groups = a.shape[1], shared[2] if len(shared) == 4 else 1
    if shared[0] != batch or shared[1] != steps or shared[-1] != states:
        raise ValueError(f"b must be {batch} x {steps} x groups x {states}")
    row = groups * states
    whole, part = (max(steps, 1) * channels, channels), (max(steps, 1) * row, row)
    near = (*_parts_of(x, "x", shape, kind, whole), *_parts_of(delta, "delta", shape, kind, whole), *_parts_of(b, "b", shared, kind, part),
            *_parts_of(c, "c", shared, kind, part), *((0, 0) if gate is None else _parts_of(gate, "gate", shape, kind, whole)),
            *_parts_of(out, name, shape, kind, whole))
    if grads is None:
        far = (0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    else:
        gx, gdelta, gb, gc, ggate = grads
        _need((gate is None) == (ggate is None), "gate and grad_gate go together")
        far = (*_parts_of(gx, "grad_x", shape, kind, whole), *_parts_of(gdelta, "grad_delta", shape, kind, whole),
               *_parts_of(gb, "grad_b", shared, kind, part), *_parts_of(gc, "grad_c", shared, kind, part),
               *((0, 0) if ggate is None else _parts_of(ggate, "grad_gate", shape, kind, whole)))
    cfg = acc_scan(batch, steps, channels, *near, *far, states, groups, _type_of(x, "x"), softplus, accumulate)
    return cfg, (channels, states), (channels,), (batch, channels, states)


def _pointer(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def scan_forward(x, delta, a, b, c, out, d=None, gate=None, delta_bias=None, softplus: bool = False, h0=None, h_last=None, lengths=None,
                 workspace=None) -> None:
    """h_t = exp(dt_t a) h_{t-1} + dt_t b_t x_t, out_t = (c_t . h_t + d x_t) silu(gate_t) along dimension 1 of batch x steps x channels
    tensors x, delta, gate and out; dt = delta + delta_bias, or its softplus; a: channels x states, b and c: batch x steps x groups x
    states (without the third dimension: one group); h0, h_last: batch x channels x states, float32.  steps = 1 with h0 and h_last: one
    token."""
    lib = load_library()
    cfg, wide, flat, ends = _scan(x, delta, a, b, c, out, "out", gate, softplus, False)
    f = _FLOAT32
    decay, skip, shift = _plain(a, "a", wide, f), _plain(d, "d", flat, f), _plain(delta_bias, "delta_bias", flat, f)
    first, last, n_steps = _plain(h0, "h0", ends, f), _plain(h_last, "h_last", ends, f), _plain(lengths, "lengths", ends[:1], _INT32)
    gpu = _gpu_of(x, delta, a, b, c, out, d, gate, delta_bias, h0, h_last, lengths)
    held, ws, n = _workspace(gpu, lib.accordion_scan_workspace_bytes, cfg, workspace, 0)
    _launch(gpu, lib.accordion_scan_forward, C.byref(cfg), x.data_ptr(), delta.data_ptr(), decay, b.data_ptr(), c.data_ptr(), skip,
            _pointer(gate), shift, first, n_steps, out.data_ptr(), last, ws, n)


def scan_backward(x, delta, a, b, c, grad_out, grad_x, grad_delta, grad_a, grad_b, grad_c, d=None, grad_d=None, gate=None, grad_gate=None,
                  delta_bias=None, grad_delta_bias=None, softplus: bool = False, h0=None, grad_last=None, grad_h0=None, lengths=None,
                  accumulate: bool = False, workspace=None) -> None:
    """Gradients of scan_forward, from its inputs alone; grad_last is the gradient of h_last (None: zeros); accumulate adds to grad_a,
    grad_d and grad_delta_bias."""
    lib = load_library()
    cfg, wide, flat, ends = _scan(x, delta, a, b, c, grad_out, "grad_out", gate, softplus, accumulate,
                                  (grad_x, grad_delta, grad_b, grad_c, grad_gate))
    f = _FLOAT32
    decay, skip, shift = _plain(a, "a", wide, f), _plain(d, "d", flat, f), _plain(delta_bias, "delta_bias", flat, f)
    da, dd = _plain(grad_a, "grad_a", wide, f), _plain(grad_d, "grad_d", flat, f)
    dbias = _plain(grad_delta_bias, "grad_delta_bias", flat, f)
    first, dl, dh = _plain(h0, "h0", ends, f), _plain(grad_last, "grad_last", ends, f), _plain(grad_h0, "grad_h0", ends, f)
    n_steps = _plain(lengths, "lengths", ends[:1], _INT32)
    gpu = _gpu_of(x, delta, a, b, c, grad_out, grad_x, grad_delta, grad_a, grad_b, grad_c, d, grad_d, gate, grad_gate, delta_bias,
                  grad_delta_bias, h0, grad_last, grad_h0, lengths)
    held, ws, n = _workspace(gpu, lib.accordion_scan_workspace_bytes, cfg, workspace, 1)
    _launch(gpu, lib.accordion_scan_backward, C.byref(cfg), x.data_ptr(), delta.data_ptr(), decay, b.data_ptr(), c.data_ptr(), skip,
            _pointer(gate), shift, first, n_steps, grad_out.data_ptr(), dl, grad_x.data_ptr(), grad_delta.data_ptr(), da, grad_b.data_ptr(),
            grad_c.data_ptr(), dd, _pointer(grad_gate), dbias, dh, ws, n)


def _logprob(logits, targets, top: int, bits: int, grad_logits=None) -> acc_logprob:
    rows, vocab, stride = _rows_of(logits, "logits")
    grad_stride = 0
    if grad_logits is not None:
        g_rows, g_vocab, grad_stride = _rows_of(grad_logits, "grad_logits")
        _need(g_rows == rows and g_vocab == vocab and grad_logits.dtype is logits.dtype, "logits and grad_logits do not fit together")
    if targets is not None:
        bits = _INDEX_BITS.get(targets.dtype)
        _need(bits is not None, "targets must be int32 or int64")
        _need(targets.numel() == rows and targets.is_contiguous(), "targets must be contiguous, one per row of logits")
    return acc_logprob(rows, vocab, stride, grad_stride, bits, _type_of(logits, "logits"), top)


def logprob_forward(logits, targets=None, logprob=None, lse=None, entropy=None, top_logprobs=None, top_ids=None, workspace=None) -> None:
    """Per row of logits: logprob of the row's target (zero where that is outside the vocabulary), lse the logarithm of the sum of
    exponentials, the entropy, and the most probable tokens' log probabilities and ids (rows x top), the largest first, of equal logits the
    lowest id first.  What is None is not computed."""
    lib = load_library()
    _need((top_logprobs is None) == (top_ids is None), "top_logprobs and top_ids go together")
    _need(logprob is None or targets is not None, "logprob needs targets")
    top, bits = 0, 64
    if top_ids is not None:
        bits = _INDEX_BITS.get(top_ids.dtype)
        _need(bits is not None and top_ids.dim() == 2, "top_ids must be int32 or int64, rows x top")
        _need(targets is None or targets.dtype is top_ids.dtype, "top_ids must be of targets' type")
        top = top_ids.shape[1]
    cfg = _logprob(logits, targets, top, bits)
    f, rows = _FLOAT32, (cfg.rows,)
    lp, ls, en = _plain(logprob, "logprob", rows, f), _plain(lse, "lse", rows, f), _plain(entropy, "entropy", rows, f)
    tv = ti = None
    if top_ids is not None:
        best = (cfg.rows, top)
        tv, ti = _plain(top_logprobs, "top_logprobs", best, f), _plain(top_ids, "top_ids", best, top_ids.dtype)
    gpu = _gpu_of(logits, targets, logprob, lse, entropy, top_logprobs, top_ids)
    held, ws, n = _workspace(gpu, lib.accordion_logprob_workspace_bytes, cfg, workspace)
    _launch(gpu, lib.accordion_logprob_forward, C.byref(cfg), logits.data_ptr(), _pointer(targets), lp, ls, en, tv, ti, ws, n)


def logprob_backward(logits, targets, lse, grad_logprob, grad_logits, entropy=None, grad_entropy=None) -> None:
    """The logits' gradient from those of logprob (may be None) and, with grad_entropy, of the entropy; lse and entropy are what the
    forward pass wrote.  grad_logits may be logits."""
    lib = load_library()
    cfg = _logprob(logits, targets, 0, 64, grad_logits)
    f, rows = _FLOAT32, (cfg.rows,)
    ls, dl = _plain(lse, "lse", rows, f), _plain(grad_logprob, "grad_logprob", rows, f)
    en, de = _plain(entropy, "entropy", rows, f), _plain(grad_entropy, "grad_entropy", rows, f)
    _launch(_gpu_of(logits, targets, lse, grad_logprob, grad_logits, entropy, grad_entropy), lib.accordion_logprob_backward, C.byref(cfg),
            logits.data_ptr(), _pointer(targets), ls, dl, en, de, grad_logits.data_ptr())


def adamw_state_elements(sizes: Sequence[int], state_bits: int = 32) -> int:
    """Elements of each moment of adamw_step for tensors of these sizes; host arithmetic only."""
    lib = load_library()
    arr = (C.c_int64 * max(1, len(sizes)))(*sizes)
    return _state_elements(lib, acc_adamw(n_tensors=len(sizes), state_bits=state_bits, sizes_host=arr))


def _state_elements(lib, cfg: acc_adamw) -> int:
    out = C.c_int64(0)
    rc = lib.accordion_adamw_state_elements(C.byref(cfg), C.byref(out))
    if rc != ACC_OK:
        raise AccordionError(rc, lib.accordion_operator_error().decode())
    return out.value


def adamw_state(sizes: Sequence[int], state_bits: int = 32, device: str = "cuda:0"):
    """(m, v, m_scale, v_scale) before the first step: float32 moments and no scales, or with 8 bits e4m3 codes (of
    sqrt(v) in v's place) and a float32 scale for each block of ACC_ADAMW_BLOCK elements."""
    import torch
    n = adamw_state_elements(sizes, state_bits)
    if state_bits == 32:
        return tuple(torch.zeros(n, device=device) for _ in range(2)) + (None, None)
    return (*(torch.zeros(n, dtype=torch.uint8, device=device).view(torch.float8_e4m3fn) for _ in range(2)),
            *(torch.zeros(n // ACC_ADAMW_BLOCK, device=device) for _ in range(2)))


def _c_array(kind, code: str, values):
    """A C array of numbers (through array.array: filling a ctypes array item by item takes twice as long)."""
    held = array.array(code, values)
    return (kind * len(held)).from_buffer(held)


def _tensors_of(tensors: Sequence, name: str):
    """(sizes, pointers, type, GPU) of contiguous tensors of one type on one GPU."""
    import torch
    t = torch.Tensor
    kinds, gpus = {x.dtype for x in tensors}, set(map(t.get_device, tensors))
    _need(len(kinds) == 1, f"{name} must be of one type")
    _need(len(gpus) == 1, "all tensors must be on one GPU")
    _need(all(map(t.is_contiguous, tensors)), f"{name} must be contiguous")
    return list(map(t.numel, tensors)), _c_array(C.c_void_p, "Q", map(t.data_ptr, tensors)), kinds.pop(), gpus.pop()


def adamw_step(weights: Sequence, grads: Sequence, state, lr: float, step: int, weight_decay=0.0,
               betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8, copies: Optional[Sequence] = None,
               grad_scale=None, dither: bool = False) -> None:
    """One AdamW step over all tensors (contiguous; all weights of one type, all gradients of one type).  state: as
    adamw_state made it for their sizes; weight_decay: one number or one per tensor; copies: bfloat16 tensors that get the
    new weights too; grad_scale: a float32 element on the GPU that multiplies every gradient.  8-bit moments are rounded to nearest
    where betas are at most (0.9, 0.95), and with thresholds that change with the step, so that they follow their averages, beyond;
    dither: with thresholds everywhere (gradients that hardly vary from step to step)."""
    import torch
    lib = load_library()
    count = len(weights)
    _need(len(grads) == count and (copies is None or len(copies) == count), "weights, grads and copies must be of one length")
    if count == 0:
        return
    m, v, m_scale, v_scale = state
    bits = 32 if m_scale is None else 8
    sizes, w_ptrs, _, gpu = _tensors_of(weights, "weights")
    g_sizes, g_ptrs, _, g_gpu = _tensors_of(grads, "grads")
    _need(sizes == g_sizes, "weights and grads do not fit together")
    _need(gpu == g_gpu, "all tensors must be on one GPU")
    c_ptrs = None
    if copies is not None:
        kept = [c for c in copies if c is not None]
        if kept:
            c_sizes, _, c_type, c_gpu = _tensors_of(kept, "copies")
            _need(c_type == torch.bfloat16 and c_gpu == gpu and c_sizes == [n for n, c in zip(sizes, copies) if c is not None],
                  "a copy must be bfloat16, of its tensor's size, on its GPU")
            c_ptrs = _c_array(C.c_void_p, "Q", [0 if c is None else c.data_ptr() for c in copies])
    cfg = acc_adamw(count, _type_of(weights[0], "weights"), _type_of(grads[0], "grads"), bits, _c_array(C.c_int64, "q", sizes), None, lr,
                    betas[0], betas[1], eps, step, dither)
    elements = _state_elements(lib, cfg)
    held = torch.float32 if bits == 32 else torch.float8_e4m3fn
    mp, vp = _plain(m, "m", (elements,), held), _plain(v, "v", (elements,), held)
    blocks = (elements // ACC_ADAMW_BLOCK,)
    ms, vs = _plain(m_scale, "m_scale", blocks, torch.float32), _plain(v_scale, "v_scale", blocks, torch.float32)
    _need(grad_scale is None or (grad_scale.dtype == torch.float32 and grad_scale.numel() == 1), "grad_scale must be one float32 element")
    if not isinstance(weight_decay, (int, float)):
        _need(len(weight_decay) == count, "one weight decay per tensor")
        cfg.weight_decay_host = _c_array(C.c_float, "f", weight_decay)
    elif weight_decay != 0.0:
        cfg.weight_decay_host = _c_array(C.c_float, "f", [weight_decay] * count)
    _launch(_gpu_of(weights[0], m, v, m_scale, v_scale, grad_scale), lib.accordion_adamw_step, C.byref(cfg), w_ptrs, g_ptrs, c_ptrs, mp,
            vp, ms, vs, grad_scale.data_ptr() if grad_scale is not None else None)


class Accordion:
    """One context.  Methods carry the names of the C entry points they call."""

    def __init__(self, method: int, layers: Sequence, n_workers: int, level_crit: int,
                 level_noncrit: int, k_den: int = 100, eta: float = 0.5, initial_level: int = 1,
                 q_init: Optional[np.ndarray] = None, device: str = "cuda:0",
                 batch_multiplier: int = 1, batch_monotone: int = 1, detector: int = 0,
                 static_workspace: bool = False):
        """static_workspace: create the context with accordion_init_static (the library's own
        static device array is the workspace; nothing is allocated for it here)."""
        import torch  # device memory and the stream handle only

        self._lib = load_library()
        self._torch = torch
        self.cfg, self._keep = make_config(method, layers, n_workers, level_crit, level_noncrit,
                                           k_den, eta, initial_level, None, batch_multiplier,
                                           batch_monotone, detector)
        self.method, self.n_workers, self.n_layers = method, n_workers, len(layers)
        self.n_params = int(self.cfg.n_params)
        self.layers = [(l.offset, l.rows, l.cols, l.is_matrix) if hasattr(l, "offset") else tuple(l)
                       for l in layers]
        self.device = torch.device(device)
        nbytes = accordion_workspace_bytes(self.cfg)
        self.workspace_bytes = nbytes
        self.workspace = None
        if not static_workspace:
            self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            base = self.workspace.data_ptr()
            self._ws_ptr = (base + 255) // 256 * 256
        with torch.cuda.device(self.device):
            self.stream = torch.cuda.current_stream().cuda_stream
        qptr = None
        if method == ACC_POWERSGD:
            q = np.ascontiguousarray(q_init, dtype=np.float32)
            self._q_keep = q
            qptr = q.ctypes.data_as(C.c_void_p)
        ctx = C.c_void_p(None)
        if static_workspace:
            with torch.cuda.device(self.device):
                rc = self._lib.accordion_init_static(C.byref(self.cfg), qptr, C.c_void_p(self.stream), C.byref(ctx))
        else:
            rc = self._lib.accordion_init(C.byref(self.cfg), C.c_void_p(self._ws_ptr), nbytes, qptr,
                                          C.c_void_p(self.stream), C.byref(ctx))
        _check(self._lib, None, rc)
        self.ctx = ctx

    # -- the hot path ---------------------------------------------------------------------
    def compress_step(self, worker: int, grad, phase: int) -> None:
        ptr = C.c_void_p(grad.data_ptr()) if grad is not None else None
        _check(self._lib, self.ctx, self._lib.accordion_compress_step(self.ctx, worker, ptr, phase))

    def aggregate(self, phase: int) -> None:
        _check(self._lib, self.ctx, self._lib.accordion_aggregate(self.ctx, phase))

    def decompress(self, out) -> None:
        _check(self._lib, self.ctx, self._lib.accordion_decompress(self.ctx, C.c_void_p(out.data_ptr())))

    def step_all(self, grads: Sequence, out) -> None:
        arr = (C.c_void_p * len(grads))(*[g.data_ptr() for g in grads])
        _check(self._lib, self.ctx,
               self._lib.accordion_step_all(self.ctx, arr, C.c_void_p(out.data_ptr())))

    def decompress_update(self, weights, velocity, lr: float, momentum: float, weight_decay: float = 0.0) -> None:
        _check(self._lib, self.ctx, self._lib.accordion_decompress_update(
            self.ctx, C.c_void_p(weights.data_ptr()), C.c_void_p(velocity.data_ptr()), lr, momentum, weight_decay))

    def step_all_update(self, grads: Sequence, weights, velocity, lr: float, momentum: float,
                        weight_decay: float = 0.0) -> None:
        arr = (C.c_void_p * len(grads))(*[g.data_ptr() for g in grads])
        _check(self._lib, self.ctx, self._lib.accordion_step_all_update(
            self.ctx, arr, C.c_void_p(weights.data_ptr()), C.c_void_p(velocity.data_ptr()), lr, momentum, weight_decay))

    def topk_overlap(self, worker_a: int, worker_b: int) -> Tuple[np.ndarray, np.ndarray]:
        common = np.zeros(self.n_layers, np.int64)
        kept = np.zeros(self.n_layers, np.int64)
        _check(self._lib, self.ctx, self._lib.accordion_topk_overlap(
            self.ctx, worker_a, worker_b, common.ctypes.data_as(C.POINTER(C.c_int64)),
            kept.ctypes.data_as(C.POINTER(C.c_int64))))
        return common, kept

    def set_stream(self, cuda_stream: int) -> None:
        """cuda_stream: the raw stream handle (torch.cuda.Stream.cuda_stream); 0 = default stream."""
        _check(self._lib, self.ctx, self._lib.accordion_set_stream(self.ctx, C.c_void_p(cuda_stream)))
        self.stream = cuda_stream

    def batch_status(self) -> dict:
        lv, pend, last = C.c_int32(0), C.c_int32(0), C.c_int32(0)
        ex, ms = C.c_int64(0), C.c_int64(0)
        _check(self._lib, self.ctx, self._lib.accordion_batch_status(
            self.ctx, C.byref(lv), C.byref(pend), C.byref(last), C.byref(ex), C.byref(ms)))
        return dict(level=lv.value, pending=pend.value, last_batch=last.value, exchanges=ex.value,
                    micro_steps=ms.value)

    def detect_regime(self, lr_curr: float, lr_next: float) -> None:
        _check(self._lib, self.ctx, self._lib.accordion_detect_regime(self.ctx, lr_curr, lr_next))

    def flush(self) -> None:
        _check(self._lib, self.ctx, self._lib.accordion_flush(self.ctx))

    def reset_accumulator(self) -> None:
        _check(self._lib, self.ctx, self._lib.accordion_reset_accumulator(self.ctx))

    # -- read-backs -----------------------------------------------------------------------
    def get_levels(self) -> np.ndarray:
        out = np.zeros(self.n_layers, dtype=np.int32)
        _check(self._lib, self.ctx, self._lib.accordion_get_levels(self.ctx, out.ctypes.data_as(C.c_void_p)))
        return out

    def get_norms(self) -> Tuple[np.ndarray, np.ndarray]:
        old = np.zeros(self.n_layers, dtype=np.float32)
        cur = np.zeros(self.n_layers, dtype=np.float32)
        _check(self._lib, self.ctx, self._lib.accordion_get_norms(
            self.ctx, old.ctypes.data_as(C.c_void_p), cur.ctypes.data_as(C.c_void_p)))
        return old, cur

    def get_payload(self, worker: int, layer: int) -> Tuple[np.ndarray, np.ndarray]:
        _, r, c, _ = self.layers[layer]
        cap = r * c
        idx = np.zeros(cap, dtype=np.int32)
        val = np.zeros(cap, dtype=np.float32)
        cnt = C.c_int64(0)
        _check(self._lib, self.ctx, self._lib.accordion_get_payload(
            self.ctx, worker, layer, idx.ctypes.data_as(C.c_void_p), val.ctypes.data_as(C.c_void_p),
            cap, C.byref(cnt)))
        k = int(cnt.value)
        return idx[:k].copy(), val[:k].copy()

    def get_factors(self, layer: int) -> Tuple[np.ndarray, np.ndarray]:
        _, r, c, _ = self.layers[layer]
        p = np.zeros(r * ACC_MAX_RANK, dtype=np.float32)
        q = np.zeros(c * ACC_MAX_RANK, dtype=np.float32)
        rank = C.c_int32(0)
        _check(self._lib, self.ctx, self._lib.accordion_get_factors(
            self.ctx, layer, p.ctypes.data_as(C.c_void_p), q.ctypes.data_as(C.c_void_p), C.byref(rank)))
        k = int(rank.value)
        return p[:r * k].reshape(r, k).copy(), q[:c * k].reshape(c, k).copy()

    def payload_words(self) -> Tuple[int, int]:
        a, b = C.c_int64(0), C.c_int64(0)
        _check(self._lib, self.ctx, self._lib.accordion_payload_words(self.ctx, C.byref(a), C.byref(b)))
        return int(a.value), int(b.value)

    def topk_stats(self) -> Tuple[int, int]:
        """(layers whose Delta was read again, because the guess missed or the lists were too short; layers sent to the
        sweeps by a large tie class) since init."""
        a, b = C.c_int64(0), C.c_int64(0)
        _check(self._lib, self.ctx, self._lib.accordion_topk_stats(self.ctx, C.byref(a), C.byref(b)))
        return int(a.value), int(b.value)

    def topk_short_lists(self) -> int:
        """Those of topk_stats()[0] whose lists were merely too short: the guess held, the layer was decided without sweeps."""
        a = C.c_int64(0)
        _check(self._lib, self.ctx, self._lib.accordion_topk_short_lists(self.ctx, C.byref(a)))
        return int(a.value)

    def state_bytes(self) -> int:
        out = C.c_size_t(0)
        _check(self._lib, self.ctx, self._lib.accordion_state_bytes(self.ctx, C.byref(out)))
        return int(out.value)

    def get_state(self) -> np.ndarray:
        buf = np.zeros(self.state_bytes(), dtype=np.uint8)
        _check(self._lib, self.ctx, self._lib.accordion_get_state(
            self.ctx, buf.ctypes.data_as(C.c_void_p), buf.nbytes))
        return buf

    def set_state(self, buf: np.ndarray) -> None:
        buf = np.ascontiguousarray(buf, dtype=np.uint8)
        _check(self._lib, self.ctx, self._lib.accordion_set_state(
            self.ctx, buf.ctypes.data_as(C.c_void_p), buf.nbytes))

    def set_profiling(self, enable) -> None:
        """0 / False: off; 1 / True: every kernel; 2: only the fused error-feedback pass; 3: every
        fourth launch of that pass."""
        _check(self._lib, self.ctx, self._lib.accordion_set_profiling(self.ctx, int(enable)))

    def get_profile(self) -> dict:
        """{kernel name: (total milliseconds, launches)} since profiling was switched on."""
        out = {}
        for s in range(ACC_N_STAGES):
            if self._lib.accordion_stage_name(s) is None:
                break
            ms, n = C.c_double(0.0), C.c_int64(0)
            _check(self._lib, self.ctx, self._lib.accordion_get_profile(self.ctx, s, C.byref(ms), C.byref(n)))
            if n.value:
                out[self._lib.accordion_stage_name(s).decode()] = (float(ms.value), int(n.value))
        return out

    # -- state blob helpers (layout documented in include/accordion.h) ---------------------
    def q_total(self) -> int:
        if self.method != ACC_POWERSGD:
            return 0
        rmax = max(self.cfg.rank_crit, self.cfg.rank_noncrit)
        return sum(c * rmax for (_, r, c, m) in self.layers if m)

    def unpack_state(self, buf: np.ndarray) -> dict:
        N, W, L = self.n_params, self.n_workers, self.n_layers
        f = buf.view(np.float32)
        pos = 0
        e = f[pos:pos + W * N].reshape(W, N); pos += W * N
        A = f[pos:pos + N]; pos += N
        qt = self.q_total()
        Q = f[pos:pos + qt]; pos += qt
        pending = None
        if self.method == ACC_BATCH:
            pending = int(buf.view(np.int32)[pos]); pos += 1
        norm_old = f[pos:pos + L]; pos += L
        has_old = buf.view(np.int32)[pos:pos + L]; pos += L
        level = buf.view(np.int32)[pos:pos + L]; pos += L
        return dict(e=e, A=A, Q=Q, norm_old=norm_old, has_old=has_old, level=level, pending=pending)

    def pack_state(self, e, A, Q, norm_old, has_old, level, pending: int = 0) -> np.ndarray:
        parts = [np.ascontiguousarray(e, np.float32).reshape(-1).view(np.uint8),
                 np.ascontiguousarray(A, np.float32).view(np.uint8)]
        if self.method == ACC_POWERSGD:
            parts.append(np.ascontiguousarray(Q, np.float32).reshape(-1).view(np.uint8))
        if self.method == ACC_BATCH:
            parts.append(np.array([pending], np.int32).view(np.uint8))
        parts += [np.ascontiguousarray(norm_old, np.float32).view(np.uint8),
                  np.ascontiguousarray(has_old, np.int32).view(np.uint8),
                  np.ascontiguousarray(level, np.int32).view(np.uint8)]
        return np.concatenate(parts)

    def destroy(self) -> None:
        if getattr(self, "ctx", None) is not None and self.ctx.value:
            self._torch.cuda.synchronize(self.device)
            self._lib.accordion_destroy(self.ctx)
            self.ctx = C.c_void_p(None)

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass
