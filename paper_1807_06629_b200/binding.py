"""ctypes binding of libprsgd.so: argument marshalling only.

Every function of include/prsgd.h is available under its own name on `lib`
(e.g. ``lib.prsgd_local_steps``).  The `PRSGD` class wraps a context together
with the torch tensors that own its device memory; its methods are named after
the C calls and do no arithmetic of their own.  There is no CPU fallback: if
the shared library is missing this module raises on import.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np
import torch

from ._build import LIB_PATH

PRSGD_OK = 0
PRECISION_FP32, PRECISION_BF16 = 0, 1
X_FP32, X_BF16 = 0, 1
OPT_FUSED_AVERAGE = 1
OPT_PROFILE = 2
OPT_UPDATE_TILE = 3
OPT_GRAPH = 4
OPT_FUSED_EPILOGUES = 5
OPT_EARLY_LOADS = 6
OPT_NEXT_FORWARD = 7
OPT_DX_IN_UPDATE = 8
OPT_CHECK_FINITE = 9
OPT_SHARED_RESTART = 10
OPT_FORWARD_CHAIN = 11
OPT_WORKER_GROUPS = 12
OPT_DX_SHARED_PAIR = 13
OPT_HEAD_KERNEL = 14
OPT_COMMON_POINT = 15
OPT_SPLIT_BLOCKS = 16
OPT_HEAD_FORWARD = 17
OPT_MERGED_SMALL_AVERAGE = 18
OPT_TILED_WEIGHTS = 19
OPT_OVERLAP_UPDATE = 20
MUON_SCALE_SPECTRAL, MUON_SCALE_RMS = 0, 1
ERR_DEVICE_TIMEOUT, ERR_NONFINITE = -6, -7
KERNEL_FAMILIES = ("forward", "softmax", "dx", "update", "update_average", "average", "misc", "head")
MAX_LAYERS = 16

EXPORTS = [
    "prsgd_layout", "prsgd_workspace_bytes", "prsgd_create", "prsgd_destroy", "prsgd_bind_data",
    "prsgd_upload_data", "prsgd_set_params", "prsgd_set_params_stacked", "prsgd_get_params_stacked",
    "prsgd_get_params", "prsgd_local_steps", "prsgd_average", "prsgd_get_average", "prsgd_get_average_async", "prsgd_get_losses",
    "prsgd_get_draws", "prsgd_set_lr", "prsgd_set_interval", "prsgd_set_active", "prsgd_get_step",
    "prsgd_set_step", "prsgd_set_option", "prsgd_get_launch_count", "prsgd_get_profile", "prsgd_sync", "prsgd_last_error",
    "prsgd_average_rows", "prsgd_draw_block", "prsgd_mean_rows_noalloc", "prsgd_selftest_wait_expiry",
    "prsgd_clear_device_error", "prsgd_enable_momentum", "prsgd_get_velocity_stacked",
    "prsgd_set_worker_offset", "prsgd_partial_sum", "prsgd_assign_rows", "prsgd_stage_data", "prsgd_swap_data",
    "prsgd_alg2_schedule", "prsgd_run_time_varying", "prsgd_run_heterogeneous_epoch",
    "prsgd_set_global_workers", "prsgd_check_finite", "prsgd_local_steps_sum",
    "prsgd_orthogonalize_workspace_bytes", "prsgd_orthogonalize", "prsgd_muon_step", "prsgd_work_status",
    "prsgd_route_workspace_bytes", "prsgd_route", "prsgd_route_grad",
    "prsgd_muon_workspace_bytes", "prsgd_enable_muon", "prsgd_set_balance",
]
NOALLOC_MAX_M = 1 << 20


class ModelSpec(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("dims", C.POINTER(C.c_int32)), ("batch", C.c_int32),
                ("precision", C.c_int32), ("pool_samples", C.c_int64), ("draw_seed", C.c_uint64)]


class Layout(C.Structure):
    _fields_ = [("m", C.c_int64), ("m_pad", C.c_int64), ("w_off", C.c_int64 * MAX_LAYERS),
                ("b_off", C.c_int64 * MAX_LAYERS)]


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it first (python -m paper_1807_06629_b200._build). "
            "There is no fallback path.")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, u64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64
    f32, szt = C.c_float, C.c_size_t
    spec_p, szp = C.POINTER(ModelSpec), C.POINTER(C.c_size_t)
    sig = {
        "prsgd_layout": (C.c_int, [spec_p, C.POINTER(Layout)]),
        "prsgd_workspace_bytes": (C.c_int, [i32, spec_p, szp, szp, szp]),
        "prsgd_create": (C.c_int, [i32, spec_p, C.c_float, i32, vp, vp, vp, vp, C.POINTER(vp)]),
        "prsgd_destroy": (C.c_int, [vp]),
        "prsgd_bind_data": (C.c_int, [vp, vp, i32, vp]),
        "prsgd_upload_data": (C.c_int, [vp, vp, vp]),
        "prsgd_set_params": (C.c_int, [vp, vp, i32, C.c_int]),
        "prsgd_set_params_stacked": (C.c_int, [vp, vp, C.c_int]),
        "prsgd_get_params_stacked": (C.c_int, [vp, vp, C.c_int]),
        "prsgd_get_params": (C.c_int, [vp, vp, i32, C.c_int]),
        "prsgd_local_steps": (C.c_int, [vp, i64]),
        "prsgd_local_steps_sum": (C.c_int, [vp, i64]),
        "prsgd_average": (C.c_int, [vp]),
        "prsgd_get_average": (C.c_int, [vp, vp, C.c_int]),
        "prsgd_get_average_async": (C.c_int, [vp, vp, vp]),
        "prsgd_get_losses": (C.c_int, [vp, vp]),
        "prsgd_get_draws": (C.c_int, [vp, vp]),
        "prsgd_set_lr": (C.c_int, [vp, C.c_float]),
        "prsgd_set_interval": (C.c_int, [vp, i32]),
        "prsgd_set_active": (C.c_int, [vp, vp]),
        "prsgd_get_step": (C.c_int, [vp, C.POINTER(i64)]),
        "prsgd_set_step": (C.c_int, [vp, i64]),
        "prsgd_set_option": (C.c_int, [vp, i32, i64]),
        "prsgd_get_launch_count": (C.c_int, [vp, C.POINTER(i64)]),
        "prsgd_get_profile": (C.c_int, [vp, i32, C.POINTER(C.c_double), C.POINTER(i64)]),
        "prsgd_sync": (C.c_int, [vp]),
        "prsgd_selftest_wait_expiry": (C.c_int, [vp, i32]),
        "prsgd_clear_device_error": (C.c_int, [vp]),
        "prsgd_enable_momentum": (C.c_int, [vp, C.c_float, vp, C.c_int]),
        "prsgd_get_velocity_stacked": (C.c_int, [vp, vp, C.c_int]),
        "prsgd_alg2_schedule": (C.c_int, [i32, i64, C.POINTER(i64), C.POINTER(C.c_float)]),
        "prsgd_run_time_varying": (C.c_int, [vp, i64, i64, C.c_float]),
        "prsgd_run_heterogeneous_epoch": (C.c_int, [vp, vp]),
        "prsgd_stage_data": (C.c_int, [vp, vp, vp, vp, vp, vp]),
        "prsgd_swap_data": (C.c_int, [vp]),
        "prsgd_set_worker_offset": (C.c_int, [vp, i32]),
        "prsgd_set_global_workers": (C.c_int, [vp, i32]),
        "prsgd_check_finite": (C.c_int, [vp, C.POINTER(i64), C.POINTER(i32)]),
        "prsgd_partial_sum": (C.c_int, [vp, vp, i64, i64]),
        "prsgd_assign_rows": (C.c_int, [vp, vp, C.c_float, i64, i64]),
        "prsgd_orthogonalize_workspace_bytes": (C.c_int, [i32, i32, i32, i32, szp]),
        "prsgd_orthogonalize": (C.c_int, [vp, i32, i64, i64, vp, i32, i64, i64, i32, i32, i32, i32, vp, f32, f32, i32, vp, szt, vp]),
        "prsgd_muon_step": (C.c_int, [vp, i32, i64, i64, vp, i64, i64, vp, i32, i64, i64, i32, i32, i32, f32, f32, i32, f32,
                                      i32, vp, f32, f32, i32, vp, szt, vp]),
        "prsgd_work_status": (C.c_int, [vp, vp]),
        "prsgd_muon_workspace_bytes": (C.c_int, [vp, C.c_uint32, szp]),
        "prsgd_enable_muon": (C.c_int, [vp, C.c_uint32, i32, i32, vp, szt]),
        "prsgd_set_balance": (C.c_int, [vp, f32, i32]),
        "prsgd_route_workspace_bytes": (C.c_int, [i64, i64, i32, szp]),
        "prsgd_route": (C.c_int, [vp, i32, i64, i64, vp, i64, i64, i32, i32, i32, f32, vp, vp, vp, vp, vp, vp, szt, vp]),
        "prsgd_route_grad": (C.c_int, [vp, i32, i64, i64, vp, i64, i64, i32, i32, i32, f32, vp, vp, vp, vp, vp, i64, i64, vp]),
        "prsgd_last_error": (C.c_char_p, [vp]),
        "prsgd_average_rows": (C.c_int, [vp, i64, i64, i64, vp]),
        "prsgd_draw_block": (u64, [u64, i32, i64, u64]),
        "prsgd_mean_rows_noalloc": (C.c_int, [vp, i64, i64, i64, vp, C.c_int, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib


lib = _load()


class PRSGDError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"prsgd error {code}: {msg}")
        self.code = code


def _check(rc: int, ctx=None) -> None:
    if rc != PRSGD_OK:
        raise PRSGDError(rc, (lib.prsgd_last_error(ctx) or b"").decode())


def make_spec(dims: Sequence[int], batch: int, precision: int, pool_samples: int, seed: int):
    arr = (C.c_int32 * len(dims))(*dims)
    spec = ModelSpec(len(dims) - 1, C.cast(arr, C.POINTER(C.c_int32)), batch, precision, pool_samples, seed)
    spec._keep = arr
    return spec


def prsgd_layout(dims, batch, precision, pool_samples, seed=0) -> Layout:
    spec, lay = make_spec(dims, batch, precision, pool_samples, seed), Layout()
    _check(lib.prsgd_layout(C.byref(spec), C.byref(lay)))
    return lay


def prsgd_workspace_bytes(N, dims, batch, precision, pool_samples, seed=0):
    spec = make_spec(dims, batch, precision, pool_samples, seed)
    a, b, c = C.c_size_t(), C.c_size_t(), C.c_size_t()
    _check(lib.prsgd_workspace_bytes(N, C.byref(spec), C.byref(a), C.byref(b), C.byref(c)))
    return a.value, b.value, c.value


def prsgd_alg2_schedule(N: int, s: int):
    """(K^s, gamma^s) of Theorem 2."""
    K, g = C.c_int64(), C.c_float()
    _check(lib.prsgd_alg2_schedule(N, s, C.byref(K), C.byref(g)))
    return K.value, g.value


def prsgd_draw_block(seed: int, worker: int, t: int, n_blocks: int) -> int:
    return int(lib.prsgd_draw_block(seed, worker, t, n_blocks))


def prsgd_average_rows(P: torch.Tensor, N: int, m: int, row_stride: Optional[int] = None, stream=None) -> None:
    """In-place node average + broadcast over the rows of a device fp32 tensor."""
    assert P.is_cuda and P.dtype == torch.float32
    s = stream if stream is not None else torch.cuda.current_stream(P.device)
    with torch.cuda.device(P.device):
        _check(lib.prsgd_average_rows(P.data_ptr(), N, m, m if row_stride is None else row_stride, s.cuda_stream))


def prsgd_mean_rows_noalloc(P: torch.Tensor, N: int, m: int, row_stride: int, out, stream=None):
    """Node average of the rows of a device fp32 tensor into `out` (numpy array, or host / device tensor),
    staged through the library's fixed device row: nothing is allocated and P is left untouched."""
    assert P.is_cuda and P.dtype == torch.float32
    s = stream if stream is not None else torch.cuda.current_stream(P.device)
    if isinstance(out, np.ndarray):
        assert out.dtype == np.float32 and out.size >= m and out.flags["C_CONTIGUOUS"]
        ptr, on_dev = out.ctypes.data, 0
    else:
        assert out.dtype == torch.float32 and out.numel() >= m and out.is_contiguous()
        ptr, on_dev = out.data_ptr(), 1 if out.is_cuda else 0
    with torch.cuda.device(P.device):
        _check(lib.prsgd_mean_rows_noalloc(P.data_ptr(), N, m, row_stride, ptr, on_dev, s.cuda_stream))
    return out


# ---- stand-alone training operators -------------------------------------------------------------------------
TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
MUON_COEFS = (3.4445, -4.7750, 2.0315)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


def _run_on(index: int, stream, fn, *args) -> None:
    """Calls fn(*args, stream) with device `index` current, on `stream` or that device's current stream."""
    if index == torch.cuda.current_device():
        rc = fn(*args, _raw_stream(index) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(index):
            rc = fn(*args, _raw_stream(index) if stream is None else stream.cuda_stream)
    if rc != PRSGD_OK:
        _check(rc)


def _empty(shape, dtype, device, stream=None) -> torch.Tensor:
    """A new tensor of the stream the call runs on: its memory is not handed out again before that work is done."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _matrices(t: torch.Tensor, name: str):
    """(pointer, type, row stride, batch stride) of a [batch, rows, cols] or [rows, cols] tensor."""
    ty = TYPES.get(t.dtype)
    if ty is None or not t.is_cuda:
        raise ValueError(f"{name} must be a float32, bfloat16 or float16 tensor on the GPU")
    shape, stride = t.shape, t.stride()
    n = len(shape)
    if n == 3:
        b, r, c = shape
        sb, sr, sc = stride
    elif n == 2:
        (r, c), (sr, sc), b, sb = shape, stride, 1, 0
    else:
        raise ValueError(f"{name} must be [batch, rows, cols] or [rows, cols]")
    if c > 1 and sc != 1:
        raise ValueError(f"the columns of {name} must be contiguous")
    if r <= 1 and sr < c:
        sr = c
    return t.data_ptr(), ty, sr, sb if b > 1 else 0


def _size3(t: torch.Tensor):
    return t.shape if t.dim() == 3 else (1, *t.shape)


def _precision_for(t: torch.Tensor) -> int:
    """Of a step on weights of t's type: 16-bit ones are rounded by more than single 16-bit operands cost the step."""
    return PRECISION_FP32 if t.dtype is torch.float32 else PRECISION_BF16


def _precision_for_result(t: torch.Tensor) -> int:
    """Of a result of t's type: single 16-bit operands cost about 2e-3, half a rounding of bfloat16, but five of float16."""
    return PRECISION_BF16 if t.dtype is torch.bfloat16 else PRECISION_FP32


def _same_place(name: str, t: torch.Tensor, index: int) -> None:
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, the call's other tensors on cuda:{index}")


def _scratch(t: torch.Tensor, index: int):
    """(pointer, bytes) of a workspace on device `index`: one piece of memory, whatever its element type."""
    if t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on cuda:{index}")
    return t.data_ptr(), t.numel() * t.element_size()


def prsgd_orthogonalize_workspace_bytes(batch: int, rows: int, cols: int, precision: int) -> int:
    n = C.c_size_t()
    _check(lib.prsgd_orthogonalize_workspace_bytes(batch, rows, cols, precision, C.byref(n)))
    return n.value


def orthogonalize_workspace(G: torch.Tensor, precision: Optional[int] = None, stream=None) -> torch.Tensor:
    """Workspace of prsgd_orthogonalize for matrices like G: for results of any type (the larger one, of 32-bit precision), or for
    calls of that `precision` alone."""
    p = PRECISION_FP32 if precision is None else precision
    return _empty(prsgd_orthogonalize_workspace_bytes(*_size3(G), p), torch.uint8, G.device, stream)


def muon_workspace(W: torch.Tensor, precision: Optional[int] = None, stream=None) -> torch.Tensor:
    """Workspace of prsgd_muon_step for weights like W."""
    return orthogonalize_workspace(W, _precision_for(W) if precision is None else precision, stream)


def _coefs(coefs):
    """The three coefficients as the C entry takes them (None: the default ones)."""
    if coefs is None or tuple(coefs) == MUON_COEFS:
        return None
    if len(coefs) != 3:
        raise ValueError("coefs must be the three of a X + (b A + c A^2) X")
    return (C.c_float * 3)(*coefs)


def prsgd_orthogonalize(G: torch.Tensor, out: Optional[torch.Tensor] = None, *, steps: int = 5, coefs=None,
                        scale: float = 1.0, eps: float = 1e-7, precision: Optional[int] = None,
                        workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Newton-Schulz orthogonalisation of every matrix of G ([batch, rows, cols] or [rows, cols]); see prsgd.h."""
    if out is None:
        out = _empty(G.shape, G.dtype, G.device, stream)
    elif out.shape != G.shape:
        raise ValueError("out must have G's shape")
    p = _precision_for_result(out) if precision is None else precision
    if workspace is None:
        workspace = orthogonalize_workspace(G, p, stream)
    index = G.get_device()
    _same_place("out", out, index)
    work, size = _scratch(workspace, index)
    _run_on(index, stream, lib.prsgd_orthogonalize, *_matrices(G, "G"), *_matrices(out, "out"), *_size3(G), steps,
            _coefs(coefs), scale, eps, p, work, size)
    return out


def prsgd_muon_step(W: torch.Tensor, V: torch.Tensor, G: torch.Tensor, lr: float, *, mu: float = 0.95,
                    nesterov: bool = True, weight_decay: float = 0.0, steps: int = 5, coefs=None, scale: float = 1.0,
                    eps: float = 1e-7, precision: Optional[int] = None, workspace: Optional[torch.Tensor] = None,
                    stream=None) -> None:
    """Muon step of every matrix of W in place, with its fp32 momentum buffers V; see prsgd.h."""
    if W.shape != V.shape or W.shape != G.shape:
        raise ValueError("W, V and G must have the same shape")
    if V.dtype != torch.float32:
        raise ValueError("V must be float32")
    p = _precision_for(W) if precision is None else precision
    if workspace is None:
        workspace = muon_workspace(W, p, stream)
    index = W.get_device()
    _same_place("V", V, index)
    _same_place("G", G, index)
    work, size = _scratch(workspace, index)
    v, _, vr, vb = _matrices(V, "V")
    _run_on(index, stream, lib.prsgd_muon_step, *_matrices(W, "W"), v, vr, vb, *_matrices(G, "G"), *_size3(W), lr, mu,
            1 if nesterov else 0, weight_decay, steps, _coefs(coefs), scale, eps, p, work, size)


def prsgd_work_status(workspace: torch.Tensor, stream=None) -> None:
    """Raises if a kernel of the last call that used this workspace recorded an error; synchronises the stream."""
    _run_on(workspace.get_device(), stream, lib.prsgd_work_status, workspace.data_ptr())


def prsgd_route_workspace_bytes(groups: int, tokens: int, experts: int) -> int:
    n = C.c_size_t()
    _check(lib.prsgd_route_workspace_bytes(groups, tokens, experts, C.byref(n)))
    return n.value


def route_workspace(logits: torch.Tensor, stream=None) -> torch.Tensor:
    return _empty(prsgd_route_workspace_bytes(*_size3(logits)), torch.uint8, logits.device, stream)


def route_outputs(logits: torch.Tensor, k: int, stream=None):
    """Tensors for prsgd_route's results: experts, weights [G, T, k], counts, mean [G, E], loss [G]."""
    (G, T, E), d = _size3(logits), logits.device
    i, f = torch.int32, torch.float32
    return tuple(_empty(shape, ty, d, stream) for shape, ty in (((G, T, k), i), ((G, T, k), f), ((G, E), i), ((G, E), f), ((G,), f)))


def _dense(t: Optional[torch.Tensor], name: str, dtype, numel: int, index: int):
    """Pointer of a contiguous tensor of `numel` elements on device `index` (None stays None)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != numel or not t.is_contiguous() or t.get_device() != index:
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {numel} elements on cuda:{index}")
    return t.data_ptr()


def _mask(live: Optional[torch.Tensor], numel: int, index: int):
    """Pointer of the live tokens' mask: bytes or truth values, 0 = padding."""
    return _dense(live, "live", torch.bool if live is not None and live.dtype is torch.bool else torch.uint8, numel, index)


def prsgd_route(logits: torch.Tensor, k: int, coef: float, *, normalize: bool = False, live: Optional[torch.Tensor] = None,
                out=None, workspace: Optional[torch.Tensor] = None, stream=None):
    """Top-k router with its balance loss over logits [G, T, E] (or [T, E]); returns (experts, weights, counts, mean,
    loss), see prsgd.h.  `live`: uint8 or bool [G, T], 0 = padding; `out`: a tuple as route_outputs makes it."""
    ptr, ty, row, group = _matrices(logits, "logits")
    G, T, E = _size3(logits)
    if out is None:
        out = route_outputs(logits, k, stream)
    if workspace is None:
        workspace = route_workspace(logits, stream)
    at = logits.get_device()
    work, size = _scratch(workspace, at)
    experts, weights, counts, mean, loss = out
    i32, f32, n, m = torch.int32, torch.float32, G * T * k, G * E
    _run_on(at, stream, lib.prsgd_route, ptr, ty, row, group, _mask(live, G * T, at),
            G, T, E, k, 1 if normalize else 0, coef, _dense(experts, "experts", i32, n, at), _dense(weights, "weights", f32, n, at),
            _dense(counts, "counts", i32, m, at), _dense(mean, "mean", f32, m, at), _dense(loss, "loss", f32, G, at),
            work, size)
    return out


def prsgd_route_grad(logits: torch.Tensor, experts: torch.Tensor, counts: torch.Tensor, coef: float, *,
                     normalize: bool = False, live: Optional[torch.Tensor] = None, dweights: Optional[torch.Tensor] = None,
                     dloss: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Gradient of the router's weights and balance loss with respect to the logits; see prsgd.h."""
    ptr, ty, row, group = _matrices(logits, "logits")
    G, T, E = _size3(logits)
    k = experts.shape[-1]
    if out is None:
        out = _empty(logits.shape, logits.dtype, logits.device, stream)
    elif out.shape != logits.shape or out.dtype != logits.dtype:
        raise ValueError("out must have the logits' shape and type")
    at = logits.get_device()
    _same_place("out", out, at)
    optr, _, orow, ogroup = _matrices(out, "out")
    i32, f32, n = torch.int32, torch.float32, G * T * k
    _run_on(at, stream, lib.prsgd_route_grad, ptr, ty, row, group, _mask(live, G * T, at),
            G, T, E, k, 1 if normalize else 0, coef, _dense(experts, "experts", i32, n, at), _dense(counts, "counts", i32, G * E, at),
            _dense(dweights, "dweights", f32, n, at), _dense(dloss, "dloss", f32, G, at), optr, orow, ogroup)
    return out


def _host_ptr(a: np.ndarray) -> int:
    assert a.flags["C_CONTIGUOUS"]
    return a.ctypes.data


class PRSGD:
    """One PR-SGD context plus the device tensors that back it."""

    def __init__(self, N: int, dims: Sequence[int], batch: int, gamma: float, I: int, precision: int,
                 pool_samples: int, seed: int, device: str = "cuda:0", stream: Optional[torch.cuda.Stream] = None):
        self.N, self.dims, self.B, self.precision, self.P = N, tuple(dims), batch, precision, pool_samples
        self.device = torch.device(device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self._spec = make_spec(dims, batch, precision, pool_samples, seed)
        self.layout = Layout()
        _check(lib.prsgd_layout(C.byref(self._spec), C.byref(self.layout)))
        self.m, self.m_pad = self.layout.m, self.layout.m_pad
        pb, sb, wb = prsgd_workspace_bytes(N, dims, batch, precision, pool_samples, seed)
        with torch.cuda.device(self.device):
            self.params = torch.empty(pb // 4, dtype=torch.float32, device=self.device)
            self.shadow = torch.empty(max(sb // 2, 1), dtype=torch.bfloat16, device=self.device) if sb else None
            self.scratch = torch.empty(wb, dtype=torch.uint8, device=self.device)
            ctx = C.c_void_p()
            _check(lib.prsgd_create(N, C.byref(self._spec), gamma, I, self.params.data_ptr(),
                                    self.shadow.data_ptr() if self.shadow is not None else None,
                                    self.scratch.data_ptr(), self.stream.cuda_stream, C.byref(ctx)))
        self.ctx = ctx
        self._X = self._Y = None
        self.average_velocity = False

    def _call(self, fn, *args):
        with torch.cuda.device(self.device):
            _check(fn(self.ctx, *args), self.ctx)

    def close(self):
        if getattr(self, "ctx", None):
            lib.prsgd_destroy(self.ctx)
            self.ctx = None

    __del__ = close

    # ---- data -------------------------------------------------------------------
    def bind_data(self, X: torch.Tensor, Y: torch.Tensor):
        want = torch.bfloat16 if self.precision == PRECISION_BF16 else torch.float32
        assert X.is_cuda and Y.is_cuda and X.dtype == want and Y.dtype == torch.int32
        assert X.is_contiguous() and Y.is_contiguous()
        assert tuple(X.shape) == (self.N, self.P, self.dims[0]) and tuple(Y.shape) == (self.N, self.P)
        self._X, self._Y = X, Y
        self._call(lib.prsgd_bind_data, X.data_ptr(), X_BF16 if want == torch.bfloat16 else X_FP32, Y.data_ptr())

    def upload_data(self, hX: torch.Tensor, hY: torch.Tensor):
        assert not hX.is_cuda and not hY.is_cuda and hX.is_contiguous() and hY.is_contiguous()
        self._call(lib.prsgd_upload_data, hX.data_ptr(), hY.data_ptr())

    def stage_data(self, hX: torch.Tensor, hY: torch.Tensor, copy_stream: torch.cuda.Stream):
        """Copy the next pools from (pinned) host tensors into the spare device pools on `copy_stream`."""
        assert not hX.is_cuda and not hY.is_cuda and hX.is_contiguous() and hY.is_contiguous()
        if getattr(self, "_spare", None) is None:
            self._spare = (torch.empty_like(self._X), torch.empty_like(self._Y))
        self._call(lib.prsgd_stage_data, hX.data_ptr(), hY.data_ptr(), self._spare[0].data_ptr(),
                   self._spare[1].data_ptr(), copy_stream.cuda_stream)

    def swap_data(self):
        """Make the staged pools current; the previous pools become the spare ones."""
        self._call(lib.prsgd_swap_data)
        (self._X, self._Y), self._spare = self._spare, (self._X, self._Y)

    # ---- parameters -------------------------------------------------------------
    def set_params(self, x, worker: int = -1):
        if isinstance(x, torch.Tensor) and x.is_cuda:
            assert x.dtype == torch.float32 and x.numel() == self.m and x.is_contiguous()
            self._call(lib.prsgd_set_params, x.data_ptr(), worker, 1)
        else:
            a = np.ascontiguousarray(np.asarray(x, dtype=np.float32))
            assert a.size == self.m
            self._call(lib.prsgd_set_params, _host_ptr(a), worker, 0)

    def set_params_stacked(self, x):
        if isinstance(x, torch.Tensor) and x.is_cuda:
            assert x.dtype == torch.float32 and x.numel() == self.N * self.m and x.is_contiguous()
            self._call(lib.prsgd_set_params_stacked, x.data_ptr(), 1)
        else:
            a = np.ascontiguousarray(np.asarray(x, dtype=np.float32))
            assert a.size == self.N * self.m
            self._call(lib.prsgd_set_params_stacked, _host_ptr(a), 0)

    def get_params_stacked(self) -> np.ndarray:
        out = np.empty((self.N, self.m), dtype=np.float32)
        self._call(lib.prsgd_get_params_stacked, _host_ptr(out), 0)
        return out

    def get_params(self, worker: int) -> np.ndarray:
        out = np.empty(self.m, dtype=np.float32)
        self._call(lib.prsgd_get_params, _host_ptr(out), worker, 0)
        return out

    # ---- Algorithm 1 ------------------------------------------------------------
    def local_steps(self, k: int):
        self._call(lib.prsgd_local_steps, k)

    def local_steps_sum(self, k: int):
        """k iterations, the last one leaving the SUM of the updated local rows in every row (see prsgd.h)."""
        self._call(lib.prsgd_local_steps_sum, k)

    def row0(self) -> torch.Tensor:
        """Row 0 of the store as a tensor of m_pad floats (the all-reduce buffer after local_steps_sum)."""
        return self.params[:self.m_pad]

    def average(self):
        self._call(lib.prsgd_average)

    def get_average(self, out=None):
        """Node average; into a host numpy array (default), a pinned host tensor or a device tensor."""
        if out is None:
            out = np.empty(self.m, dtype=np.float32)
        if isinstance(out, np.ndarray):
            self._call(lib.prsgd_get_average, _host_ptr(out), 0)
        else:
            assert out.dtype == torch.float32 and out.numel() == self.m and out.is_contiguous()
            self._call(lib.prsgd_get_average, out.data_ptr(), 1 if out.is_cuda else 0)
        return out

    def get_average_async(self, out, copy_stream):
        """Node average into a pinned host tensor through `copy_stream`; valid once that stream is synchronised."""
        assert out.dtype == torch.float32 and out.numel() == self.m and out.is_contiguous() and out.is_pinned()
        self._call(lib.prsgd_get_average_async, out.data_ptr(), copy_stream.cuda_stream)
        return out

    def get_losses(self) -> np.ndarray:
        out = np.empty(self.N, dtype=np.float32)
        self._call(lib.prsgd_get_losses, _host_ptr(out))
        return out

    def get_draws(self) -> np.ndarray:
        out = np.empty(self.N, dtype=np.int32)
        self._call(lib.prsgd_get_draws, _host_ptr(out))
        return out

    # ---- shard of a multi-GPU job ------------------------------------------------
    def set_worker_offset(self, first_worker: int):
        self._call(lib.prsgd_set_worker_offset, first_worker)

    def set_global_workers(self, N_global: int):
        self._call(lib.prsgd_set_global_workers, N_global)

    def new_row(self) -> torch.Tensor:
        """A device row of m_pad floats (the buffer an all-reduce works on)."""
        return torch.zeros(self.m_pad, dtype=torch.float32, device=self.device)

    def partial_sum(self, row: torch.Tensor, col0: int = 0, ncols: Optional[int] = None):
        assert row.is_cuda and row.dtype == torch.float32 and row.numel() == self.m_pad
        self._call(lib.prsgd_partial_sum, row.data_ptr(), col0, self.m_pad - col0 if ncols is None else ncols)

    def assign_rows(self, row: torch.Tensor, divisor: float, col0: int = 0, ncols: Optional[int] = None):
        assert row.is_cuda and row.dtype == torch.float32 and row.numel() == self.m_pad
        self._call(lib.prsgd_assign_rows, row.data_ptr(), float(divisor), col0, self.m_pad - col0 if ncols is None else ncols)

    def enable_momentum(self, mu: float, average_velocity: bool = False):
        """Allocate the momentum buffers (same size as the store) and switch the local step to SGD with momentum."""
        with torch.cuda.device(self.device):
            self.velocity = torch.empty(self.N * self.m_pad, dtype=torch.float32, device=self.device)
        self._call(lib.prsgd_enable_momentum, mu, self.velocity.data_ptr(), 1 if average_velocity else 0)
        self.average_velocity = bool(average_velocity)

    def enable_muon(self, layers: Optional[Sequence[int]] = None, scale: int = MUON_SCALE_SPECTRAL, steps: int = 5):
        """Muon step for the weights of `layers` (1-based; default: all but the class layer; [] switches it off), after
        enable_momentum; allocates the workspace."""
        chosen = range(1, len(self.dims) - 1) if layers is None else layers
        bits = 0
        for l in chosen:
            if not 1 <= l < len(self.dims):
                raise ValueError(f"the model has no layer {l}")
            bits |= 1 << (l - 1)
        n = C.c_size_t()
        self._call(lib.prsgd_muon_workspace_bytes, bits, C.byref(n))
        with torch.cuda.device(self.device):
            work = _empty(max(n.value, 1), torch.uint8, self.device, self.stream)
        self._call(lib.prsgd_enable_muon, bits, scale, steps, work.data_ptr(), n.value)
        self._muon_work = work

    def set_balance(self, coef: float, top_k: int):
        """Adds the balance loss over the classes to F_i (top_k = 0: off)."""
        self._call(lib.prsgd_set_balance, coef, top_k)

    def get_velocity_stacked(self) -> np.ndarray:
        out = np.empty((self.N, self.m), dtype=np.float32)
        self._call(lib.prsgd_get_velocity_stacked, _host_ptr(out), 0)
        return out

    # ---- Algorithms 2 and 3 ------------------------------------------------------
    def run_time_varying(self, s_begin: int, s_end: int, gamma_scale: float = 1.0):
        self._call(lib.prsgd_run_time_varying, s_begin, s_end, gamma_scale)

    def run_heterogeneous_epoch(self, I_i: Sequence[int]):
        a = np.ascontiguousarray(np.asarray(I_i, dtype=np.int32))
        assert a.size == self.N
        self._call(lib.prsgd_run_heterogeneous_epoch, _host_ptr(a))

    # ---- schedule ---------------------------------------------------------------
    def set_lr(self, gamma: float):
        self._call(lib.prsgd_set_lr, gamma)

    def set_interval(self, I: int):
        self._call(lib.prsgd_set_interval, I)

    def set_active(self, mask):
        if mask is None:
            self._call(lib.prsgd_set_active, None)
        else:
            a = np.ascontiguousarray(np.asarray(mask, dtype=np.uint8))
            assert a.size == self.N
            self._call(lib.prsgd_set_active, _host_ptr(a))

    def get_step(self) -> int:
        t = C.c_int64()
        self._call(lib.prsgd_get_step, C.byref(t))
        return t.value

    def set_step(self, t: int):
        self._call(lib.prsgd_set_step, t)

    def set_option(self, option: int, value: int):
        self._call(lib.prsgd_set_option, option, value)

    def get_launch_count(self) -> int:
        n = C.c_int64()
        self._call(lib.prsgd_get_launch_count, C.byref(n))
        return n.value

    def get_profile(self) -> dict:
        """{family: (ms_total, launches)} since the last call; needs OPT_PROFILE."""
        out = {}
        for k, name in enumerate(KERNEL_FAMILIES):
            ms, n = C.c_double(), C.c_int64()
            self._call(lib.prsgd_get_profile, k, C.byref(ms), C.byref(n))
            out[name] = (ms.value, n.value)
        return out

    def selftest_wait_expiry(self, limit_us: int = 1000):
        self._call(lib.prsgd_selftest_wait_expiry, limit_us)

    def clear_device_error(self):
        self._call(lib.prsgd_clear_device_error)

    def sync(self):
        self._call(lib.prsgd_sync)

    def check_finite(self):
        """(return code, count of non-finite words, lowest worker that holds one or -1); does not raise."""
        n, first = C.c_int64(), C.c_int32()
        with torch.cuda.device(self.device):
            rc = lib.prsgd_check_finite(self.ctx, C.byref(n), C.byref(first))
        return rc, n.value, first.value
