"""Python binding of the gfx950 ParaDiGMS library (libparadigms.so).

Argument marshalling only: every step of the sampling path runs in the HIP
library through its C ABI (include/paradigms.h), whose entry points carry
the same names.  PyTorch supplies device memory and streams; it is imported
before the library is loaded so that the process uses one HIP runtime.

If the library has not been built, ``load()`` raises: there is no fallback.
"""
from __future__ import annotations

import ctypes
import dataclasses
import os
import struct
from typing import Dict, List, Optional, Sequence

import numpy as np
import torch  # noqa: F401  (loads the HIP runtime first)

__all__ = [
    "PdError", "load", "lib_path", "Schedule", "Denoiser", "Workspace", "SampleStats",
    "pd_init_schedule", "pd_denoiser_create", "pd_denoiser_forward",
    "pd_denoiser_forward_static", "pd_normals",
    "pd_workspace_create", "pd_sample_sequential", "pd_sample_picard",
    "PD_DDPM", "PD_DDIM", "PD_DDIM_HEUN", "PD_DDIM_DPM2M", "PD_STOP_RELAXED", "PD_STOP_PROP2",
    "PD_MODEL_GMM2D", "PD_MODEL_MLP", "PD_MODEL_CONV1X1",
    "PD_F32", "PD_BF16", "EXPORTED_SYMBOLS",
    "pd_rmsnorm_forward", "pd_rmsnorm_backward", "pd_rotary_table", "pd_rotary_apply",
    "pd_attention_forward", "pd_attention_backward",
    "PD_F8E4M3", "PD_ROTARY_HALF", "PD_ROTARY_INTERLEAVED",
    "PD_ROTARY_PLAIN", "PD_ROTARY_LINEAR", "PD_ROTARY_BASE", "PD_ROTARY_BY_PARTS",
]

PD_OK, PD_ERR_INVALID_ARG, PD_ERR_OOM, PD_ERR_DEVICE, PD_ERR_NUMERIC, PD_ERR_UNSUPPORTED = range(6)
STATUS_NAMES = {0: "PD_OK", 1: "PD_ERR_INVALID_ARG", 2: "PD_ERR_OOM", 3: "PD_ERR_DEVICE",
                4: "PD_ERR_NUMERIC", 5: "PD_ERR_UNSUPPORTED"}
PD_DDPM, PD_DDIM, PD_DDIM_HEUN, PD_DDIM_DPM2M = 0, 1, 2, 3
PD_STOP_RELAXED, PD_STOP_PROP2 = 0, 1
STOP_RULES = {"relaxed": PD_STOP_RELAXED, "prop2": PD_STOP_PROP2}
PD_MODEL_GMM2D, PD_MODEL_MLP, PD_MODEL_CONV1X1 = 0, 1, 2
PD_F32, PD_BF16, PD_F8E4M3 = 0, 1, 2
PD_ROTARY_HALF, PD_ROTARY_INTERLEAVED = 0, 1
PD_ROTARY_PLAIN, PD_ROTARY_LINEAR, PD_ROTARY_BASE, PD_ROTARY_BY_PARTS = 0, 1, 2, 3

EXPORTED_SYMBOLS = [
    "pd_last_error", "pd_version", "pd_init_schedule", "pd_destroy_schedule",
    "pd_schedule_tables", "pd_schedule_multistep_tables", "pd_denoiser_create", "pd_denoiser_destroy",
    "pd_denoiser_forward", "pd_denoiser_forward_static",
    "pd_normals", "pd_workspace_create", "pd_workspace_destroy", "pd_sample_sequential",
    "pd_sample_picard",
    "pd_rmsnorm_forward", "pd_rmsnorm_backward_scratch", "pd_rmsnorm_backward",
    "pd_rotary_table", "pd_rotary_apply",
    "pd_attention_forward_scratch", "pd_attention_forward",
    "pd_attention_backward_scratch", "pd_attention_backward",
]


class PdError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(code, code)}: {msg}")
        self.code = code


class _ScheduleDesc(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("T_train", ctypes.c_int32), ("T", ctypes.c_int32),
                ("tol_index_offset", ctypes.c_int32), ("stop_rule", ctypes.c_int32),
                ("beta_start", ctypes.c_double),
                ("beta_end", ctypes.c_double), ("eta", ctypes.c_double)]


class _ModelDesc(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("dtype", ctypes.c_int32), ("width", ctypes.c_int32),
                ("cond_dim", ctypes.c_int32), ("n_components", ctypes.c_int32),
                ("guidance", ctypes.c_float)]


class _Stats(ctypes.Structure):
    _fields_ = [("iters", ctypes.c_int32), ("trace_cap", ctypes.c_int32),
                ("evals_per_sample", ctypes.c_int64), ("network_rows", ctypes.c_int64),
                ("stride_trace", ctypes.POINTER(ctypes.c_int32)),
                ("time_kernels", ctypes.c_int32), ("denoiser_launches", ctypes.c_int32),
                ("update_launches", ctypes.c_int32), ("finalize_launches", ctypes.c_int32),
                ("denoiser_ms", ctypes.c_double), ("update_ms", ctypes.c_double),
                ("finalize_ms", ctypes.c_double)]


_I64x3 = ctypes.c_int64 * 3


class _RmsnormDesc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("width", ctypes.c_int64), ("x_stride", ctypes.c_int64),
                ("residual_stride", ctypes.c_int64), ("sum_stride", ctypes.c_int64),
                ("y_stride", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("out_dtype", ctypes.c_int32), ("group", ctypes.c_int32), ("eps", ctypes.c_float)]


class _RotaryTableDesc(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("scaling", ctypes.c_int32),
                ("base", ctypes.c_double), ("factor", ctypes.c_double),
                ("original_length", ctypes.c_double), ("turns_low", ctypes.c_double),
                ("turns_high", ctypes.c_double), ("magnitude", ctypes.c_double)]


class _RotaryDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("length", ctypes.c_int64), ("heads_q", ctypes.c_int32),
                ("heads_k", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("rotary_dim", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("backward", ctypes.c_int32),
                ("table_rows", ctypes.c_int64), ("position_stride", ctypes.c_int64),
                ("q_stride", _I64x3), ("k_stride", _I64x3), ("q_out_stride", _I64x3),
                ("k_out_stride", _I64x3)]


class _AttentionDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads_q", ctypes.c_int32), ("heads_kv", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("q_len", ctypes.c_int32), ("kv_len", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32), ("window", ctypes.c_int32),
                ("sinks", ctypes.c_int32), ("scale", ctypes.c_float), ("q_stride", _I64x3),
                ("k_stride", _I64x3), ("v_stride", _I64x3), ("out_stride", _I64x3),
                ("dq_stride", _I64x3), ("dk_stride", _I64x3), ("dv_stride", _I64x3),
                ("dout_stride", _I64x3)]


# the same three as bytes: the calls pack them (a Structure with its arrays takes 2 us more)
_RMSNORM_BYTES = struct.Struct("6q3if")
_ROTARY_BYTES = struct.Struct("2q7i14q")
_ATTENTION_BYTES = struct.Struct("10if24q")

_LIB: Optional[ctypes.CDLL] = None


def lib_path() -> str:
    return os.path.join(os.path.dirname(os.path.abspath(__file__)), "libparadigms.so")


def load() -> ctypes.CDLL:
    """Load libparadigms.so (raises if it has not been built)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with "
                           "`python -m paper_2305_16317_amd.build` (no fallback exists)")
    L = ctypes.CDLL(path)
    vp, i32, i64, u64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_float
    P = ctypes.POINTER
    sig = {
        "pd_last_error": ([], ctypes.c_char_p),
        "pd_version": ([], ctypes.c_char_p),
        "pd_init_schedule": ([P(_ScheduleDesc), P(vp)], i32),
        "pd_destroy_schedule": ([vp], None),
        "pd_schedule_tables": ([vp, P(i32), P(f32), P(f32), P(f32), P(f32), P(i32)], i32),
        "pd_schedule_multistep_tables": ([vp, P(f32), P(f32)], i32),
        "pd_denoiser_create": ([P(_ModelDesc), P(i64), i32, P(P(f32)), i32, vp, P(vp)], i32),
        "pd_denoiser_destroy": ([vp], None),
        "pd_denoiser_forward": ([vp, vp, vp, i64, vp, vp], i32),
        "pd_denoiser_forward_static": ([vp, vp, vp, i64, vp, vp], i32),
        "pd_normals": ([u64, ctypes.c_uint32, i64, vp, vp], i32),
        "pd_workspace_create": ([vp, vp, i32, i32, P(vp)], i32),
        "pd_workspace_destroy": ([vp], None),
        "pd_sample_sequential": ([vp, vp, u64, i32, P(i64), i32, vp, P(_Stats), vp, vp], i32),
        "pd_sample_picard": ([vp, vp, i32, f32, u64, i32, P(i64), i32, vp, P(_Stats), vp, vp], i32),
        "pd_rmsnorm_forward": ([vp] + [vp] * 8, i32),
        "pd_rmsnorm_backward_scratch": ([vp, P(i64)], i32),
        "pd_rmsnorm_backward": ([vp] + [vp] * 8 + [i64, vp], i32),
        "pd_rotary_table": ([P(_RotaryTableDesc), i64, i64, vp, vp], i32),
        "pd_rotary_apply": ([vp] + [vp] * 7, i32),
        "pd_attention_forward_scratch": ([vp, P(i64)], i32),
        "pd_attention_forward": ([vp] + [vp] * 8 + [i64, vp], i32),
        "pd_attention_backward_scratch": ([vp, P(i64)], i32),
        "pd_attention_backward": ([vp] + [vp] * 12 + [i64, vp], i32),
    }
    for name, (args, res) in sig.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = res
    _LIB = L
    return L


def _check(code: int) -> None:
    if code != PD_OK:
        raise PdError(code, load().pd_last_error().decode())


# the current stream's handle without a Stream object around it (2.6 us a call less), where torch has it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _shape(shape: Sequence[int]):
    arr = (ctypes.c_int64 * len(shape))(*[int(v) for v in shape])
    return arr, len(shape)


# --------------------------------------------------------------------- handles
class Schedule:
    def __init__(self, handle: ctypes.c_void_p, T: int, T_train: int):
        self._h = handle
        self.T = T
        self.T_train = T_train

    @property
    def handle(self):
        return self._h

    def tables(self) -> Dict[str, np.ndarray]:
        T = self.T
        A, B, zs, tv = (np.empty(T, np.float32) for _ in range(4))
        nt = np.empty(T, np.int32)
        Tout = ctypes.c_int32(0)
        fp = lambda a: a.ctypes.data_as(ctypes.POINTER(ctypes.c_float))
        _check(load().pd_schedule_tables(self._h, ctypes.byref(Tout), fp(A), fp(B), fp(zs), fp(tv),
                                          nt.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))))
        R, S = np.empty(T, np.float32), np.empty(T, np.float32)
        _check(load().pd_schedule_multistep_tables(self._h, fp(R), fp(S)))
        return {"A": A, "B": B, "noise_std": zs, "tol_var": tv, "model_t": nt, "R": R, "S": S}

    def __del__(self):
        if getattr(self, "_h", None) and _LIB is not None:
            _LIB.pd_destroy_schedule(self._h)
            self._h = None


class Denoiser:
    def __init__(self, handle, sample_shape, guided: bool):
        self._h = handle
        self.sample_shape = tuple(sample_shape)
        self.D = int(np.prod(sample_shape))
        self.guided = guided

    @property
    def handle(self):
        return self._h

    def __del__(self):
        if getattr(self, "_h", None) and _LIB is not None:
            _LIB.pd_denoiser_destroy(self._h)
            self._h = None


class Workspace:
    def __init__(self, handle):
        self._h = handle

    @property
    def handle(self):
        return self._h

    def __del__(self):
        if getattr(self, "_h", None) and _LIB is not None:
            _LIB.pd_workspace_destroy(self._h)
            self._h = None


@dataclasses.dataclass
class SampleStats:
    iters: int
    evals_per_sample: int
    network_rows: int
    trace: List[int]
    kernel_times: Optional[Dict[str, float]] = dataclasses.field(default=None, compare=False)


# ------------------------------------------------------------------ entry points
def pd_init_schedule(kind: int, T_train: int, T: int, beta_start: float = 1e-4,
                     beta_end: float = 0.02, eta: float = 0.0,
                     tol_index_offset: int = 0, stop_rule: int = PD_STOP_RELAXED) -> Schedule:
    d = _ScheduleDesc(kind, T_train, T, tol_index_offset, stop_rule, beta_start, beta_end, eta)
    h = ctypes.c_void_p()
    _check(load().pd_init_schedule(ctypes.byref(d), ctypes.byref(h)))
    return Schedule(h, T, T_train)


WEIGHT_ORDER = {
    PD_MODEL_GMM2D: ["means", "sigma0"],
    PD_MODEL_MLP: ["W1", "b1", "W2", "b2", "W3", "b3", "W4", "b4"],
    PD_MODEL_CONV1X1: ["W1", "b1", "W2", "b2", "W3", "b3", "W4", "b4"],
}


def pd_denoiser_create(kind: int, sample_shape: Sequence[int], weights: Dict[str, np.ndarray],
                       train: Schedule, width: int = 0, dtype: int = PD_F32,
                       cond_dim: int = 0, guidance: float = 1.0,
                       n_components: int = 0) -> Denoiser:
    names = list(WEIGHT_ORDER[kind]) + (["Wc", "c"] if cond_dim else [])
    arrs = [np.ascontiguousarray(weights[k], dtype=np.float32) for k in names]
    ptrs = (ctypes.POINTER(ctypes.c_float) * len(arrs))(
        *[a.ctypes.data_as(ctypes.POINTER(ctypes.c_float)) for a in arrs])
    if kind == PD_MODEL_GMM2D and not n_components:
        n_components = arrs[0].size // 2
    d = _ModelDesc(kind, dtype, width, cond_dim, n_components, guidance)
    shp, nd = _shape(sample_shape)
    h = ctypes.c_void_p()
    _check(load().pd_denoiser_create(ctypes.byref(d), shp, nd, ptrs, len(arrs), train.handle,
                                     ctypes.byref(h)))
    return Denoiser(h, sample_shape, cond_dim > 0)


def pd_denoiser_forward(den: Denoiser, x: torch.Tensor, model_t: torch.Tensor,
                        eps: torch.Tensor, stream=None) -> None:
    M = x.shape[0] if x.dim() else 0
    for t, dt in ((x, torch.float32), (eps, torch.float32), (model_t, torch.int32)):
        if t.dtype != dt or not t.is_contiguous() or not t.is_cuda:
            raise ValueError("x/eps must be contiguous float32 and model_t int32, on the GPU")
    _check(load().pd_denoiser_forward(den.handle, _ptr(x), _ptr(model_t), M, _ptr(eps),
                                      _stream(stream)))


def pd_denoiser_forward_static(den: Denoiser, x: torch.Tensor, model_t: torch.Tensor,
                               eps: torch.Tensor, stream=None) -> None:
    """pd_denoiser_forward without any allocation or synchronisation (the
    MLP's scratch is a static per-GPU array: M * 2 * width <= 2^20)."""
    M = x.shape[0] if x.dim() else 0
    for t, dt in ((x, torch.float32), (eps, torch.float32), (model_t, torch.int32)):
        if t.dtype != dt or not t.is_contiguous() or not t.is_cuda:
            raise ValueError("x/eps must be contiguous float32 and model_t int32, on the GPU")
    _check(load().pd_denoiser_forward_static(den.handle, _ptr(x), _ptr(model_t), M, _ptr(eps),
                                             _stream(stream)))


def pd_normals(seed: int, rng_stream: int, out: torch.Tensor, stream=None) -> None:
    if out.dtype != torch.float32 or not out.is_contiguous() or not out.is_cuda:
        raise ValueError("out must be a contiguous float32 GPU tensor")
    _check(load().pd_normals(seed, rng_stream, out.numel(), _ptr(out), _stream(stream)))


def pd_workspace_create(sched: Schedule, den: Denoiser, p: int, batch: int) -> Workspace:
    h = ctypes.c_void_p()
    _check(load().pd_workspace_create(sched.handle, den.handle, p, batch, ctypes.byref(h)))
    return Workspace(h)


def _stats(trace_cap: int, time_kernels: bool = False):
    buf = (ctypes.c_int32 * max(trace_cap, 1))()
    st = _Stats(0, trace_cap, 0, 0, ctypes.cast(buf, ctypes.POINTER(ctypes.c_int32)),
                int(time_kernels))
    return st, buf


def _out_stats(st, buf) -> SampleStats:
    n = min(st.iters, st.trace_cap)
    kt = None
    if st.time_kernels:
        kt = {"denoiser_ms": st.denoiser_ms, "denoiser_launches": st.denoiser_launches,
              "update_ms": st.update_ms, "update_launches": st.update_launches,
              "finalize_ms": st.finalize_ms, "finalize_launches": st.finalize_launches}
    return SampleStats(st.iters, st.evals_per_sample, st.network_rows, list(buf[:n]), kt)


def _check_out(x_out: torch.Tensor, batch: int, den: Denoiser):
    if (x_out.dtype != torch.float32 or not x_out.is_contiguous() or not x_out.is_cuda
            or x_out.numel() != batch * den.D):
        raise ValueError("x_out must be a contiguous float32 GPU tensor of batch * D elements")


def pd_sample_sequential(sched: Schedule, den: Denoiser, noise_seed: int, batch: int,
                         sample_shape: Sequence[int], x_out: torch.Tensor,
                         workspace: Optional[Workspace] = None, stream=None,
                         trace_cap: int = 0, time_kernels: bool = False) -> SampleStats:
    _check_out(x_out, batch, den)
    shp, nd = _shape(sample_shape)
    st, buf = _stats(trace_cap, time_kernels)
    _check(load().pd_sample_sequential(sched.handle, den.handle, noise_seed, batch, shp, nd,
                                       _ptr(x_out), ctypes.byref(st),
                                       workspace.handle if workspace else None, _stream(stream)))
    return _out_stats(st, buf)


def pd_sample_picard(sched: Schedule, den: Denoiser, p: int, tau: float, noise_seed: int,
                     batch: int, sample_shape: Sequence[int], x_out: torch.Tensor,
                     workspace: Optional[Workspace] = None, stream=None,
                     trace_cap: Optional[int] = None, time_kernels: bool = False) -> SampleStats:
    _check_out(x_out, batch, den)
    shp, nd = _shape(sample_shape)
    st, buf = _stats(sched.T if trace_cap is None else trace_cap, time_kernels)
    _check(load().pd_sample_picard(sched.handle, den.handle, p, float(tau), noise_seed, batch,
                                   shp, nd, _ptr(x_out), ctypes.byref(st),
                                   workspace.handle if workspace else None, _stream(stream)))
    return _out_stats(st, buf)


# ------------------------------------------------------------ transformer operators
_DTYPES = {torch.float32: PD_F32, torch.bfloat16: PD_BF16}


def _pack(layout: struct.Struct, *values) -> bytes:
    try:
        return layout.pack(*values)
    except (struct.error, OverflowError) as e:
        raise ValueError(f"an argument does not fit its type: {e}") from None


def _dtype(t: torch.Tensor) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise ValueError(f"float32 or bfloat16 is needed, got {t.dtype}")
    return d


def _on_gpu(first: torch.Tensor, *others) -> None:
    dev = first.get_device()                     # -1 on the host
    if dev < 0 or dev != torch.cuda.current_device():
        raise ValueError("tensors must be on the current GPU")
    for t in others:
        if t is not None and t.get_device() != dev:
            raise ValueError("tensors must be on the current GPU")


def _rows_of(t: torch.Tensor, shape, dtype, what: str) -> int:
    """Elements from row to row of a tensor seen as rows of its last dimension."""
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{what} must be {dtype} of shape {tuple(shape)}")
    if t.is_contiguous():
        return shape[-1]
    if t.stride(-1) != 1 and shape[-1] > 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")
    if t.dim() != 2:
        try:
            t = t.view(-1, shape[-1])
        except RuntimeError:
            raise ValueError(f"{what}: rows must lie at one stride") from None
    return t.stride(0)


def _dense(t: Optional[torch.Tensor], shape, dtype, what: str):
    if t is not None and (t.dtype != dtype or t.shape != shape or not t.is_contiguous()):
        raise ValueError(f"{what} must be contiguous {dtype} of shape {tuple(shape)}")


def _strides(t: torch.Tensor, shape, dtype, what: str):
    """Strides of a [batch, token, head, dim] tensor."""
    if t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{what} must be {dtype} of shape {tuple(shape)}")
    s = t.stride()
    if s[3] != 1 and shape[3] > 1:
        raise ValueError(f"{what}: the last dimension must be contiguous")
    return s[:3]


def _written(t: torch.Tensor, what: str) -> None:
    """An output whose elements share memory (an expanded view) has no result."""
    st = t.stride()
    if 0 in st and any(s == 0 and n > 1 for n, s in zip(t.shape, st)):
        raise ValueError(f"{what} is an output and must not be an expanded view")


def _scratch(given: Optional[torch.Tensor], need: int, stream):
    """The caller's scratch, or one from torch's allocator that belongs to the call's stream."""
    if given is not None:
        if not given.is_contiguous():
            raise ValueError("scratch must be contiguous")
        return given, given.numel() * given.element_size()
    if not need:
        return None, 0
    if stream is None:
        return torch.empty(need, dtype=torch.uint8, device="cuda"), need
    s = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream))
    with torch.cuda.stream(s):
        return torch.empty(need, dtype=torch.uint8, device="cuda"), need


def pd_rmsnorm_forward(x: torch.Tensor, weight: torch.Tensor, y: torch.Tensor,
                       residual: Optional[torch.Tensor] = None,
                       sum_out: Optional[torch.Tensor] = None,
                       scale: Optional[torch.Tensor] = None,
                       rstd: Optional[torch.Tensor] = None, eps: float = 1e-6, group: int = 0,
                       stream=None) -> None:
    """y = norm(x + residual) * weight over the last dimension; y of x's type, or float8_e4m3fn
    with `scale` [rows, ceil(width / group)] (group 0: one a row).  sum_out: x + residual."""
    dt, sh = _dtype(x), x.shape
    _on_gpu(x, weight, y, residual, sum_out, scale, rstd)
    width = sh[-1] if x.dim() else 0
    if not width:
        raise ValueError("x must have a last dimension of at least 1")
    rows = x.numel() // width
    f8 = y.dtype == torch.float8_e4m3fn
    _dense(weight, (width,), torch.float32, "weight")
    if f8:
        if scale is None:
            raise ValueError("an output in 8 bits needs scale")
        per = -(-width // group) if group > 0 else 1
        if scale.dtype != torch.float32 or not scale.is_contiguous() or scale.numel() != rows * per:
            raise ValueError(f"scale must be contiguous float32 of {rows} x {per} elements")
    if rstd is not None and (rstd.dtype != torch.float32 or not rstd.is_contiguous() or rstd.numel() != rows):
        raise ValueError(f"rstd must be contiguous float32 of {rows} elements")
    for t in (y, sum_out):
        if t is not None:
            _written(t, "y or sum_out")
    d = _pack(_RMSNORM_BYTES, rows, width, _rows_of(x, sh, x.dtype, "x"),
                     _rows_of(residual, sh, x.dtype, "residual") if residual is not None else 0,
                     _rows_of(sum_out, sh, x.dtype, "sum_out") if sum_out is not None else 0,
                     _rows_of(y, sh, y.dtype if f8 else x.dtype, "y"),
                     dt, PD_F8E4M3 if f8 else dt, group, eps)
    _check(load().pd_rmsnorm_forward(d, _ptr(x), _ptr(residual), _ptr(weight),
                                     _ptr(sum_out), _ptr(y), _ptr(scale), _ptr(rstd), _stream(stream)))


def pd_rmsnorm_backward(dy: torch.Tensor, sum_in: torch.Tensor, weight: torch.Tensor,
                        rstd: torch.Tensor, dx: torch.Tensor,
                        dweight: Optional[torch.Tensor] = None,
                        dsum: Optional[torch.Tensor] = None,
                        scratch: Optional[torch.Tensor] = None, stream=None) -> None:
    """Gradients of pd_rmsnorm_forward from its sum_out (sum_in) and rstd: dx (of x and of
    residual) and dweight.  dsum: the gradient that reaches sum_out from elsewhere."""
    dt, sh = _dtype(dy), dy.shape
    _on_gpu(dy, sum_in, weight, rstd, dx, dweight, dsum, scratch)
    width = sh[-1] if dy.dim() else 0
    if not width:
        raise ValueError("dy must have a last dimension of at least 1")
    rows = dy.numel() // width
    _dense(weight, (width,), torch.float32, "weight")
    _dense(dweight, (width,), torch.float32, "dweight")
    if rstd.dtype != torch.float32 or not rstd.is_contiguous() or rstd.numel() != rows:
        raise ValueError(f"rstd must be contiguous float32 of {rows} elements")
    _written(dx, "dx")
    d = _pack(_RMSNORM_BYTES, rows, width, _rows_of(dx, sh, dy.dtype, "dx"),
                     _rows_of(dsum, sh, dy.dtype, "dsum") if dsum is not None else 0,
                     _rows_of(sum_in, sh, dy.dtype, "sum_in"), _rows_of(dy, sh, dy.dtype, "dy"),
                     dt, dt, 0, 0.0)
    L, need = load(), ctypes.c_int64(0)
    if dweight is not None:
        _check(L.pd_rmsnorm_backward_scratch(d, ctypes.byref(need)))
    buf, have = _scratch(scratch, need.value, stream)
    _check(L.pd_rmsnorm_backward(d, _ptr(dy), _ptr(sum_in), _ptr(weight), _ptr(rstd),
                                 _ptr(dsum), _ptr(dx), _ptr(dweight), _ptr(buf), have, _stream(stream)))


def pd_rotary_table(table: torch.Tensor, base: float = 10000.0, scaling: int = PD_ROTARY_PLAIN,
                    factor: float = 1.0, original_length: float = 0.0, turns_low: float = 1.0,
                    turns_high: float = 32.0, magnitude: float = 1.0, first: int = 0,
                    stream=None) -> None:
    """Fill table [positions, rotary_dim / 2, 2] with cos and sin from position `first` on."""
    _on_gpu(table)
    if table.dtype != torch.float32 or table.dim() != 3 or table.shape[2] != 2 or not table.is_contiguous():
        raise ValueError("table must be contiguous float32 of shape (positions, rotary_dim / 2, 2)")
    d = _RotaryTableDesc(2 * table.shape[1], scaling, base, factor, original_length, turns_low,
                         turns_high, magnitude)
    _check(load().pd_rotary_table(ctypes.byref(d), first, table.shape[0], _ptr(table), _stream(stream)))


_NO_STRIDES = (0, 0, 0)


def pd_rotary_apply(q: torch.Tensor, k: Optional[torch.Tensor], positions: torch.Tensor,
                    table: torch.Tensor, q_out: torch.Tensor, k_out: Optional[torch.Tensor] = None,
                    layout: int = PD_ROTARY_HALF, backward: bool = False, stream=None) -> None:
    """Turn q and k [batch, token, head, dim] by the table's rows at positions ([token] or
    [batch, token], int32); q_out may be q, k_out may be k."""
    dt = _dtype(q)
    _on_gpu(q, k, positions, table, q_out, k_out)
    if q.dim() != 4 or (k is None) != (k_out is None):
        raise ValueError("q must be (batch, token, head, dim), and k_out goes with k")
    B, n, H, D = q.shape
    if table.dtype != torch.float32 or table.dim() != 3 or table.shape[2] != 2 or not table.is_contiguous():
        raise ValueError("table must be contiguous float32 of shape (positions, rotary_dim / 2, 2)")
    shape = tuple(positions.shape)
    if positions.dtype != torch.int32 or shape not in ((n,), (B, n)) or (n > 1 and positions.stride(-1) != 1):
        raise ValueError("positions must be int32 of shape (token,) or (batch, token), tokens contiguous")
    K = 0
    if k is not None:
        if k.dim() != 4:
            raise ValueError("k must be (batch, token, head, dim)")
        K = k.shape[2]
        _written(k_out, "k_out")
    _written(q_out, "q_out")
    ks = (B, n, K, D)
    d = _pack(_ROTARY_BYTES, B, n, H, K, D, 2 * table.shape[1], layout, dt, bool(backward), table.shape[0],
                           positions.stride(0) if len(shape) == 2 else 0,
                           *_strides(q, q.shape, q.dtype, "q"),
                           *(_strides(k, ks, q.dtype, "k") if K else _NO_STRIDES),
                           *_strides(q_out, q.shape, q.dtype, "q_out"),
                           *(_strides(k_out, ks, q.dtype, "k_out") if K else _NO_STRIDES))
    _check(load().pd_rotary_apply(d, _ptr(q), _ptr(k), _ptr(positions), _ptr(table), _ptr(q_out),
                                  _ptr(k_out), _stream(stream)))


def _attention(q, k, v, out, lse, causal, window, sinks, scale, q_lens, kv_lens, grads=_NO_STRIDES * 4):
    dt = _dtype(q)
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q and k must be (batch, token, head, dim)")
    B, n, H, D = q.shape
    ks = (B, k.shape[1], k.shape[2], D)
    if max(B, n, H, D, ks[1], ks[2]) > 0x7fffffff:
        raise ValueError("a dimension is longer than 2^31 - 1")
    _written(out, "out")
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != (B, H, n) or not lse.is_contiguous()):
        raise ValueError(f"lse must be contiguous float32 of shape {(B, H, n)}")
    for t, what in ((q_lens, "q_lens"), (kv_lens, "kv_lens")):
        if t is not None and (t.dtype != torch.int32 or t.shape != (B,) or not t.is_contiguous()):
            raise ValueError(f"{what} must be contiguous int32 of shape {(B,)}")
    sh, t = q.shape, q.dtype
    return _pack(
        _ATTENTION_BYTES, B, H, ks[2], D, n, ks[1], dt, bool(causal), min(window, 0x7fffffff), min(sinks, 0x7fffffff),
        D ** -0.5 if scale is None else scale, *_strides(q, sh, t, "q"), *_strides(k, ks, t, "k"),
        *_strides(v, ks, t, "v"), *_strides(out, sh, t, "out"), *grads)


def pd_attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                         lse: Optional[torch.Tensor] = None, causal: bool = True, window: int = 0,
                         sinks: int = 0, scale: Optional[float] = None,
                         q_lens: Optional[torch.Tensor] = None,
                         kv_lens: Optional[torch.Tensor] = None,
                         scratch: Optional[torch.Tensor] = None, stream=None) -> None:
    """Attention of q on k, v, all [batch, token, head, dim] at any strides (a head-major cache is
    a transposed view); lse float32 [batch, head, token]; scale: default dim ** -0.5."""
    _on_gpu(q, k, v, out, lse, q_lens, kv_lens, scratch)
    d = _attention(q, k, v, out, lse, causal, window, sinks, scale, q_lens, kv_lens)
    L, need = load(), ctypes.c_int64(0)
    if scratch is None:
        _check(L.pd_attention_forward_scratch(d, ctypes.byref(need)))
    buf, have = _scratch(scratch, need.value, stream)
    _check(L.pd_attention_forward(d, _ptr(q), _ptr(k), _ptr(v), _ptr(q_lens),
                                  _ptr(kv_lens), _ptr(out), _ptr(lse), _ptr(buf), have,
                                  _stream(stream)))


def pd_attention_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                          lse: torch.Tensor, dout: torch.Tensor, dq: torch.Tensor,
                          dk: torch.Tensor, dv: torch.Tensor, causal: bool = True, window: int = 0,
                          sinks: int = 0, scale: Optional[float] = None,
                          q_lens: Optional[torch.Tensor] = None,
                          kv_lens: Optional[torch.Tensor] = None,
                          scratch: Optional[torch.Tensor] = None, stream=None) -> None:
    """Gradients dq, dk, dv of pd_attention_forward, from its out and lse and the gradient dout."""
    _on_gpu(q, k, v, out, lse, dout, dq, dk, dv, q_lens, kv_lens, scratch)
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q and k must be (batch, token, head, dim)")
    grads = []
    for t, like, what in ((dq, q, "dq"), (dk, k, "dk"), (dv, k, "dv"), (dout, q, "dout")):
        if t is not dout:
            _written(t, what)
        grads += _strides(t, like.shape, q.dtype, what)
    d = _attention(q, k, v, out, lse, causal, window, sinks, scale, q_lens, kv_lens, grads)
    L, need = load(), ctypes.c_int64(0)
    if scratch is None:
        _check(L.pd_attention_backward_scratch(d, ctypes.byref(need)))
    buf, have = _scratch(scratch, need.value, stream)
    _check(L.pd_attention_backward(d, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse),
                                   _ptr(dout), _ptr(q_lens), _ptr(kv_lens), _ptr(dq), _ptr(dk),
                                   _ptr(dv), _ptr(buf), have, _stream(stream)))


# ------------------------------------------------------------ workload helpers
def from_workload(w, weights: Dict[str, np.ndarray], tol_index_offset: int = 0,
                  rule: str = "relaxed"):
    """(schedule, denoiser) handles for a ``workloads.Workload``.  The schedule
    carries the training chain (T_train, abar) that the denoiser needs, and
    the stride test's reading (``tol_index_offset``) and rule ("relaxed" or
    "prop2")."""
    s = w.schedule
    if s.kind == "ddpm":
        kind = PD_DDPM
    else:
        kind = {"euler": PD_DDIM, "heun": PD_DDIM_HEUN,
                "dpm2m": PD_DDIM_DPM2M}[getattr(s, "solver", "euler")]
    sched = pd_init_schedule(kind, s.T_train, s.T, s.beta_start, s.beta_end, s.eta,
                             tol_index_offset, STOP_RULES[rule])
    m = w.model
    mk = {"gmm2d": PD_MODEL_GMM2D, "mlp": PD_MODEL_MLP, "conv1x1": PD_MODEL_CONV1X1}[m.kind]
    den = pd_denoiser_create(mk, m.sample_shape, weights, sched, width=m.width,
                             dtype=PD_BF16 if m.dtype == "bf16" else PD_F32,
                             cond_dim=m.cond_dim, guidance=m.guidance,
                             n_components=m.n_components if m.kind == "gmm2d" else 0)
    return sched, den
