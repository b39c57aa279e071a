"""ctypes binding of libgbmuf.so: argument marshalling only, same names as include/gbmuf.h.

Device buffers are passed as integers (``tensor.data_ptr()``) or as any object with a
``data_ptr()`` method; streams as ``torch.cuda.Stream.cuda_stream`` integers (0/None = the
default stream).  Nothing here computes: every step runs in the library's kernels.  If the
library has not been built the import of this module fails loudly.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np
import torch  # noqa: F401  -- first: libgbmuf must bind to the HIP runtime that torch has loaded, not a second copy

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgbmuf.so")

GBMUF_OK, GBMUF_EINVAL, GBMUF_ENOMEM, GBMUF_EDEVICE, GBMUF_EUNSUPPORTED = 0, 1, 2, 3, 4
MODE_NO_RESTART, MODE_PAPER, MODE_LITERAL, MODE_GOSSIP_MA = 0, 1, 2, 3
SAMPLING_AUTO, SAMPLING_IN_KERNEL, SAMPLING_SEPARATE = 0, 1, 2
SWEEP_AUTO, SWEEP_FORWARD = 0, 1
LAYOUT_ROWS, LAYOUT_BLOCKED = 0, 1
MAX_K = 1024
STATIC_TABLE_ENTRIES = 1 << 19
MAX_TOP = 1024
F32, BF16, F16 = 0, 1, 2
ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU, ACT_SIGMOID, ACT_TANH = range(6)
RESIDUAL_NONE, RESIDUAL_BEFORE, RESIDUAL_AFTER = 0, 1, 2
_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


class GbmufError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        detail = _lib.gbmuf_last_error_detail().decode()
        super().__init__(f"{what}: {strerror(code)} (status {code})" + (f" [{detail}]" if detail else ""))


class Info(ctypes.Structure):
    _fields_ = [("m", ctypes.c_int32), ("K", ctypes.c_int32), ("q", ctypes.c_int32), ("p", ctypes.c_int32),
                ("C", ctypes.c_int32), ("has_device", ctypes.c_int32), ("P", ctypes.c_int64),
                ("n_tiles", ctypes.c_int64), ("tile_columns", ctypes.c_int32), ("threads", ctypes.c_int32),
                ("seed", ctypes.c_uint64), ("mixed_q", ctypes.c_int32), ("has_periods", ctypes.c_int32),
                ("in_kernel_sampling", ctypes.c_int32), ("tile_columns_blocked", ctypes.c_int32),
                ("threads_blocked", ctypes.c_int32), ("workgroups_per_cu_blocked", ctypes.c_int32),
                ("tile_columns_blocked_ma", ctypes.c_int32), ("min_block_floats", ctypes.c_int32)]


class PlanDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("m", ctypes.c_int32), ("K", ctypes.c_int32), ("q", ctypes.c_int32),
                ("comp_offsets", ctypes.c_void_p), ("q_per_component", ctypes.c_void_p), ("periods", ctypes.c_void_p),
                ("p", ctypes.c_int32), ("reserved0", ctypes.c_int32), ("seed", ctypes.c_uint64),
                ("tile_threads", ctypes.c_int32), ("tile_slots", ctypes.c_int32), ("sampling", ctypes.c_int32),
                ("sweep", ctypes.c_int32), ("cache_hints", ctypes.c_int32), ("workgroups_per_cu", ctypes.c_int32)]


class State(ctypes.Structure):
    """gbmuf_state_t: where theta, omega, delta are (device pointers as integers) and how they are laid out."""
    _fields_ = [("theta", ctypes.c_void_p), ("omega", ctypes.c_void_p), ("delta", ctypes.c_void_p),
                ("worker_stride", ctypes.c_int64), ("block_floats", ctypes.c_int64), ("block_stride", ctypes.c_int64)]


class Layout(ctypes.Structure):
    _fields_ = [("worker_stride", ctypes.c_int64), ("block_floats", ctypes.c_int64), ("block_stride", ctypes.c_int64),
                ("omega_offset", ctypes.c_int64), ("delta_offset", ctypes.c_int64), ("arena_floats", ctypes.c_int64)]


class LinearDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("batch", ctypes.c_int32),
                ("activation", ctypes.c_int32), ("residual", ctypes.c_int32), ("weight_grad_f32", ctypes.c_int32),
                ("accumulate", ctypes.c_int32), ("reserved0", ctypes.c_int32), ("rows", ctypes.c_int64),
                ("out_features", ctypes.c_int64), ("in_features", ctypes.c_int64)]


class Matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("ld", ctypes.c_int64), ("batch_stride", ctypes.c_int64)]


class _LinearIo(ctypes.Structure):
    tensors = ()                    # kept alive as long as their addresses are here
    on_host = False


class LinearIo(_LinearIo):
    _fields_ = [(n, Matrix) for n in ("x", "w", "bias", "residual", "y", "pre")]


class LinearGradIo(_LinearIo):
    _fields_ = [(n, Matrix) for n in ("x", "w", "pre", "dy", "dx", "dw", "dbias", "dresidual")]


class LossDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", ctypes.c_int32), ("batch", ctypes.c_int32), ("top", ctypes.c_int32),
                ("weight_grad_f32", ctypes.c_int32), ("accumulate", ctypes.c_int32), ("temperature", ctypes.c_float),
                ("reserved0", ctypes.c_int32), ("rows", ctypes.c_int64), ("vocab", ctypes.c_int64), ("in_features", ctypes.c_int64)]


class LossIo(_LinearIo):
    _fields_ = [(n, Matrix) for n in ("x", "w", "bias", "target", "teacher", "loss", "lse")]


class LossGradIo(_LinearIo):
    _fields_ = [(n, Matrix) for n in ("x", "w", "bias", "target", "teacher", "lse", "dloss", "dx", "dw", "dbias")]


class GradTensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("row_stride", ctypes.c_int64),
                ("offset", ctypes.c_int64), ("worker", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class GradsDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("workers", ctypes.c_int32), ("n_tensors", ctypes.c_int64),
                ("tensors", ctypes.c_void_p)]


class StepDesc(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("skip_nonfinite", ctypes.c_int32), ("P", ctypes.c_int64),
                ("rate", ctypes.c_float), ("eps", ctypes.c_float), ("max_norm", ctypes.c_float), ("reserved0", ctypes.c_float)]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        # nothing built yet: build once with hipcc; there is no other (CPU, eager) path to fall back to
        try:
            from .build import build_library
            build_library(verbose=False)
        except Exception as e:  # noqa: BLE001
            raise ImportError(
                f"{LIB_PATH} is missing and could not be built ({e!r}): run "
                "python -c 'import __graft_entry__ as g; g.build()'.  There is no fallback path.") from e
    L = ctypes.CDLL(LIB_PATH)
    i32, i64, u64, f32, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_float, ctypes.c_void_p
    L.gbmuf_plan.argtypes = [ctypes.POINTER(vp), vp, i32, i32, i32, i32, u64]
    L.gbmuf_plan_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(PlanDesc)]
    L.gbmuf_plan_destroy.argtypes = [vp]
    L.gbmuf_plan_info.argtypes = [vp, ctypes.POINTER(Info)]
    L.gbmuf_candidates_host.argtypes = [vp, i32, vp]
    L.gbmuf_neighbours_host.argtypes = [vp, u64, vp]
    L.gbmuf_neighbours_device.argtypes = [vp, u64, vp, vp]
    L.gbmuf_sync.argtypes = [vp, vp, vp, vp, i64, f32, f32, i32, u64, vp]
    L.gbmuf_sync_table.argtypes = [vp, vp, vp, vp, vp, i64, f32, f32, i32, vp]
    L.gbmuf_sync_step.argtypes = [vp, vp, vp, vp, i64, f32, f32, i32, u64, vp]
    L.gbmuf_final_average.argtypes = [vp, vp, i64, vp, vp]
    sp = ctypes.POINTER(State)
    L.gbmuf_sync_state.argtypes = [vp, sp, f32, f32, i32, u64, vp]
    L.gbmuf_sync_step_state.argtypes = [vp, sp, f32, f32, i32, u64, vp]
    L.gbmuf_sync_static.argtypes = [vp, sp, f32, f32, i32, u64, vp]
    L.gbmuf_sync_static.restype = ctypes.c_int
    L.gbmuf_sync_table_state.argtypes = [vp, vp, sp, f32, f32, i32, vp]
    L.gbmuf_final_average_state.argtypes = [vp, sp, vp, vp]
    L.gbmuf_state_copy.argtypes = [vp, sp, sp, i32, vp]
    L.gbmuf_recommend_layout.argtypes = [vp, i64, i32, i32, ctypes.POINTER(Layout)]
    for name in ("gbmuf_plan_create", "gbmuf_sync_step", "gbmuf_final_average", "gbmuf_sync_state",
                 "gbmuf_sync_step_state", "gbmuf_sync_table_state", "gbmuf_final_average_state", "gbmuf_state_copy",
                 "gbmuf_recommend_layout"):
        getattr(L, name).restype = ctypes.c_int
    L.gbmuf_probe_copy.argtypes = [vp, vp, i64, i32, vp]
    L.gbmuf_probe_copy.restype = ctypes.c_int
    ld, lo, gp = ctypes.POINTER(LinearDesc), ctypes.POINTER(LossDesc), ctypes.POINTER(vp)
    for name, args in (("gbmuf_linear_workspace", [ld, i32, ctypes.POINTER(i64)]),
                       ("gbmuf_linear", [ld, ctypes.POINTER(LinearIo), vp, i64, vp]),
                       ("gbmuf_linear_backward", [ld, ctypes.POINTER(LinearGradIo), vp, i64, vp]),
                       ("gbmuf_loss_workspace", [lo, i32, ctypes.POINTER(i64)]),
                       ("gbmuf_cross_entropy", [lo, ctypes.POINTER(LossIo), vp, i64, vp]),
                       ("gbmuf_cross_entropy_backward", [lo, ctypes.POINTER(LossGradIo), vp, i64, vp]),
                       ("gbmuf_distill", [lo, ctypes.POINTER(LossIo), vp, i64, vp]),
                       ("gbmuf_distill_backward", [lo, ctypes.POINTER(LossGradIo), vp, i64, vp]),
                       ("gbmuf_grads_create", [gp, ctypes.POINTER(GradsDesc)]), ("gbmuf_grads_destroy", [vp]),
                       ("gbmuf_grad_norm", [vp, vp, vp]), ("gbmuf_grad_clip", [vp, vp, f32, vp, vp]),
                       ("gbmuf_local_step", [vp, ctypes.POINTER(StepDesc), sp, sp, vp, vp])):
        getattr(L, name).argtypes = args
        getattr(L, name).restype = ctypes.c_int
    L.gbmuf_strerror.argtypes = [ctypes.c_int]
    L.gbmuf_strerror.restype = ctypes.c_char_p
    L.gbmuf_last_error_detail.argtypes = []
    L.gbmuf_last_error_detail.restype = ctypes.c_char_p
    for name in ("gbmuf_plan", "gbmuf_plan_destroy", "gbmuf_plan_info", "gbmuf_candidates_host",
                 "gbmuf_neighbours_host", "gbmuf_neighbours_device", "gbmuf_sync", "gbmuf_sync_table"):
        getattr(L, name).restype = ctypes.c_int
    return L


_lib = _load()
# calls that take microseconds: no look-up each time
_linear, _linear_backward = _lib.gbmuf_linear, _lib.gbmuf_linear_backward
_grad_norm, _grad_clip, _local_step = _lib.gbmuf_grad_norm, _lib.gbmuf_grad_clip, _lib.gbmuf_local_step


def lib() -> ctypes.CDLL:
    return _lib


def strerror(code: int) -> str:
    return _lib.gbmuf_strerror(code).decode()


def _dev(x) -> Optional[int]:
    if x is None:
        return None
    if hasattr(x, "data_ptr"):
        return int(x.data_ptr())
    return int(x)


def _stream(s) -> Optional[int]:
    if s is None:
        return None
    return int(getattr(s, "cuda_stream", s)) or None


def recommend_layout(P: int, K: int, kind: int = LAYOUT_BLOCKED, plan: "Optional[Plan]" = None) -> Layout:
    out = Layout()
    rc = _lib.gbmuf_recommend_layout(plan._h if plan is not None else None, P, K, kind, ctypes.byref(out))
    if rc != GBMUF_OK:
        raise GbmufError(rc, "gbmuf_recommend_layout")
    return out


def make_state(theta, omega, delta, worker_stride: int, block_floats: int = 0, block_stride: int = 0) -> State:
    return State(_dev(theta), _dev(omega), _dev(delta), worker_stride, block_floats, block_stride)


def probe_copy(dst_dev, src_dev, n_floats: int, flags: int = 0, stream=None) -> None:
    rc = _lib.gbmuf_probe_copy(_dev(dst_dev), _dev(src_dev), n_floats, flags, _stream(stream))
    if rc != GBMUF_OK:
        raise GbmufError(rc, "gbmuf_probe_copy")


class Plan:
    """Owns one ``gbmuf_plan_t``.  Methods mirror the C entry points one to one."""

    def __init__(self, comp_offsets: Sequence[int], K: int, q=0, p: int = 0, seed: int = 0, periods=None,
                 tile=None, sampling: int = SAMPLING_AUTO, sweep: int = SWEEP_AUTO, cache_hints: int = 0,
                 workgroups_per_cu: int = 0):
        """gbmuf_plan_create.  ``q``: an int, or a sequence of m ints (neighbours per component).
        ``periods``: m sync periods H_i or None.  ``tile``: (threads, slots) or None."""
        off = np.ascontiguousarray(comp_offsets, dtype=np.int64)
        if off.ndim != 1 or off.size < 1:
            raise GbmufError(GBMUF_EINVAL, "gbmuf_plan_create")
        m = off.size - 1
        d = PlanDesc()
        d.struct_size = ctypes.sizeof(PlanDesc)
        d.m, d.K, d.p, d.seed = m, K, p, seed & 0xFFFFFFFFFFFFFFFF
        d.comp_offsets = off.ctypes.data
        keep = [off]
        if np.ndim(q) == 0:
            d.q = int(q)
        else:
            qv = np.ascontiguousarray(q, dtype=np.int32)
            if qv.shape != (m,):
                raise GbmufError(GBMUF_EINVAL, "gbmuf_plan_create")
            d.q_per_component = qv.ctypes.data if m else None
            keep.append(qv)
        if periods is not None:
            h = np.ascontiguousarray(periods, dtype=np.int32)
            if h.shape != (m,):
                raise GbmufError(GBMUF_EINVAL, "gbmuf_plan_create")
            d.periods = h.ctypes.data if m else None
            keep.append(h)
        if tile is not None:
            d.tile_threads, d.tile_slots = int(tile[0]), int(tile[1])
        d.sampling, d.sweep, d.cache_hints, d.workgroups_per_cu = sampling, sweep, cache_hints, workgroups_per_cu
        self._h = ctypes.c_void_p()
        rc = _lib.gbmuf_plan_create(ctypes.byref(self._h), ctypes.byref(d))
        del keep
        if rc != GBMUF_OK:
            self._h = ctypes.c_void_p()
            raise GbmufError(rc, "gbmuf_plan_create")
        self.info = self.plan_info()

    def destroy(self) -> None:
        if getattr(self, "_h", None) is not None and self._h:
            _lib.gbmuf_plan_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def plan_info(self) -> Info:
        info = Info()
        rc = _lib.gbmuf_plan_info(self._h, ctypes.byref(info))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_plan_info")
        return info

    def candidates_host(self, w: int) -> np.ndarray:
        out = np.zeros(max(self.info.C, 1), dtype=np.int32)
        rc = _lib.gbmuf_candidates_host(self._h, w, out.ctypes.data_as(ctypes.c_void_p))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_candidates_host")
        return out[: self.info.C].copy()

    def neighbours_host(self, round: int) -> np.ndarray:
        out = np.full((self.info.m, self.info.K, self.info.q), -1, dtype=np.int32)
        rc = _lib.gbmuf_neighbours_host(self._h, round, out.ctypes.data_as(ctypes.c_void_p))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_neighbours_host")
        return out

    def neighbours_device(self, round: int, out_dev, stream=None) -> None:
        rc = _lib.gbmuf_neighbours_device(self._h, round, _dev(out_dev), _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_neighbours_device")

    def sync(self, replicas, global_, delta, worker_stride: int, eta: float, zeta: float,
             nesterov: int = MODE_PAPER, round: int = 0, stream=None) -> None:
        rc = _lib.gbmuf_sync(self._h, _dev(replicas), _dev(global_), _dev(delta), worker_stride, eta, zeta,
                             nesterov, round, _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_sync")

    def sync_step(self, replicas, global_, delta, worker_stride: int, eta: float, zeta: float,
                  nesterov: int = MODE_PAPER, step: int = 0, stream=None) -> None:
        rc = _lib.gbmuf_sync_step(self._h, _dev(replicas), _dev(global_), _dev(delta), worker_stride, eta, zeta,
                                  nesterov, step, _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_sync_step")

    def final_average(self, replicas, worker_stride: int, out_dev, stream=None) -> None:
        rc = _lib.gbmuf_final_average(self._h, _dev(replicas), worker_stride, _dev(out_dev), _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_final_average")

    def sync_table(self, nbr_dev, replicas, global_, delta, worker_stride: int, eta: float, zeta: float,
                   nesterov: int = MODE_PAPER, stream=None) -> None:
        rc = _lib.gbmuf_sync_table(self._h, _dev(nbr_dev), _dev(replicas), _dev(global_), _dev(delta),
                                   worker_stride, eta, zeta, nesterov, _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_sync_table")

    def sync_state(self, state: State, eta: float, zeta: float, nesterov: int = MODE_PAPER, round: int = 0,
                   stream=None) -> None:
        rc = _lib.gbmuf_sync_state(self._h, ctypes.byref(state), eta, zeta, nesterov, round, _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_sync_state")

    def sync_static(self, state: State, eta: float, zeta: float, nesterov: int = MODE_PAPER, round: int = 0,
                    stream=None) -> None:
        rc = _lib.gbmuf_sync_static(self._h, ctypes.byref(state), eta, zeta, nesterov, round, _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_sync_static")

    def sync_step_state(self, state: State, eta: float, zeta: float, nesterov: int = MODE_PAPER, step: int = 0,
                        stream=None) -> None:
        rc = _lib.gbmuf_sync_step_state(self._h, ctypes.byref(state), eta, zeta, nesterov, step, _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_sync_step_state")

    def sync_table_state(self, nbr_dev, state: State, eta: float, zeta: float, nesterov: int = MODE_PAPER,
                         stream=None) -> None:
        rc = _lib.gbmuf_sync_table_state(self._h, _dev(nbr_dev), ctypes.byref(state), eta, zeta, nesterov,
                                         _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_sync_table_state")

    def final_average_state(self, state: State, out_dev, stream=None) -> None:
        rc = _lib.gbmuf_final_average_state(self._h, ctypes.byref(state), _dev(out_dev), _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_final_average_state")

    def state_copy(self, dst: State, src: State, which: int = 7, stream=None) -> None:
        rc = _lib.gbmuf_state_copy(self._h, ctypes.byref(dst), ctypes.byref(src), which, _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_state_copy")


def _on_host(tensors, what: str) -> bool:
    """Whether tensors lie where no GPU reads them (pinned memory it does); all of them have to lie on one device."""
    devices = {t.device for t in tensors if t is not None and t.numel() and not (t.device.type == "cpu" and t.is_pinned())}
    if len(devices) > 1:
        raise GbmufError(GBMUF_EINVAL, what + ": tensors of several devices")
    return any(d.type != "cuda" for d in devices)


def _refuse_host(what: str) -> None:
    """Without a GPU the library itself says what is missing."""
    if torch.cuda.is_available():
        raise GbmufError(GBMUF_EINVAL, what + ": a tensor in the host's memory")


def _norms(t, workers: int, what: str) -> Optional[int]:
    if not isinstance(t, torch.Tensor):
        return _dev(t)
    if t.dtype is not torch.float32 or t.numel() < workers or not t.is_contiguous():
        raise GbmufError(GBMUF_EINVAL, what + ": norms are `workers` floats")
    if not t.is_cuda and not t.is_pinned():
        _refuse_host(what)
    return t.data_ptr()


def _matrix(t, batch: int, rows: int, cols: int, dtype, what: str) -> Matrix:
    """A [batch, rows, cols] tensor (or [rows, cols] where batch is 1) whose last axis is contiguous, as gbmuf_matrix_t."""
    if t is None:
        return Matrix()
    if t.dim() == 2 and batch == 1:
        t = t.unsqueeze(0)
    if tuple(t.shape) != (batch, rows, cols) or t.dtype != dtype or (cols > 1 and t.stride(2) != 1):
        raise GbmufError(GBMUF_EINVAL, what)
    return Matrix(t.data_ptr(), t.stride(1), t.stride(0))


def _vector(t, batch: int, cols: int, dtype, what: str) -> Matrix:
    if t is None:
        return Matrix()
    if t.dim() == 1 and batch == 1:
        t = t.unsqueeze(0)
    if tuple(t.shape) != (batch, cols) or t.dtype != dtype or (cols > 1 and t.stride(1) != 1):
        raise GbmufError(GBMUF_EINVAL, what)
    return Matrix(t.data_ptr(), 0, t.stride(0))


class Linear:
    """gbmuf_linear_desc_t: one product y = act(x w' + bias ...) for each of ``batch`` workers.  Tensors are [batch, rows, columns] (or
    [rows, columns] where batch is 1), views with strides among them; ``forward_io`` / ``backward_io`` check them, keep them alive
    and return what ``forward`` / ``backward`` take, as often as is wanted."""

    def __init__(self, rows: int, out_features: int, in_features: int, batch: int = 1, dtype=torch.float32,
                 activation: int = ACT_NONE, residual: int = RESIDUAL_NONE, weight_grad_f32: bool = False, accumulate: bool = False):
        if dtype not in _TYPES:
            raise GbmufError(GBMUF_EINVAL, "gbmuf_linear_desc_t")
        self.dtype, self.grad_dtype = dtype, torch.float32 if weight_grad_f32 else dtype
        self.desc = LinearDesc(ctypes.sizeof(LinearDesc), _TYPES[dtype], batch, activation, residual, int(weight_grad_f32),
                               int(accumulate), 0, rows, out_features, in_features)
        self._at = ctypes.byref(self.desc)
        self.workspace_bytes()                               # the description's own checks

    def workspace_bytes(self, backward: bool = False) -> int:
        n = ctypes.c_int64()
        rc = _lib.gbmuf_linear_workspace(self._at, int(backward), ctypes.byref(n))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_linear_workspace")
        return n.value

    def forward_io(self, x, w, y, bias=None, residual=None, pre=None) -> LinearIo:
        d, t = self.desc, self.dtype
        G, M, N, K = d.batch, d.rows, d.out_features, d.in_features
        io = LinearIo(_matrix(x, G, M, K, t, "x"), _matrix(w, G, N, K, t, "w"), _vector(bias, G, N, t, "bias"),
                      _matrix(residual, G, M, N, t, "residual"), _matrix(y, G, M, N, t, "y"), _matrix(pre, G, M, N, t, "pre"))
        io.tensors = (x, w, y, bias, residual, pre)
        io.on_host = _on_host(io.tensors, "gbmuf_linear")
        return io

    def backward_io(self, dy, x=None, w=None, pre=None, dx=None, dw=None, dbias=None, dresidual=None) -> LinearGradIo:
        d, t, gt = self.desc, self.dtype, self.grad_dtype
        G, M, N, K = d.batch, d.rows, d.out_features, d.in_features
        io = LinearGradIo(_matrix(x, G, M, K, t, "x"), _matrix(w, G, N, K, t, "w"), _matrix(pre, G, M, N, t, "pre"),
                          _matrix(dy, G, M, N, t, "dy"), _matrix(dx, G, M, K, t, "dx"), _matrix(dw, G, N, K, gt, "dw"),
                          _vector(dbias, G, N, gt, "dbias"), _matrix(dresidual, G, M, N, t, "dresidual"))
        io.tensors = (dy, x, w, pre, dx, dw, dbias, dresidual)
        io.on_host = _on_host(io.tensors, "gbmuf_linear_backward")
        return io

    def forward(self, io: LinearIo, workspace=None, stream=None) -> None:
        if io.on_host or (workspace is not None and not workspace.is_cuda and not workspace.is_pinned()):
            _refuse_host("gbmuf_linear")
        if workspace is None:
            rc = _linear(self._at, ctypes.byref(io), None, 0, _stream(stream))
        else:
            rc = _linear(self._at, ctypes.byref(io), workspace.data_ptr(), workspace.nbytes, _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_linear")

    def backward(self, io: LinearGradIo, workspace=None, stream=None) -> None:
        if io.on_host or (workspace is not None and not workspace.is_cuda and not workspace.is_pinned()):
            _refuse_host("gbmuf_linear_backward")
        if workspace is None:
            rc = _linear_backward(self._at, ctypes.byref(io), None, 0, _stream(stream))
        else:
            rc = _linear_backward(self._at, ctypes.byref(io), workspace.data_ptr(), workspace.nbytes, _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_linear_backward")


def _column(t, batch: int, rows: int, dtype, what: str) -> Matrix:
    """A [batch, rows] tensor (or [rows] where batch is 1) with any strides, as a gbmuf_matrix_t of one column."""
    if t is None:
        return Matrix()
    if t.dim() == 1 and batch == 1:
        t = t.unsqueeze(0)
    if tuple(t.shape) != (batch, rows) or t.dtype != dtype:
        raise GbmufError(GBMUF_EINVAL, what)
    return Matrix(t.data_ptr(), t.stride(1), t.stride(0))


class _Loss:
    """gbmuf_loss_desc_t: a loss over a vocabulary for each of ``batch`` workers, from the rows x that go into its output matrix w, whose
    logits are never kept.  Tensors are [batch, rows, columns], [batch, rows] or, the bias, [batch, vocab] (without the first where batch is 1), views with
    strides among them; ``forward_io`` / ``backward_io`` check them, keep them alive and return what ``forward`` / ``backward``
    take, as often as is wanted."""

    _top = 0

    def __init__(self, rows: int, vocab: int, in_features: int, batch: int, dtype, weight_grad_f32: bool, accumulate: bool, temperature: float):
        if dtype not in _TYPES:
            raise GbmufError(GBMUF_EINVAL, "gbmuf_loss_desc_t")
        self.dtype, self.grad_dtype = dtype, torch.float32 if weight_grad_f32 else dtype
        self.desc = LossDesc(ctypes.sizeof(LossDesc), _TYPES[dtype], batch, self._top, int(weight_grad_f32), int(accumulate), temperature, 0,
                             rows, vocab, in_features)
        self._at = ctypes.byref(self.desc)
        self.workspace_bytes()                               # the description's own checks

    def workspace_bytes(self, backward: bool = False) -> int:
        n = ctypes.c_int64()
        rc = _lib.gbmuf_loss_workspace(self._at, int(backward), ctypes.byref(n))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_loss_workspace")
        return n.value

    def _inputs(self, x, w, bias, target, teacher):
        d, t = self.desc, self.dtype
        G, M, V, K, T = d.batch, d.rows, d.vocab, d.in_features, self._top
        return (_matrix(x, G, M, K, t, "x"), _matrix(w, G, V, K, t, "w"), _vector(bias, G, V, t, "bias"),
                _matrix(target, G, M, T, torch.int64, "words") if T else _column(target, G, M, torch.int64, "target"),
                _matrix(teacher, G, M, T, torch.float32, "teacher"))

    def _forward_io(self, x, w, target, teacher, loss, lse, bias) -> LossIo:
        G, M = self.desc.batch, self.desc.rows
        io = LossIo(*self._inputs(x, w, bias, target, teacher), _column(loss, G, M, torch.float32, "loss"), _column(lse, G, M, torch.float32, "lse"))
        io.tensors = (x, w, target, teacher, loss, lse, bias)
        io.on_host = _on_host(io.tensors, self._names[0])
        return io

    def _backward_io(self, x, w, target, teacher, lse, dloss, bias, dx, dw, dbias) -> LossGradIo:
        d, t, gt = self.desc, self.dtype, self.grad_dtype
        G, M, V, K = d.batch, d.rows, d.vocab, d.in_features
        io = LossGradIo(*self._inputs(x, w, bias, target, teacher), _column(lse, G, M, torch.float32, "lse"),
                        _column(dloss, G, M, torch.float32, "dloss"), _matrix(dx, G, M, K, t, "dx"), _matrix(dw, G, V, K, gt, "dw"),
                        _vector(dbias, G, V, gt, "dbias"))
        io.tensors = (x, w, target, teacher, lse, dloss, bias, dx, dw, dbias)
        io.on_host = _on_host(io.tensors, self._names[1])
        return io

    def _call(self, fn, name, io, workspace, stream) -> None:
        if io.on_host or (workspace is not None and not workspace.is_cuda and not workspace.is_pinned()):
            _refuse_host(name)
        if workspace is None:
            rc = fn(self._at, ctypes.byref(io), None, 0, _stream(stream))
        else:
            rc = fn(self._at, ctypes.byref(io), workspace.data_ptr(), workspace.nbytes, _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, name)

    def forward(self, io: LossIo, workspace=None, stream=None) -> None:
        self._call(self._forward, self._names[0], io, workspace, stream)

    def backward(self, io: LossGradIo, workspace=None, stream=None) -> None:
        self._call(self._backward, self._names[1], io, workspace, stream)


class CrossEntropy(_Loss):
    """Each row is held to one word: target is int64, negative where a row does not count."""

    _forward, _backward = _lib.gbmuf_cross_entropy, _lib.gbmuf_cross_entropy_backward
    _names = ("gbmuf_cross_entropy", "gbmuf_cross_entropy_backward")

    def __init__(self, rows: int, vocab: int, in_features: int, batch: int = 1, dtype=torch.float32, weight_grad_f32: bool = False,
                 accumulate: bool = False):
        super().__init__(rows, vocab, in_features, batch, dtype, weight_grad_f32, accumulate, 1.0)

    def forward_io(self, x, w, target, loss, lse=None, bias=None) -> LossIo:
        return self._forward_io(x, w, target, None, loss, lse, bias)

    def backward_io(self, x, w, target, lse, dloss, bias=None, dx=None, dw=None, dbias=None) -> LossGradIo:
        return self._backward_io(x, w, target, None, lse, dloss, bias, dx, dw, dbias)


class Distill(_Loss):
    """Each row is held to a teacher's logits (f32) of ``top`` words (int64, negative: not there), [batch, rows, top] both, at a temperature."""

    _forward, _backward = _lib.gbmuf_distill, _lib.gbmuf_distill_backward
    _names = ("gbmuf_distill", "gbmuf_distill_backward")

    def __init__(self, rows: int, vocab: int, in_features: int, top: int, temperature: float = 1.0, batch: int = 1, dtype=torch.float32,
                 weight_grad_f32: bool = False, accumulate: bool = False):
        if top < 1:
            raise GbmufError(GBMUF_EINVAL, "gbmuf_loss_desc_t")
        self._top = top
        super().__init__(rows, vocab, in_features, batch, dtype, weight_grad_f32, accumulate, temperature)

    def forward_io(self, x, w, words, teacher, loss, lse=None, bias=None) -> LossIo:
        return self._forward_io(x, w, words, teacher, loss, lse, bias)

    def backward_io(self, x, w, words, teacher, lse, dloss, bias=None, dx=None, dw=None, dbias=None) -> LossGradIo:
        return self._backward_io(x, w, words, teacher, lse, dloss, bias, dx, dw, dbias)


class Grads:
    """Owns one ``gbmuf_grads_t``: the gradients of K workers where they lie.  ``tensors[w]`` lists worker w's tensors in the order of its
    flat parameter vector (vectors, matrices whose last axis is contiguous, or contiguous tensors of any shape); ``offsets[w]``,
    if given, says where each begins among the worker's parameters.  Keeps the tensors alive."""

    def __init__(self, tensors: Sequence[Sequence], offsets: Optional[Sequence[Sequence[int]]] = None):
        rows = []
        for w, ts in enumerate(tensors):
            for i, t in enumerate(ts):
                if t.dtype not in _TYPES:
                    raise GbmufError(GBMUF_EINVAL, "gbmuf_grads_create")
                if t.is_contiguous():
                    shape = (1, t.numel(), t.numel())
                elif t.dim() == 2 and (t.shape[1] <= 1 or t.stride(1) == 1):
                    shape = (t.shape[0], t.shape[1], t.stride(0))
                elif t.dim() == 1:
                    shape = (t.shape[0], 1, t.stride(0))
                else:
                    raise GbmufError(GBMUF_EINVAL, "gbmuf_grads_create")
                rows.append(GradTensor(t.data_ptr(), *shape, -1 if offsets is None else int(offsets[w][i]), w, _TYPES[t.dtype]))
        if _on_host([t for ts in tensors for t in ts], "gbmuf_grads_create"):
            _refuse_host("gbmuf_grads_create")
        table = (GradTensor * max(len(rows), 1))(*rows)
        d = GradsDesc(ctypes.sizeof(GradsDesc), len(tensors), len(rows), ctypes.addressof(table))
        self._h = ctypes.c_void_p()
        rc = _lib.gbmuf_grads_create(ctypes.byref(self._h), ctypes.byref(d))
        if rc != GBMUF_OK:
            self._h = ctypes.c_void_p()
            raise GbmufError(rc, "gbmuf_grads_create")
        self._keep = [list(ts) for ts in tensors]
        self.workers = len(tensors)

    def destroy(self) -> None:
        if getattr(self, "_h", None) is not None and self._h:
            _lib.gbmuf_grads_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def norm(self, norms, stream=None) -> None:
        rc = _grad_norm(self._h, _norms(norms, self.workers, "gbmuf_grad_norm"), _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_grad_norm")

    def clip(self, max_norm: float, norms, out: "Optional[Grads]" = None, stream=None) -> None:
        """In place, or into the tensors of ``out``."""
        rc = _grad_clip(self._h, (out or self)._h, max_norm, _norms(norms, self.workers, "gbmuf_grad_clip"), _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_grad_clip")

    def local_step(self, theta: State, sums: Optional[State], P: int, rate: float, eps: float = 1e-7,
                   max_norm: float = float("inf"), norms=None, skip_nonfinite: bool = False, stream=None) -> None:
        """Adagrad with ``sums`` (a state whose theta holds them), SGD with None.  ``eps`` 0 makes NaN of a parameter whose sum is 0."""
        d = StepDesc(ctypes.sizeof(StepDesc), int(skip_nonfinite), P, rate, eps, max_norm, 0.0)
        rc = _local_step(self._h, ctypes.byref(d), ctypes.byref(theta), ctypes.byref(sums) if sums is not None else None,
                         _norms(norms, self.workers, "gbmuf_local_step"), _stream(stream))
        if rc != GBMUF_OK:
            raise GbmufError(rc, "gbmuf_local_step")
