"""ctypes binding of libqn.so: the same entry points as ``include/qn.h``, arguments marshalled only.

Tensors are ``torch`` CUDA tensors used purely as device memory (``data_ptr()``); streams are
``torch.cuda`` streams passed by handle.  No arithmetic of the method happens in Python.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence, Tuple

import torch

QN_F32 = 0
QN_BF16 = 1
QN_MAX_M = 64
QN_GRAM_PATH_AUTO = 0
QN_GRAM_PATH_PLAIN_ALU = 1
QN_GRAM_PATH_FP64 = 2
QN_TOP_MAX = 128
QN_TEACHER_LOGITS = 0
QN_TEACHER_LOGPROBS = 1
QN_GRAD_MAX_VOCAB = 393208
QN_PREFERENCE_LOGISTIC = 0
QN_PREFERENCE_HINGE = 1
QN_PREFERENCE_SQUARED = 2
QN_ADAM_BLOCK = 32
QN_STATE_F32 = 0
QN_STATE_8BIT = 1
QN_ROUND_NEAREST = 0
QN_ROUND_STOCHASTIC = 1

(QN_OK, QN_ERR_INVALID, QN_ERR_ALLOC, QN_ERR_CUDA, QN_ERR_STATE, QN_ERR_NOT_CONVERGED, QN_ERR_NONFINITE,
 QN_ERR_DEVICE_TIMEOUT) = range(8)

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libqn.so")
_lib: Optional[ctypes.CDLL] = None

EXPORTS = (
    "qn_strerror", "qn_create", "qn_destroy", "qn_update", "qn_gram", "qn_update_from_gram", "qn_apply_hinv",
    "qn_set_rank_cap", "qn_set_sweep_limit", "qn_set_gram_path", "qn_set_tau_cap", "qn_last_tau", "qn_push",
    "qn_update_window", "qn_rebuild",
    "qn_window_alloc", "qn_window_theta", "qn_window_g", "qn_window_mark_full", "qn_update_host", "qn_status_sync",
    "qn_last_launches", "qn_total_launches", "qn_last_sweeps", "qn_last_gram_kernel", "qn_precision_flag",
    "qn_timing_begin",
    "qn_timing_end",
    "qn_gram_static", "qn_selftest_bounded_wait",
    "qn_logprobs", "qn_logprobs_backward", "qn_distill", "qn_policy", "qn_preference",
    "qn_adam_create", "qn_adam_destroy", "qn_adam_grads", "qn_adam_norm", "qn_adam_step", "qn_adam_places", "qn_adam_state",
    "qn_selftest_roots",
)
TIME_KINDS = ("gram", "solve", "combine", "row")
KERNEL_NAMES = {
    0: "none",
    1: "direct (m <= 8, register-fed, plain ALUs)",
    2: "bulk-copy (m <= 8, shared-memory stages, packed fp32 ALUs, fp64 flush)",
    3: "tiled (plain ALUs)",
    4: "tcgen05 (bf16 hi/lo split, fp32 accumulation in short chains, fp64 flush)",
    5: "row refresh, register-fed",
    6: "row refresh, bulk-copy (fp32 sums per work item, fp64 across)",
}


class QNError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (status %d)" % (where, qn_strerror(status), status))


def lib() -> ctypes.CDLL:
    """Load libqn.so (built by ``paper_1709_05069_b200.build``).  Raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise FileNotFoundError(
                "%s not found: build it with `python -m paper_1709_05069_b200.build` (there is no CPU fallback)" % _LIB_PATH)
        L = ctypes.CDLL(_LIB_PATH)
        vp, i32, i64, dbl = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double
        L.qn_strerror.argtypes, L.qn_strerror.restype = [i32], ctypes.c_char_p
        L.qn_create.argtypes, L.qn_create.restype = [i64, i32, i32, ctypes.POINTER(vp)], i32
        L.qn_destroy.argtypes, L.qn_destroy.restype = [vp], i32
        L.qn_update.argtypes, L.qn_update.restype = [vp, vp, vp, dbl, dbl, vp, vp, vp, vp], i32
        L.qn_gram.argtypes, L.qn_gram.restype = [vp, vp, vp, vp], i32
        L.qn_selftest_bounded_wait.argtypes, L.qn_selftest_bounded_wait.restype = [vp, vp], i32
        L.qn_set_tau_cap.argtypes, L.qn_set_tau_cap.restype = [vp, i32], i32
        L.qn_last_tau.argtypes, L.qn_last_tau.restype = [vp], dbl
        L.qn_set_rank_cap.argtypes, L.qn_set_rank_cap.restype = [vp, i32], i32
        L.qn_set_sweep_limit.argtypes, L.qn_set_sweep_limit.restype = [vp, i32], i32
        L.qn_set_gram_path.argtypes, L.qn_set_gram_path.restype = [vp, i32], i32
        L.qn_apply_hinv.argtypes, L.qn_apply_hinv.restype = [vp, vp, vp, dbl, vp, vp, vp, vp, vp], i32
        L.qn_update_from_gram.argtypes, L.qn_update_from_gram.restype = [vp, vp, vp, vp, dbl, dbl, vp, vp, vp, vp], i32
        L.qn_push.argtypes, L.qn_push.restype = [vp, i32, vp, vp, vp], i32
        L.qn_update_window.argtypes, L.qn_update_window.restype = [vp, dbl, dbl, vp, vp, vp, vp], i32
        L.qn_rebuild.argtypes, L.qn_rebuild.restype = [vp, vp], i32
        L.qn_window_alloc.argtypes, L.qn_window_alloc.restype = [vp], i32
        L.qn_window_theta.argtypes, L.qn_window_theta.restype = [vp], vp
        L.qn_window_g.argtypes, L.qn_window_g.restype = [vp], vp
        L.qn_window_mark_full.argtypes, L.qn_window_mark_full.restype = [vp], i32
        L.qn_update_host.argtypes, L.qn_update_host.restype = [vp, vp, vp, dbl, dbl, vp, vp, vp, vp], i32
        L.qn_status_sync.argtypes, L.qn_status_sync.restype = [vp], i32
        L.qn_last_launches.argtypes, L.qn_last_launches.restype = [vp], i32
        L.qn_total_launches.argtypes, L.qn_total_launches.restype = [vp], i64
        L.qn_last_sweeps.argtypes, L.qn_last_sweeps.restype = [vp], i32
        L.qn_last_gram_kernel.argtypes, L.qn_last_gram_kernel.restype = [vp], i32
        L.qn_precision_flag.argtypes, L.qn_precision_flag.restype = [vp], i32
        L.qn_gram_static.argtypes, L.qn_gram_static.restype = [i64, i32, i32, vp, vp, vp], i32
        L.qn_timing_begin.argtypes, L.qn_timing_begin.restype = [vp, i32], i32
        L.qn_timing_end.argtypes, L.qn_timing_end.restype = [vp, vp, vp], i32
        L.qn_logprobs.argtypes = [i64, i64, i32, vp, i64, vp, dbl, vp, vp, vp, i32, vp, vp, vp]
        L.qn_logprobs_backward.argtypes = [i64, i64, i32, vp, i64, vp, dbl, vp, vp, vp, i32, vp, vp, vp, i64, vp]
        L.qn_distill.argtypes = [i64, i64, i32, vp, i64, i32, vp, i32, vp, i32, dbl, vp, vp, vp, i64, vp]
        L.qn_logprobs.restype = L.qn_logprobs_backward.restype = L.qn_distill.restype = i32
        L.qn_policy.argtypes = [i64, i64, i32, vp, i64, vp, dbl, vp, vp, vp, vp, dbl, dbl, dbl, dbl, dbl, vp, vp, vp, vp, i64, vp]
        L.qn_preference.argtypes = [i64, i64, vp, i32, vp, vp, vp, i32, vp, i32, dbl, dbl, dbl, i32, vp, vp, vp, vp]
        L.qn_policy.restype = L.qn_preference.restype = i32
        L.qn_adam_create.argtypes = [i32, vp, i32, i32, i32, ctypes.POINTER(vp)]
        L.qn_adam_destroy.argtypes = [vp]
        L.qn_adam_grads.argtypes = [vp, vp, vp]
        L.qn_adam_norm.argtypes = [vp, vp, vp]
        L.qn_adam_step.argtypes = [vp, vp, dbl, vp, dbl, dbl, dbl, vp, dbl, dbl, i32, ctypes.c_uint64, vp]
        L.qn_adam_state.argtypes = [vp, i32, vp, vp, vp]
        for name in ("create", "destroy", "grads", "norm", "step", "state"):
            getattr(L, "qn_adam_" + name).restype = i32
        L.qn_adam_places.argtypes, L.qn_adam_places.restype = [vp], i64
        L.qn_selftest_roots.argtypes, L.qn_selftest_roots.restype = [i64, i64, vp, vp], i32
        _lib = L
    return _lib


def qn_strerror(status: int) -> str:
    return lib().qn_strerror(int(status)).decode()


def _check(status: int, where: str, allow=()) -> int:
    if status != QN_OK and status not in allow:
        raise QNError(status, where)
    return status


def dtype_code(dtype: torch.dtype) -> int:
    if dtype == torch.float32:
        return QN_F32
    if dtype == torch.bfloat16:
        return QN_BF16
    raise TypeError("storage dtype must be torch.float32 or torch.bfloat16")


class Handle:
    """Owner of a ``qn_handle``.  ``n``, ``m``, ``dtype`` as passed to ``qn_create``; ``device`` is the index of
    the CUDA device the handle lives on (every tensor passed with it must live there too)."""

    def __init__(self, ptr: int, n: int, m: int, dtype: torch.dtype, device: int = 0):
        self.ptr, self.n, self.m, self.dtype, self.device = ptr, n, m, dtype, device
        self.gram_path = QN_GRAM_PATH_AUTO  # as last set through qn_set_gram_path

    def close(self):
        if self.ptr:
            lib().qn_destroy(self.ptr)
            self.ptr = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    @property
    def last_launches(self) -> int:
        return lib().qn_last_launches(self.ptr)

    @property
    def total_launches(self) -> int:
        return lib().qn_total_launches(self.ptr)

    @property
    def last_sweeps(self) -> int:
        return lib().qn_last_sweeps(self.ptr)

    @property
    def last_gram_kernel(self) -> str:
        """Name of the kernel the most recent Gram pass (or row refresh) was dispatched to."""
        code = lib().qn_last_gram_kernel(self.ptr)
        name = KERNEL_NAMES.get(code & 0xff, "unknown")
        return name + (", fp64 products and sums" if code & 0x100 else "")


def _stream_ptr(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def _same_device(t, h: Handle, name: str) -> None:
    # a tensor on another GPU would make the kernels dereference memory they cannot reach
    if t.device.index != h.device:
        raise ValueError("%s lives on cuda:%s but the handle was created on cuda:%d" % (name, t.device.index, h.device))


def _dev_matrix(t: torch.Tensor, h: Handle, name: str) -> int:
    if not t.is_cuda or t.dtype != h.dtype or tuple(t.shape) != (h.m, h.n) or not t.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA tensor [m][n] of the handle's dtype" % name)
    _same_device(t, h, name)
    return t.data_ptr()


def _dev_vector(t: torch.Tensor, h: Handle, name: str) -> int:
    if not t.is_cuda or t.dtype != h.dtype or tuple(t.shape) != (h.n,) or not t.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA tensor [n] of the handle's dtype" % name)
    _same_device(t, h, name)
    return t.data_ptr()


def qn_create(n: int, m: int, dtype: torch.dtype) -> Handle:
    """Handle on the current CUDA device (``torch.cuda.current_device()``)."""
    out = ctypes.c_void_p(0)
    device = 0
    if torch.cuda.is_available():
        device = torch.cuda.current_device()
        torch.cuda.set_device(device)  # make torch's device the runtime's current one
    _check(lib().qn_create(int(n), int(m), dtype_code(dtype), ctypes.byref(out)), "qn_create")
    return Handle(out.value, int(n), int(m), dtype, device)


def qn_destroy(h: Handle) -> None:
    h.close()


def _host_outputs(h: Handle, want: bool):
    if not want:
        return None, None, None, None
    j = ctypes.c_int32(0)
    sigma = (ctypes.c_double * h.m)()
    return j, sigma, ctypes.byref(j), ctypes.cast(sigma, ctypes.c_void_p)


def qn_update(h: Handle, theta: torch.Tensor, g: torch.Tensor, tau: float, lam: float, theta_new: torch.Tensor,
              want_host: bool = True, stream=None, allow=(QN_ERR_NOT_CONVERGED, QN_ERR_NONFINITE)):
    """One Server step on device tensors.  Returns (j, sigma list, status) or None when ``want_host`` is False
    (then nothing waits for the device)."""
    j, sigma, jp, sp = _host_outputs(h, want_host)
    st = lib().qn_update(h.ptr, _dev_matrix(theta, h, "theta"), _dev_matrix(g, h, "g"), float(tau), float(lam),
                         _dev_vector(theta_new, h, "theta_new"), jp, sp, _stream_ptr(stream))
    _check(st, "qn_update", allow)
    if want_host:
        return j.value, list(sigma), st
    return None


def qn_gram(h: Handle, g: torch.Tensor, gram_out: torch.Tensor, stream=None) -> None:
    """Centred Gram (m*m) followed by w = G^T gbar (m) into ``gram_out`` (CUDA float64, m*m + m)."""
    _check_gram_buffer(h, gram_out)
    _check(lib().qn_gram(h.ptr, _dev_matrix(g, h, "g"), gram_out.data_ptr(), _stream_ptr(stream)), "qn_gram")


def qn_set_rank_cap(h: Handle, j_cap: Optional[int]) -> None:
    """Keep at most ``j_cap`` modes in later steps on this handle (``None`` or a negative value: no cap)."""
    _check(lib().qn_set_rank_cap(h.ptr, -1 if j_cap is None else int(j_cap)), "qn_set_rank_cap")


def qn_set_sweep_limit(h: Handle, max_sweeps: Optional[int]) -> None:
    """Limit the fp64 Jacobi sweeps of later steps on this handle (``None`` or 0: the built-in limit of 30).  A step
    that reaches the limit still writes its outputs and reports QN_ERR_NOT_CONVERGED."""
    _check(lib().qn_set_sweep_limit(h.ptr, 0 if max_sweeps is None else int(max_sweeps)), "qn_set_sweep_limit")


def qn_set_gram_path(h: Handle, path: int) -> None:
    """``QN_GRAM_PATH_AUTO`` (default), ``QN_GRAM_PATH_PLAIN_ALU`` (register-fed plain-ALU Gram kernels only) or
    ``QN_GRAM_PATH_FP64`` (those kernels with fp64 products and sums whatever n)."""
    _check(lib().qn_set_gram_path(h.ptr, int(path)), "qn_set_gram_path")
    h.gram_path = int(path)


def qn_set_tau_cap(h: Handle, on: bool) -> None:
    """Bound tau by the reciprocal of the method's estimate of the Hessian's largest singular value in later
    ``qn_update`` / ``qn_update_host`` calls on this handle (one more pass, over theta)."""
    _check(lib().qn_set_tau_cap(h.ptr, 1 if on else 0), "qn_set_tau_cap")


def qn_last_tau(h: Handle) -> float:
    """Learning rate used by the most recent step whose results were fetched to the host."""
    return float(lib().qn_last_tau(h.ptr))


def qn_apply_hinv(h: Handle, theta: torch.Tensor, g: torch.Tensor, lam: float, z: torch.Tensor, out: torch.Tensor,
                  want_host: bool = True, stream=None, allow=(QN_ERR_NOT_CONVERGED, QN_ERR_NONFINITE)):
    """``out = Hbar^{-1} z`` (Eq. (3)/(4)) for an arbitrary device vector ``z``.  Returns like ``qn_update``."""
    j, sigma, jp, sp = _host_outputs(h, want_host)
    st = lib().qn_apply_hinv(h.ptr, _dev_matrix(theta, h, "theta"), _dev_matrix(g, h, "g"), float(lam),
                             _dev_vector(z, h, "z"), _dev_vector(out, h, "out"), jp, sp, _stream_ptr(stream))
    _check(st, "qn_apply_hinv", allow)
    if want_host:
        return j.value, list(sigma), st
    return None


def _check_gram_buffer(h: Handle, gram: torch.Tensor) -> None:
    if not gram.is_cuda or gram.dtype != torch.float64 or gram.numel() != h.m * h.m + h.m or not gram.is_contiguous():
        raise ValueError("the Gram buffer must be a contiguous CUDA float64 tensor with m*m + m elements")
    _same_device(gram, h, "the Gram buffer")


def qn_update_from_gram(h: Handle, theta: torch.Tensor, g: torch.Tensor, gram: torch.Tensor, tau: float, lam: float,
                        theta_new: torch.Tensor, want_host: bool = True, stream=None,
                        allow=(QN_ERR_NOT_CONVERGED, QN_ERR_NONFINITE)):
    """The step without its Gram pass: ``gram`` is what ``qn_gram`` wrote, or the sum of such buffers over the
    column slices of an n-sharded problem.  Returns like ``qn_update``."""
    _check_gram_buffer(h, gram)
    j, sigma, jp, sp = _host_outputs(h, want_host)
    st = lib().qn_update_from_gram(h.ptr, _dev_matrix(theta, h, "theta"), _dev_matrix(g, h, "g"), gram.data_ptr(),
                                   float(tau), float(lam), _dev_vector(theta_new, h, "theta_new"), jp, sp,
                                   _stream_ptr(stream))
    _check(st, "qn_update_from_gram", allow)
    if want_host:
        return j.value, list(sigma), st
    return None


def shard_columns(n: int, world: int, rank: int, align: int = 8):
    """Column range [begin, end) of ``rank`` when n columns are split over ``world`` ranks in contiguous slices whose
    boundaries are multiples of ``align`` (so that every slice keeps 16-byte aligned rows).  Host logic only."""
    if world < 1 or not 0 <= rank < world or n < 0 or align < 1:
        raise ValueError("bad shard request")
    blocks = (n + align - 1) // align
    b0 = blocks * rank // world
    b1 = blocks * (rank + 1) // world
    return min(b0 * align, n), min(b1 * align, n)


def qn_update_sharded(h: Handle, theta: torch.Tensor, g: torch.Tensor, tau: float, lam: float, theta_new: torch.Tensor,
                      gram_buf: torch.Tensor, group=None, want_host: bool = True, stream=None):
    """One Server step on this rank's column slice of an n-sharded problem (one process per GPU).

    ``theta``, ``g``: [m][n_local] of this rank; ``gram_buf``: CUDA float64 scratch with m*m + m elements.  The only
    exchange is one all-reduce of ``gram_buf`` (``torch.distributed``, NCCL between GPUs); every other byte stays on
    its GPU.  With no initialised process group this is ``qn_gram`` + ``qn_update_from_gram``; with a group of one
    rank the all-reduce still runs (it is the identity).

    The collective is ordered against torch's CURRENT stream, so the three calls run with ``stream`` made current:
    the all-reduce then sits between the Gram pass and the step on the same stream.

    With ``want_host`` the step's precision flag is read as well (``qn_precision_flag``): if the spectrum has a
    retained mode too small for the reduced-precision Gram pass, the three calls are repeated once with the handle on
    ``QN_GRAM_PATH_FP64``.  sigma and j are identical on every rank, so all ranks repeat together.  Without
    ``want_host`` nothing is read back and nothing is repeated."""
    import torch.distributed as dist

    if stream is None:
        stream = torch.cuda.current_stream()

    def three_calls():
        qn_gram(h, g, gram_buf, stream=stream)
        if dist.is_available() and dist.is_initialized():
            dist.all_reduce(gram_buf, op=dist.ReduceOp.SUM, group=group)
        return qn_update_from_gram(h, theta, g, gram_buf, tau, lam, theta_new, want_host=want_host, stream=stream)

    with torch.cuda.stream(stream):
        res = three_calls()
        if want_host and lib().qn_precision_flag(h.ptr):
            before = h.gram_path
            qn_set_gram_path(h, QN_GRAM_PATH_FP64)
            try:
                res = three_calls()
            finally:
                qn_set_gram_path(h, before)
        return res


def qn_push(h: Handle, slot: int, theta_col: torch.Tensor, g_col: torch.Tensor, stream=None) -> None:
    _check(lib().qn_push(h.ptr, int(slot), _dev_vector(theta_col, h, "theta_col"), _dev_vector(g_col, h, "g_col"),
                         _stream_ptr(stream)), "qn_push")


def qn_update_window(h: Handle, tau: float, lam: float, theta_new: torch.Tensor, want_host: bool = True, stream=None,
                     allow=(QN_ERR_NOT_CONVERGED, QN_ERR_NONFINITE)):
    j, sigma, jp, sp = _host_outputs(h, want_host)
    st = lib().qn_update_window(h.ptr, float(tau), float(lam), _dev_vector(theta_new, h, "theta_new"), jp, sp,
                                _stream_ptr(stream))
    _check(st, "qn_update_window", allow)
    if want_host:
        return j.value, list(sigma), st
    return None


def qn_rebuild(h: Handle, stream=None) -> None:
    _check(lib().qn_rebuild(h.ptr, _stream_ptr(stream)), "qn_rebuild")


def qn_window_alloc(h: Handle) -> None:
    _check(lib().qn_window_alloc(h.ptr), "qn_window_alloc")


def qn_window_ptrs(h: Handle) -> Tuple[int, int]:
    return lib().qn_window_theta(h.ptr) or 0, lib().qn_window_g(h.ptr) or 0


def qn_window_mark_full(h: Handle) -> None:
    _check(lib().qn_window_mark_full(h.ptr), "qn_window_mark_full")


def qn_update_host(h: Handle, theta_host: torch.Tensor, g_host: torch.Tensor, tau: float, lam: float,
                   theta_new_host: torch.Tensor, stream=None, allow=(QN_ERR_NOT_CONVERGED, QN_ERR_NONFINITE)):
    """The step with HOST tensors (pinned recommended): copies in, computes, copies theta_new out, waits."""
    for t, shape, name in ((theta_host, (h.m, h.n), "theta_host"), (g_host, (h.m, h.n), "g_host"),
                           (theta_new_host, (h.n,), "theta_new_host")):
        if t.is_cuda or t.dtype != h.dtype or tuple(t.shape) != shape or not t.is_contiguous():
            raise ValueError("%s must be a contiguous host tensor of shape %s and the handle's dtype" % (name, shape))
    j, sigma, jp, sp = _host_outputs(h, True)
    st = lib().qn_update_host(h.ptr, theta_host.data_ptr(), g_host.data_ptr(), float(tau), float(lam),
                              theta_new_host.data_ptr(), jp, sp, _stream_ptr(stream))
    _check(st, "qn_update_host", allow)
    return j.value, list(sigma), st


def qn_selftest_bounded_wait(h: Handle, stream=None) -> None:
    """Enqueue the bounded-wait self-test: the next step on ``h`` reports QN_ERR_DEVICE_TIMEOUT."""
    _check(lib().qn_selftest_bounded_wait(h.ptr, _stream_ptr(stream)), "qn_selftest_bounded_wait")


def qn_status_sync(h: Handle) -> int:
    return lib().qn_status_sync(h.ptr)


def qn_timing_begin(h: Handle, max_kernels: int) -> None:
    _check(lib().qn_timing_begin(h.ptr, int(max_kernels)), "qn_timing_begin")


def qn_timing_end(h: Handle):
    """{kind: (total_ms, launches)} for the kernels launched since ``qn_timing_begin``."""
    ms = (ctypes.c_double * len(TIME_KINDS))()
    cnt = (ctypes.c_int32 * len(TIME_KINDS))()
    _check(lib().qn_timing_end(h.ptr, ctypes.cast(ms, ctypes.c_void_p), ctypes.cast(cnt, ctypes.c_void_p)),
           "qn_timing_end")
    return {k: (ms[i], cnt[i]) for i, k in enumerate(TIME_KINDS)}


QN_STATIC_MAX_M = 32


def qn_gram_static(g: torch.Tensor, gram_out: torch.Tensor, stream=None) -> None:
    """``qn_gram`` for callers that must not allocate: no handle, scratch in a fixed array inside the library.

    ``g`` is a contiguous CUDA tensor [m][n] (float32 or bfloat16, m <= 32), ``gram_out`` a CUDA float64
    tensor with m*m + m elements.  Calls on one device share the scratch: do not let two overlap."""
    if not g.is_cuda or g.dim() != 2 or not g.is_contiguous():
        raise ValueError("g must be a contiguous CUDA tensor [m][n]")
    m, n = g.shape
    if not gram_out.is_cuda or gram_out.dtype != torch.float64 or gram_out.numel() != m * m + m \
            or not gram_out.is_contiguous():
        raise ValueError("gram_out must be a contiguous CUDA float64 tensor with m*m + m elements")
    if gram_out.device != g.device:
        raise ValueError("g and gram_out must live on the same device")
    # the call runs on the runtime's current device: make that the tensors' device for its duration
    with torch.cuda.device(g.device):
        _check(lib().qn_gram_static(int(n), int(m), dtype_code(g.dtype), g.data_ptr(), gram_out.data_ptr(),
                                    _stream_ptr(stream)), "qn_gram_static")


# ---- losses over a vocabulary (no handle) ---------------------------------------------------------------------------


def _logit_matrix(t: torch.Tensor, name: str) -> Tuple[int, int, int, int]:
    """rows, vocab, row stride, dtype code of a matrix of logits (or their gradient)."""
    if not t.is_cuda or t.dim() != 2:
        raise ValueError("%s must be a CUDA tensor [rows][vocab]" % name)
    rows, vocab = t.shape
    stride, inner = t.stride()
    if rows <= 1 and stride < vocab:
        stride = vocab
    if vocab < 1 or (inner != 1 and vocab != 1) or stride < vocab:
        raise ValueError("%s must have contiguous rows that do not overlap" % name)
    return rows, vocab, stride, dtype_code(t.dtype)


def _beside(t: Optional[torch.Tensor], dtype: torch.dtype, rows: int, width: int, device: int, name: str) -> int:
    """Address of a small array that goes with the logits, [rows] (width 0) or [rows][width]; 0 for None."""
    if t is None:
        return 0
    # what the calls cost beside their kernels is mostly these checks: few and cheap ones
    if t.dtype is dtype and t.get_device() == device and t.is_contiguous():
        if width == 0:
            if t.dim() == 1 and t.numel() == rows:
                return t.data_ptr()
        elif t.dim() == 2 and t.shape[1] == width and t.numel() == rows * width:
            return t.data_ptr()
    raise ValueError("%s must be a contiguous %s tensor of shape %s on cuda:%d"
                     % (name, dtype, [rows, width] if width else [rows], device))


def _gradient(t: torch.Tensor, logits: torch.Tensor, name: str) -> Tuple[int, int]:
    """Address and row stride of the gradient of ``logits``."""
    if t.shape != logits.shape or t.dtype is not logits.dtype or t.get_device() != logits.get_device():
        raise ValueError("%s must have the shape, dtype and device of the logits" % name)
    return t.data_ptr(), _logit_matrix(t, name)[2]


# torch's current stream by device index without a Stream object around it (2 us a call); the public way otherwise
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_on(device: int, stream) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    return _raw_stream(device) if _raw_stream is not None else int(torch.cuda.current_stream(device).cuda_stream)


def qn_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, logprob: Optional[torch.Tensor] = None,
                lse: Optional[torch.Tensor] = None, entropy: Optional[torch.Tensor] = None,
                top_token: Optional[torch.Tensor] = None, top_logprob: Optional[torch.Tensor] = None,
                temperature: float = 1.0, stream=None) -> None:
    """Log probability of one given token in each row of ``logits`` [rows][vocab], with lse, entropy and the ``k``
    largest alternatives (k: the width of ``top_token``), in one launch.

    Outputs are the tensors that are passed: ``logprob``, ``lse``, ``entropy`` float32 [rows], ``top_token`` int64 and
    ``top_logprob`` float32 [rows][k]; ``tokens`` is int64 [rows], negative for "none".  Nothing waits for the device."""
    rows, vocab, stride, code = _logit_matrix(logits, "logits")
    dev, k = logits.get_device(), 0
    if top_token is not None or top_logprob is not None:
        if top_token is None or top_logprob is None or top_token.dim() != 2 or top_token.shape != top_logprob.shape:
            raise ValueError("top_token and top_logprob go together, [rows][k] each")
        k = top_token.shape[1]
    f32 = torch.float32
    _check(lib().qn_logprobs(rows, vocab, code, logits.data_ptr(), stride,
                             _beside(tokens, torch.int64, rows, 0, dev, "tokens"), temperature,
                             _beside(logprob, f32, rows, 0, dev, "logprob"), _beside(lse, f32, rows, 0, dev, "lse"),
                             _beside(entropy, f32, rows, 0, dev, "entropy"), k,
                             _beside(top_token, torch.int64, rows, k, dev, "top_token") if k else 0,
                             _beside(top_logprob, f32, rows, k, dev, "top_logprob") if k else 0, _stream_on(dev, stream)),
           "qn_logprobs")


def qn_logprobs_backward(logits: torch.Tensor, dlogits: torch.Tensor, tokens: Optional[torch.Tensor] = None,
                         d_logprob: Optional[torch.Tensor] = None, d_lse: Optional[torch.Tensor] = None,
                         d_entropy: Optional[torch.Tensor] = None, top_token: Optional[torch.Tensor] = None,
                         d_top_logprob: Optional[torch.Tensor] = None, temperature: float = 1.0, stream=None) -> None:
    """Gradient with respect to the logits, into ``dlogits`` (which may be ``logits`` itself), of a loss whose upstream
    gradients with respect to ``qn_logprobs``' outputs are ``d_logprob``, ``d_lse``, ``d_entropy`` [rows] and
    ``d_top_logprob`` [rows][k] (with the ``top_token`` that the forward call wrote), in one launch."""
    rows, vocab, stride, code = _logit_matrix(logits, "logits")
    dev, k = logits.get_device(), 0
    if d_top_logprob is not None:
        if top_token is None or d_top_logprob.dim() != 2:
            raise ValueError("d_top_logprob [rows][k] goes with top_token")
        k = d_top_logprob.shape[1]
    f32 = torch.float32
    out, out_stride = _gradient(dlogits, logits, "dlogits")
    _check(lib().qn_logprobs_backward(rows, vocab, code, logits.data_ptr(), stride,
                                      _beside(tokens, torch.int64, rows, 0, dev, "tokens"), temperature,
                                      _beside(d_logprob, f32, rows, 0, dev, "d_logprob"),
                                      _beside(d_lse, f32, rows, 0, dev, "d_lse"),
                                      _beside(d_entropy, f32, rows, 0, dev, "d_entropy"), k,
                                      _beside(top_token, torch.int64, rows, k, dev, "top_token") if k else 0,
                                      _beside(d_top_logprob, f32, rows, k, dev, "d_top_logprob") if k else 0, out,
                                      out_stride, _stream_on(dev, stream)), "qn_logprobs_backward")


def qn_distill(logits: torch.Tensor, teacher_token: torch.Tensor, teacher_value: torch.Tensor, loss: torch.Tensor,
               dlogits: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None, temperature: float = 1.0,
               teacher: int = QN_TEACHER_LOGPROBS, stream=None) -> None:
    """Loss of each row of the student's ``logits`` against a teacher's top tokens (into ``loss`` float32 [rows]) and, if
    ``dlogits`` is given (it may be ``logits`` itself), the gradient of sum(weight * loss), in one launch.

    ``teacher_token`` int64 [rows][k] (negative: absent), ``teacher_value`` float32 or bfloat16 [rows][k]: log
    probabilities as ``qn_logprobs`` writes them (``QN_TEACHER_LOGPROBS``: the rest of the vocabulary is one more outcome)
    or logits (``QN_TEACHER_LOGITS``: normalised over the list).  ``weight`` float32 [rows], 0 for padding."""
    rows, vocab, stride, code = _logit_matrix(logits, "logits")
    dev = logits.get_device()
    if teacher_token is None or teacher_value is None or loss is None or teacher_token.dim() != 2:
        raise ValueError("teacher_token and teacher_value [rows][k] and loss [rows] are required")
    k = teacher_token.shape[1]
    out, out_stride = _gradient(dlogits, logits, "dlogits") if dlogits is not None else (0, 0)
    _check(lib().qn_distill(rows, vocab, code, logits.data_ptr(), stride, k,
                            _beside(teacher_token, torch.int64, rows, k, dev, "teacher_token"),
                            dtype_code(teacher_value.dtype),
                            _beside(teacher_value, teacher_value.dtype, rows, k, dev, "teacher_value"), teacher,
                            temperature, _beside(weight, torch.float32, rows, 0, dev, "weight"),
                            _beside(loss, torch.float32, rows, 0, dev, "loss"), out, out_stride,
                            _stream_on(dev, stream)), "qn_distill")


def qn_policy(logits: torch.Tensor, tokens: torch.Tensor, old_logprob: torch.Tensor, advantage: torch.Tensor,
              loss: torch.Tensor, dlogits: Optional[torch.Tensor] = None, ref_logprob: Optional[torch.Tensor] = None,
              weight: Optional[torch.Tensor] = None, logprob: Optional[torch.Tensor] = None,
              entropy: Optional[torch.Tensor] = None, clip_low: float = 0.2, clip_high: float = 0.2, dual: float = 0.0,
              kl: float = 0.0, entropy_bonus: float = 0.0, temperature: float = 1.0, stream=None) -> None:
    """Clipped policy loss of the given ``tokens`` int64 [rows] (into ``loss`` float32 [rows]) and, if ``dlogits`` is given (it
    may be ``logits`` itself), the gradient of sum(weight * loss), in one launch.

    ``old_logprob``, ``advantage``, ``ref_logprob`` (needed with ``kl`` > 0) and ``weight`` are float32 [rows]; a row whose
    token is negative or whose weight is 0 is padding.  ``logprob`` and ``entropy`` float32 [rows] are written if given."""
    rows, vocab, stride, code = _logit_matrix(logits, "logits")
    dev, f32 = logits.get_device(), torch.float32
    if tokens is None or old_logprob is None or advantage is None or loss is None:
        raise ValueError("tokens, old_logprob, advantage and loss [rows] are required")
    out, out_stride = _gradient(dlogits, logits, "dlogits") if dlogits is not None else (0, 0)
    _check(lib().qn_policy(rows, vocab, code, logits.data_ptr(), stride, _beside(tokens, torch.int64, rows, 0, dev, "tokens"),
                           temperature, _beside(old_logprob, f32, rows, 0, dev, "old_logprob"),
                           _beside(ref_logprob, f32, rows, 0, dev, "ref_logprob"),
                           _beside(advantage, f32, rows, 0, dev, "advantage"), _beside(weight, f32, rows, 0, dev, "weight"),
                           clip_low, clip_high, dual, kl, entropy_bonus, _beside(loss, f32, rows, 0, dev, "loss"),
                           _beside(logprob, f32, rows, 0, dev, "logprob"), _beside(entropy, f32, rows, 0, dev, "entropy"), out,
                           out_stride, _stream_on(dev, stream)), "qn_policy")


def qn_preference(logprob: torch.Tensor, offsets: torch.Tensor, loss: torch.Tensor, d_logprob: Optional[torch.Tensor] = None,
                  ref_logprob: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                  pair_weight: Optional[torch.Tensor] = None, reward: Optional[torch.Tensor] = None,
                  kind: int = QN_PREFERENCE_LOGISTIC, beta: float = 0.1, margin: float = 0.0, smoothing: float = 0.0,
                  normalise: bool = False, split: bool = False, stream=None) -> None:
    """Preference loss of pairs of packed sequences (into ``loss`` float32 [pairs]) and, if ``d_logprob`` is given, the gradient
    of sum(pair_weight * loss) with respect to ``logprob``, in one launch.

    ``logprob`` float32 [tokens], ``ref_logprob`` float32 or bfloat16 [tokens], ``weight`` float32 [tokens] (0: does not count),
    ``offsets`` int64 [2 * pairs + 1]; ``reward`` float32 [2 * pairs] is written if given.  Sequences 2 k and 2 k + 1 are pair
    k's chosen and rejected one, or k and pairs + k with ``split``."""
    if loss is None or not loss.is_cuda or loss.dim() != 1:
        raise ValueError("loss must be a CUDA tensor [pairs]")
    if logprob is None or offsets is None or logprob.dim() != 1:
        raise ValueError("logprob [tokens] and offsets [2 * pairs + 1] are required")
    dev, f32, pairs, tokens = loss.get_device(), torch.float32, loss.numel(), logprob.numel()
    ref_dtype = f32 if ref_logprob is None else ref_logprob.dtype
    _check(lib().qn_preference(pairs, tokens, _beside(logprob, f32, tokens, 0, dev, "logprob"), dtype_code(ref_dtype),
                               _beside(ref_logprob, ref_dtype, tokens, 0, dev, "ref_logprob"),
                               _beside(weight, f32, tokens, 0, dev, "weight"),
                               _beside(offsets, torch.int64, 2 * pairs + 1, 0, dev, "offsets"), bool(split),
                               _beside(pair_weight, f32, pairs, 0, dev, "pair_weight"), kind, beta, margin, smoothing,
                               bool(normalise), _beside(loss, f32, pairs, 0, dev, "loss"),
                               _beside(reward, f32, 2 * pairs, 0, dev, "reward"),
                               _beside(d_logprob, f32, tokens, 0, dev, "d_logprob"), _stream_on(dev, stream)), "qn_preference")


# ---- AdamW over many tensors ------------------------------------------------------------------------------------------


class _AdamTensor(ctypes.Structure):
    _fields_ = [("numel", ctypes.c_int64), ("param", ctypes.c_void_p), ("grad", ctypes.c_void_p),
                ("master", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("weight_decay", ctypes.c_double),
                ("lr_scale", ctypes.c_double)]


class Adam:
    """Owner of a ``qn_adam_handle`` and of references to the tensors whose addresses it holds."""

    def __init__(self, ptr: int, tensors: Sequence, grads: Sequence, sizes: Sequence[int], grad_dtype: torch.dtype, device: int):
        self.ptr, self.tensors, self.grads, self.sizes = ptr, tensors, grads, sizes
        self.grad_dtype, self.device = grad_dtype, device

    def close(self):
        if self.ptr:
            lib().qn_adam_destroy(self.ptr)
            self.ptr = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    @property
    def places(self) -> int:
        """Elements of the vectors that ``qn_adam_state`` writes."""
        return lib().qn_adam_places(self.ptr)


def _of_tensor(t: Optional[torch.Tensor], dtype: torch.dtype, numel: int, device: int, name: str) -> int:
    if t is None:
        return 0
    if t.dtype is not dtype or t.get_device() != device or t.numel() != numel or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of %d elements on cuda:%d" % (name, dtype, numel, device))
    return t.data_ptr()


def _one_each(given, count: int, name: str) -> Sequence:
    if given is None:
        return [None] * count
    if isinstance(given, torch.Tensor) or len(given) != count:
        raise ValueError("%s must be a list with an entry for each of the %d tensors" % (name, count))
    return list(given)


def _number_each(given, count: int, name: str) -> Sequence[float]:
    return [float(given)] * count if isinstance(given, (int, float)) else [float(x) for x in _one_each(given, count, name)]


def qn_adam_create(params: Sequence[torch.Tensor], grads: Sequence[Optional[torch.Tensor]], m: Sequence[torch.Tensor],
                   v: Sequence[torch.Tensor], master: Optional[Sequence[torch.Tensor]] = None,
                   m_scale: Optional[Sequence[torch.Tensor]] = None, v_scale: Optional[Sequence[torch.Tensor]] = None,
                   weight_decay=0.0, lr_scale=1.0) -> Adam:
    """A plan for AdamW steps on ``params`` (float32 or bfloat16), whose gradients are ``grads`` (None: left alone).

    ``m`` and ``v`` are float32, or uint8 with ``m_scale`` and ``v_scale`` (uint8, one for each ``QN_ADAM_BLOCK`` elements)
    for states in 8 bits; all begin as zeros.  ``master``: float32 copies of bfloat16 parameters.  ``weight_decay`` and
    ``lr_scale``: a number, or one for each tensor.  The tensors must stay where they are; the plan keeps them alive."""
    params = list(params)
    count = len(params)
    if not count or not params[0].is_cuda:
        raise ValueError("params must be CUDA tensors, one at least")
    lists = [params] + [_one_each(x, count, name) for x, name in ((grads, "grads"), (m, "m"), (v, "v"), (master, "master"),
                                                                  (m_scale, "m_scale"), (v_scale, "v_scale"))]
    decay, scale = _number_each(weight_decay, count, "weight_decay"), _number_each(lr_scale, count, "lr_scale")
    device, eight = params[0].get_device(), m_scale is not None or v_scale is not None
    grad_dtype = next((g.dtype for g in lists[1] if g is not None), params[0].dtype)
    state = torch.uint8 if eight else torch.float32
    names, sizes = ("params", "grads", "m", "v", "master", "m_scale", "v_scale"), [p.numel() for p in params]
    dtypes = (params[0].dtype, grad_dtype, state, state, torch.float32, torch.uint8, torch.uint8)
    table = (_AdamTensor * count)()
    for i, size in enumerate(sizes):
        blocks = (size + QN_ADAM_BLOCK - 1) // QN_ADAM_BLOCK
        at = [_of_tensor(x[i], dtype, blocks if "scale" in name else size, device, name)
              for x, dtype, name in zip(lists, dtypes, names)]
        table[i] = _AdamTensor(size, at[0], at[1], at[4], at[2], at[3], at[5], at[6], decay[i], scale[i])
    out = ctypes.c_void_p(0)
    with torch.cuda.device(device):
        _check(lib().qn_adam_create(count, ctypes.addressof(table), dtype_code(params[0].dtype), dtype_code(grad_dtype),
                                    QN_STATE_8BIT if eight else QN_STATE_F32, ctypes.byref(out)), "qn_adam_create")
    return Adam(out.value, lists[:1] + lists[2:], lists[1], sizes, grad_dtype, device)


def qn_adam_destroy(h: Adam) -> None:
    h.close()


def qn_adam_grads(h: Adam, grads: Sequence[Optional[torch.Tensor]], stream=None) -> None:
    """Gradients that have moved (None: the tensor has none, and is left alone from now on)."""
    grads = _one_each(grads, len(h.sizes), "grads")
    at = (ctypes.c_void_p * len(grads))(*[_of_tensor(g, h.grad_dtype, size, h.device, "grads") or None
                                          for g, size in zip(grads, h.sizes)])
    _check(lib().qn_adam_grads(h.ptr, ctypes.addressof(at), _stream_on(h.device, stream)), "qn_adam_grads")
    h.grads = grads


def qn_adam_norm(h: Adam, sumsq: torch.Tensor, stream=None) -> None:
    """The sum of the squares of all gradients into ``sumsq`` (float64, one element)."""
    _check(lib().qn_adam_norm(h.ptr, _of_tensor(sumsq, torch.float64, 1, h.device, "sumsq"), _stream_on(h.device, stream)),
           "qn_adam_norm")


def qn_adam_step(h: Adam, step: torch.Tensor, lr=1e-3, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                 sumsq: Optional[torch.Tensor] = None, max_norm: float = 0.0, grad_scale: float = 1.0,
                 stochastic: bool = False, seed: int = 0, stream=None) -> None:
    """One AdamW step on all tensors of the plan, in one launch that waits for nothing.

    ``step`` (int64, one element, on the device): steps so far, counted up.  ``lr``: a number, or a float32 CUDA tensor of one
    element.  ``sumsq``: what ``qn_adam_norm`` wrote; with ``max_norm`` > 0 the gradients are clipped to that norm, and nothing
    changes if it is not finite.  ``stochastic``: bfloat16 parameters without a master copy are rounded by chance."""
    on_device = isinstance(lr, torch.Tensor)
    _check(lib().qn_adam_step(h.ptr, _of_tensor(step, torch.int64, 1, h.device, "step"), 0.0 if on_device else lr,
                              _of_tensor(lr, torch.float32, 1, h.device, "lr") if on_device else 0, beta1, beta2, eps,
                              _of_tensor(sumsq, torch.float64, 1, h.device, "sumsq"), max_norm, grad_scale,
                              QN_ROUND_STOCHASTIC if stochastic else QN_ROUND_NEAREST, seed & 0xFFFFFFFFFFFFFFFF,
                              _stream_on(h.device, stream)), "qn_adam_step")


def qn_adam_state(h: Adam, m: Optional[torch.Tensor], root: Optional[torch.Tensor], stream=None) -> None:
    """What the states stand for: the moving average and the root of that of squares, into vectors of ``h.places`` elements
    (float32 or bfloat16), where tensors follow one another in whole blocks of ``QN_ADAM_BLOCK``."""
    dtype = next((x.dtype for x in (m, root) if x is not None), torch.float32)
    _check(lib().qn_adam_state(h.ptr, dtype_code(dtype), _of_tensor(m, dtype, h.places, h.device, "m"),
                               _of_tensor(root, dtype, h.places, h.device, "root"), _stream_on(h.device, stream)), "qn_adam_state")


def qn_selftest_roots(first: int, last: int, differ: torch.Tensor, stream=None) -> None:
    """Adds to ``differ`` (int64, one element, on the device) how many float32 numbers with the bits ``first`` to ``last`` have a
    root that is not the correctly rounded one in the AdamW step with states in 8 bits (none from 2^-100 to 2^30)."""
    if differ is None or not differ.is_cuda:
        raise ValueError("differ must be a CUDA tensor")
    dev = differ.get_device()
    _check(lib().qn_selftest_roots(first, last, _of_tensor(differ, torch.int64, 1, dev, "differ"), _stream_on(dev, stream)),
           "qn_selftest_roots")
