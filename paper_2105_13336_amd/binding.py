"""Thin ctypes binding of libtensile.so: argument marshalling only.

Function names are those of ``include/tensile.h``.  Device buffers are torch
tensors on the GPU (torch is used for device memory and streams, nothing
else); every step of the computation runs in the library's HIP kernels.  There
is no CPU fallback: if the library is missing, importing fails loudly.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libtensile.so")

TENSILE_OK, TENSILE_E_INVAL, TENSILE_E_RANGE, TENSILE_E_NOMEM, TENSILE_E_HIP, TENSILE_E_CAPACITY = 0, -1, -2, -3, -4, -5

EXPORTS = ["tensile_last_error", "tensile_version", "tensile_tas_load", "tensile_tas_free", "tensile_tas_info",
           "tensile_tas_update_latencies",
           "tensile_tas_base_timeline", "tensile_eval_plans", "tensile_eval_plans_per_job", "tensile_eval_link", "tensile_apply_intervals", "tensile_score_candidates", "tensile_score_recompute",
           "tensile_validate_plans",
           "tensile_greedy_plan", "tensile_eval_plans_static", "tensile_eval_score_plans", "tensile_tuning_set", "tensile_tuning_reset",
           "tensile_ops_create", "tensile_ops_free", "tensile_ckpt_pack", "tensile_ckpt_unpack", "tensile_layer_norm",
           "tensile_layer_norm_backward", "tensile_gelu", "tensile_gelu_backward", "tensile_linear_grad"]


class TensileError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"tensile error {code}: {message}")
        self.code = code


class _TasDesc(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("N", ctypes.c_int32), ("J", ctypes.c_int32),
                ("size_bytes", ctypes.c_void_p), ("alloc_step", ctypes.c_void_p), ("free_step", ctypes.c_void_p),
                ("access_offsets", ctypes.c_void_p), ("access_steps", ctypes.c_void_p), ("job_id", ctypes.c_void_p),
                ("step_ns", ctypes.c_void_p), ("base_bytes", ctypes.c_int64), ("link_bytes_per_us", ctypes.c_int64)]


class _Plans(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("n_intervals", ctypes.c_int64), ("plan_offsets", ctypes.c_void_p),
                ("iv_tensor", ctypes.c_void_p), ("iv_out", ctypes.c_void_p), ("iv_in", ctypes.c_void_p),
                ("iv_kind", ctypes.c_void_p)]


class _GreedyOpts(ctypes.Structure):
    _fields_ = [("max_iters", ctypes.c_int32), ("min_iters", ctypes.c_int32), ("stop_at_budget", ctypes.c_int32),
                ("msr_num", ctypes.c_void_p), ("msr_den", ctypes.c_int64), ("recompute", ctypes.c_int32)]


class _Matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("ld", ctypes.c_int64),
                ("type", ctypes.c_int32)]


class _Ckpt(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("ld_q", ctypes.c_int64), ("ld_scale", ctypes.c_int64)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python paper_2105_13336_amd/build.py` "
                          "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    lib.tensile_last_error.restype = ctypes.c_char_p
    lib.tensile_tas_free.restype = None
    lib.tensile_tas_free.argtypes = [ctypes.c_void_p]
    lib.tensile_tuning_reset.restype = None
    lib.tensile_tuning_set.argtypes = [ctypes.c_char_p, ctypes.c_int]
    lib.tensile_ops_free.restype = None
    lib.tensile_ops_free.argtypes = [ctypes.c_void_p]
    m, c, p, i32 = ctypes.POINTER(_Matrix), ctypes.POINTER(_Ckpt), ctypes.c_void_p, ctypes.c_int32
    lib.tensile_ckpt_pack.argtypes = [p, m, c, p]
    lib.tensile_ckpt_unpack.argtypes = [p, c, m, p]
    lib.tensile_layer_norm.argtypes = [p, m, m, p, p, i32, ctypes.c_double, m, m, c, p, p]
    lib.tensile_layer_norm_backward.argtypes = [p, m, c, p, p, i32, m, m, p, p, p]
    lib.tensile_gelu.argtypes = [p, m, m, c, i32, p]
    lib.tensile_gelu_backward.argtypes = [p, m, c, m, c, i32, p]
    lib.tensile_linear_grad.argtypes = [p, m, c, p, p, i32, m, p, p]
    return lib


_lib = _load()


def _check(rc: int) -> None:
    if rc != TENSILE_OK:
        raise TensileError(rc, _lib.tensile_last_error().decode())


def _np(a, dtype):
    if a is None:
        return None
    return np.ascontiguousarray(a, dtype=dtype)


def _hp(a: Optional[np.ndarray]):
    return None if a is None else ctypes.c_void_p(a.ctypes.data)


def _dp(t: Optional[torch.Tensor], dtype, n: int, name: str):
    if t is None:
        return None
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous() or t.numel() < n:
        raise TensileError(TENSILE_E_INVAL, f"{name}: need a contiguous CUDA tensor of {dtype} with >= {n} elements")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def tensile_version() -> int:
    return _lib.tensile_version()


class TasHandle:
    """Owner of a ``tensile_tas*``; freed on ``close()`` / garbage collection."""

    def __init__(self, ptr: int, T: int, N: int, J: int):
        self._ptr, self.T, self.N, self.J = ptr, T, N, J

    @property
    def ptr(self) -> ctypes.c_void_p:
        if not self._ptr:
            raise TensileError(TENSILE_E_INVAL, "TAS handle already freed")
        return ctypes.c_void_p(self._ptr)

    def close(self) -> None:
        if self._ptr:
            _lib.tensile_tas_free(ctypes.c_void_p(self._ptr))
            self._ptr = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def tensile_tas_load(T, size_bytes, alloc_step, free_step, access_offsets, access_steps, job_id=None, step_ns=None,
                     base_bytes: int = 0, link_bytes_per_us: int = 0, J: int = 1, N: Optional[int] = None) -> TasHandle:
    size = _np(size_bytes, np.int64); alloc = _np(alloc_step, np.int32); free = _np(free_step, np.int32)
    offs = _np(access_offsets, np.int64); acc = _np(access_steps, np.int32)
    job = _np(job_id, np.int32); sn = _np(step_ns, np.int64)
    n = int(size.shape[0]) if N is None else int(N)
    desc = _TasDesc(int(T), n, int(J), _hp(size), _hp(alloc), _hp(free), _hp(offs), _hp(acc), _hp(job), _hp(sn),
                    int(base_bytes), int(link_bytes_per_us))
    out = ctypes.c_void_p()
    _check(_lib.tensile_tas_load(ctypes.byref(desc), ctypes.byref(out)))
    return TasHandle(out.value, int(T), n, int(J))


def tas_load(tas) -> TasHandle:
    """Load from an object with the attributes of the description (e.g. workloads.TAS)."""
    return tensile_tas_load(tas.T, tas.size_bytes, tas.alloc_step, tas.free_step, tas.access_offsets, tas.access_steps,
                            tas.job_id, tas.step_ns, tas.base_bytes, tas.link_bytes_per_us, tas.J)


def tensile_tas_free(h: TasHandle) -> None:
    h.close()


def tensile_tas_update_latencies(h: TasHandle, step_ns, link_bytes_per_us: int = 0) -> None:
    """New operator latencies (HOST array of T values, or None) and link speed for a loaded sequence."""
    sn = None if step_ns is None else np.ascontiguousarray(step_ns, dtype=np.int64)
    if sn is not None and sn.shape[0] != h.T:
        raise TensileError(TENSILE_E_INVAL, "step_ns must have T entries")
    _check(_lib.tensile_tas_update_latencies(h.ptr, _hp(sn), ctypes.c_int64(int(link_bytes_per_us))))


def tensile_tas_info(h: TasHandle):
    peak, arg = ctypes.c_int64(), ctypes.c_int32()
    _check(_lib.tensile_tas_info(h.ptr, ctypes.byref(peak), ctypes.byref(arg)))
    return peak.value, arg.value


def tensile_tas_base_timeline(h: TasHandle) -> np.ndarray:
    out = np.empty(h.T, dtype=np.int64)
    _check(_lib.tensile_tas_base_timeline(h.ptr, _hp(out)))
    return out


class DevicePlans:
    """A batch of plans resident on the GPU (torch tensors), CSR layout of ``tensile_plans``."""

    def __init__(self, plan_offsets: torch.Tensor, iv_tensor: torch.Tensor, iv_out: torch.Tensor, iv_in: torch.Tensor,
                 iv_kind: Optional[torch.Tensor] = None):
        self.B = int(plan_offsets.numel()) - 1
        self.n_intervals = int(iv_tensor.numel())
        self.plan_offsets, self.iv_tensor, self.iv_out, self.iv_in, self.iv_kind = plan_offsets, iv_tensor, iv_out, iv_in, iv_kind

    @classmethod
    def from_numpy(cls, plan_offsets, iv_tensor, iv_out, iv_in, iv_kind=None, device="cuda") -> "DevicePlans":
        up = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a, dtype=dt)).to(device)
        return cls(up(plan_offsets, np.int64), up(iv_tensor, np.int32), up(iv_out, np.int32), up(iv_in, np.int32),
                   None if iv_kind is None else up(iv_kind, np.uint8))

    def struct(self) -> _Plans:
        K = self.n_intervals
        return _Plans(self.B, K, _dp(self.plan_offsets, torch.int64, self.B + 1, "plan_offsets"),
                      _dp(self.iv_tensor, torch.int32, K, "iv_tensor"), _dp(self.iv_out, torch.int32, K, "iv_out"),
                      _dp(self.iv_in, torch.int32, K, "iv_in"), _dp(self.iv_kind, torch.uint8, K, "iv_kind"))


def tensile_eval_plans(h: TasHandle, plans: DevicePlans, resident: Optional[torch.Tensor], peak: torch.Tensor,
                       argmax: torch.Tensor, min_resident: Optional[torch.Tensor] = None, stream=None) -> None:
    B = plans.B
    st = plans.struct()
    _check(_lib.tensile_eval_plans(h.ptr, ctypes.byref(st), _dp(resident, torch.int64, B * h.T, "resident"),
                                   _dp(peak, torch.int64, B, "peak"), _dp(argmax, torch.int32, B, "argmax"),
                                   _dp(min_resident, torch.int64, B, "min_resident"), _stream(stream)))


def tensile_eval_plans_static(h: TasHandle, plans: DevicePlans, resident: Optional[torch.Tensor], peak: torch.Tensor,
                              argmax: torch.Tensor, min_resident: Optional[torch.Tensor] = None, stream=None) -> None:
    """tensile_eval_plans with its scratch in the library's preallocated device array (allocates nothing)."""
    B = plans.B
    st = plans.struct()
    _check(_lib.tensile_eval_plans_static(h.ptr, ctypes.byref(st), _dp(resident, torch.int64, B * h.T, "resident"),
                                          _dp(peak, torch.int64, B, "peak"), _dp(argmax, torch.int32, B, "argmax"),
                                          _dp(min_resident, torch.int64, B, "min_resident"), _stream(stream)))


def tensile_tuning_set(knob: str, value: int) -> None:
    _check(_lib.tensile_tuning_set(knob.encode(), ctypes.c_int(int(value))))


def tensile_tuning_reset() -> None:
    _lib.tensile_tuning_reset()


def tensile_eval_plans_per_job(h: TasHandle, plans: DevicePlans, job_peak: torch.Tensor,
                               job_argmax: Optional[torch.Tensor] = None, sum_peak: Optional[torch.Tensor] = None,
                               stream=None) -> None:
    """job_peak / job_argmax: [J, B] (job-major), sum_peak: [B]"""
    B, J = plans.B, h.J
    st = plans.struct()
    _check(_lib.tensile_eval_plans_per_job(h.ptr, ctypes.byref(st), _dp(job_peak, torch.int64, J * B, "job_peak"),
                                           _dp(job_argmax, torch.int32, J * B, "job_argmax"),
                                           _dp(sum_peak, torch.int64, B, "sum_peak"), _stream(stream)))


def tensile_apply_intervals(h: TasHandle, tensor: torch.Tensor, out_step: torch.Tensor, in_step: torch.Tensor,
                            resident: torch.Tensor, peak: torch.Tensor, argmax: torch.Tensor,
                            min_resident: Optional[torch.Tensor] = None, stream=None) -> None:
    """tensor / out_step / in_step: [B] int32 (one new interval per plan), resident: [B, T] int64 in/out"""
    B = int(tensor.numel())
    _check(_lib.tensile_apply_intervals(h.ptr, ctypes.c_int32(B), _dp(tensor, torch.int32, B, "tensor"),
                                        _dp(out_step, torch.int32, B, "out_step"), _dp(in_step, torch.int32, B, "in_step"),
                                        _dp(resident, torch.int64, B * h.T, "resident"), _dp(peak, torch.int64, B, "peak"),
                                        _dp(argmax, torch.int32, B, "argmax"), _dp(min_resident, torch.int64, B, "min_resident"),
                                        _stream(stream)))


def tensile_eval_link(h: TasHandle, plans: DevicePlans, link_peak: torch.Tensor, link: Optional[torch.Tensor] = None,
                      link_argmax: Optional[torch.Tensor] = None, overbooked: Optional[torch.Tensor] = None,
                      reuse_host_copies: bool = False, stream=None) -> None:
    """link: [B, T] int32, link_peak / link_argmax / overbooked: [B] int32"""
    B = plans.B
    st = plans.struct()
    _check(_lib.tensile_eval_link(h.ptr, ctypes.byref(st), ctypes.c_int32(1 if reuse_host_copies else 0),
                                  _dp(link, torch.int32, B * h.T, "link"), _dp(link_peak, torch.int32, B, "link_peak"),
                                  _dp(link_argmax, torch.int32, B, "link_argmax"), _dp(overbooked, torch.int32, B, "overbooked"),
                                  _stream(stream)))


def tensile_score_candidates(h: TasHandle, plans: DevicePlans, resident: torch.Tensor, peak: torch.Tensor,
                             argmax: torch.Tensor, score: torch.Tensor, win_out: Optional[torch.Tensor] = None,
                             win_in: Optional[torch.Tensor] = None, stream=None) -> None:
    B, N = plans.B, h.N
    st = plans.struct()
    _check(_lib.tensile_score_candidates(h.ptr, ctypes.byref(st), _dp(resident, torch.int64, B * h.T, "resident"),
                                         _dp(peak, torch.int64, B, "peak"), _dp(argmax, torch.int32, B, "argmax"),
                                         _dp(score, torch.int64, B * N, "score"), _dp(win_out, torch.int32, B * N, "win_out"),
                                         _dp(win_in, torch.int32, B * N, "win_in"), _stream(stream)))


def tensile_eval_score_plans(h: TasHandle, plans: DevicePlans, resident: torch.Tensor, peak: torch.Tensor, argmax: torch.Tensor,
                             min_resident: Optional[torch.Tensor], score: torch.Tensor, win_out: Optional[torch.Tensor] = None,
                             win_in: Optional[torch.Tensor] = None, stream=None) -> None:
    """tensile_eval_plans followed by tensile_score_candidates on the same batch, in one call (one kernel when possible)."""
    B, N = plans.B, h.N
    st = plans.struct()
    _check(_lib.tensile_eval_score_plans(h.ptr, ctypes.byref(st), _dp(resident, torch.int64, B * h.T, "resident"),
                                         _dp(peak, torch.int64, B, "peak"), _dp(argmax, torch.int32, B, "argmax"),
                                         _dp(min_resident, torch.int64, B, "min_resident"),
                                         _dp(score, torch.int64, B * N, "score"), _dp(win_out, torch.int32, B * N, "win_out"),
                                         _dp(win_in, torch.int32, B * N, "win_in"), _stream(stream)))


def tensile_score_recompute(h: TasHandle, plans: DevicePlans, resident: torch.Tensor, peak: torch.Tensor,
                             argmax: torch.Tensor, score: torch.Tensor, win_out: Optional[torch.Tensor] = None,
                             win_in: Optional[torch.Tensor] = None, stream=None) -> None:
    B, N = plans.B, h.N
    st = plans.struct()
    _check(_lib.tensile_score_recompute(h.ptr, ctypes.byref(st), _dp(resident, torch.int64, B * h.T, "resident"),
                                         _dp(peak, torch.int64, B, "peak"), _dp(argmax, torch.int32, B, "argmax"),
                                         _dp(score, torch.int64, B * N, "score"), _dp(win_out, torch.int32, B * N, "win_out"),
                                         _dp(win_in, torch.int32, B * N, "win_in"), _stream(stream)))


def tensile_validate_plans(h: TasHandle, plans: DevicePlans):
    """-> (index of the first invalid interval or -1, reason code)"""
    bad, why = ctypes.c_int64(), ctypes.c_int32()
    st = plans.struct()
    _check(_lib.tensile_validate_plans(h.ptr, ctypes.byref(st), ctypes.byref(bad), ctypes.byref(why)))
    return bad.value, why.value


def tensile_greedy_plan(h: TasHandle, budget_bytes: int = 0, max_iters: int = 0, min_iters: int = 100,
                        stop_at_budget: bool = False, msr_num=None, msr_den: int = 1, capacity: Optional[int] = None,
                        initial=None, recompute: bool = False) -> dict:
    """-> dict(iv_tensor, iv_out, iv_in, iv_kind, peak_trace, final_peak, n_initial)"""
    n0 = 0 if initial is None else len(initial[0])
    cap = int(capacity) if capacity is not None else n0 + (max_iters if max_iters > 0 else 1 << 20)
    t = np.zeros(max(cap, 1), dtype=np.int32); o = np.zeros_like(t); r = np.zeros_like(t)
    k = np.zeros(max(cap, 1), dtype=np.uint8)
    if n0:
        t[:n0], o[:n0], r[:n0], k[:n0] = initial
    trace = np.zeros(cap - n0 + 1, dtype=np.int64)
    num = _np(msr_num, np.int64)
    if num is not None and num.shape != (h.J,):
        raise TensileError(TENSILE_E_INVAL, f"msr_num: need one entry per job ({h.J})")
    opts = _GreedyOpts(int(max_iters), int(min_iters), int(bool(stop_at_budget)), _hp(num), int(msr_den), int(bool(recompute)))
    n, fp = ctypes.c_int32(), ctypes.c_int64()
    _check(_lib.tensile_greedy_plan(h.ptr, ctypes.c_int64(int(budget_bytes)), ctypes.byref(opts), ctypes.c_int32(cap),
                                    ctypes.c_int32(n0), _hp(t), _hp(o), _hp(r), _hp(k), ctypes.byref(n), _hp(trace),
                                    ctypes.byref(fp)))
    m = n.value
    return dict(iv_tensor=t[:m].copy(), iv_out=o[:m].copy(), iv_in=r[:m].copy(), iv_kind=k[:m].copy(),
                peak_trace=trace[:m - n0 + 1].copy(), final_peak=fp.value, n_initial=n0)


# ---------------------------------------------------------------- activations in 8 bits

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}   # TENSILE_F32, TENSILE_BF16, TENSILE_F16
_I8, _U8, _F32 = torch.int8, torch.uint8, torch.float32
GROUP = 32                                                         # columns that share a scale


class OpsHandle:
    """Owner of a ``tensile_ops*`` (scratch memory of the operators, per stream); freed on ``close()`` / garbage collection."""

    def __init__(self, ptr: int, device: int):
        self._ptr, self.device = ptr, device

    @property
    def ptr(self) -> int:
        if not self._ptr:
            raise TensileError(TENSILE_E_INVAL, "operators' handle already freed")
        return self._ptr

    def close(self) -> None:
        if self._ptr:
            _lib.tensile_ops_free(self._ptr)
            self._ptr = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Checkpoint:
    """A matrix of activations in 8 bits: ``q`` [rows, cols] int8 and ``scale`` [rows, ceil(cols / 32)] uint8, both on the GPU,
    the columns of a row contiguous (rows may lie further apart).  Either may be replaced, or be given other memory (as where a
    checkpoint leaves the GPU and comes back): the next call that takes the checkpoint looks at them anew."""

    __slots__ = ("_q", "_scale", "_q_at", "_scale_at", "_device", "_st")

    def __init__(self, q: torch.Tensor, scale: torch.Tensor):
        """What a call is told of the two tensors; done again when they are found elsewhere."""
        self._q, self._scale = q, scale
        q_shape, s_shape = q.shape, scale.shape
        self._device = q.get_device()                                    # -1: not on a GPU
        if q.dtype is not _I8 or scale.dtype is not _U8 or len(q_shape) != 2 or len(s_shape) != 2 or self._device < 0 or scale.get_device() != self._device:
            raise TensileError(TENSILE_E_INVAL, "checkpoint: need CUDA tensors q [rows, cols] int8 and scale [rows, ceil(cols/32)] uint8 on one device")
        rows, cols = q_shape
        groups = (cols + GROUP - 1) // GROUP
        ld_q, ld_s, wrong = cols, groups, s_shape[0] != rows or s_shape[1] != groups
        if not q.is_contiguous():
            row, col = q.stride()
            wrong = wrong or (cols > 1 and col != 1)
            if rows > 1:
                ld_q = row
        if not scale.is_contiguous():
            row, col = scale.stride()
            wrong = wrong or (groups > 1 and col != 1)
            if rows > 1:
                ld_s = row
        if wrong:
            raise TensileError(TENSILE_E_INVAL, f"checkpoint: q {tuple(q_shape)} and scale {tuple(s_shape)} do not belong together, "
                                                "or a row's columns are not contiguous")
        self._q_at, self._scale_at = q.data_ptr(), scale.data_ptr()
        self._st = _Ckpt(self._q_at, self._scale_at, rows, cols, ld_q, ld_s)

    @property
    def q(self) -> torch.Tensor:
        return self._q

    @q.setter
    def q(self, q: torch.Tensor) -> None:
        self._q, self._q_at = q, None

    @property
    def scale(self) -> torch.Tensor:
        return self._scale

    @scale.setter
    def scale(self, scale: torch.Tensor) -> None:
        self._scale, self._scale_at = scale, None

    @classmethod
    def empty(cls, rows: int, cols: int, device="cuda") -> "Checkpoint":
        """Room for rows x cols values; rows start at multiples of 16 bytes."""
        return cls(torch.empty(rows, (cols + 15) // 16 * 16, dtype=torch.int8, device=device)[:, :cols],
                   torch.empty(rows, (cols + GROUP - 1) // GROUP, dtype=torch.uint8, device=device))

    @property
    def shape(self):
        return tuple(self.q.shape)

    @property
    def nbytes(self) -> int:
        if self._q.data_ptr() != self._q_at or self._scale.data_ptr() != self._scale_at:
            self.__init__(self._q, self._scale)
        return self._st.rows * (self._st.ld_q + self._st.ld_scale)


def _mat(device: int, t: Optional[torch.Tensor], name: str):
    """[..., cols] with contiguous columns and evenly spaced rows, as a matrix."""
    if t is None:
        return None
    code, shape = _TYPES.get(t.dtype), t.shape
    if code is None or t.get_device() != device or not shape:
        raise TensileError(TENSILE_E_INVAL, f"{name}: need a CUDA tensor on the handle's device ({device}), of float32, bfloat16 or float16, "
                                            "with at least one dimension")
    if t.is_contiguous():                                              # (one question fewer than the strides: small calls are bound here)
        cols = shape[-1]
        return _Matrix(t.data_ptr(), shape[0] if len(shape) == 2 else t.numel() // cols if cols else 0, cols, cols, code)
    if len(shape) != 2:
        raise TensileError(TENSILE_E_INVAL, f"{name}: a tensor of {len(shape)} dimensions has to be contiguous")
    rows, cols = shape
    row, col = t.stride()
    if cols > 1 and col != 1:
        raise TensileError(TENSILE_E_INVAL, f"{name}: the columns of a row have to be contiguous")
    return _Matrix(t.data_ptr(), rows, cols, row if rows > 1 else cols, code)


def _vec(device: int, t: Optional[torch.Tensor], dtype, n: int, name: str):
    if t is None:
        return None
    if t.get_device() != device or t.dtype != dtype or t.numel() != n or not t.is_contiguous():
        raise TensileError(TENSILE_E_INVAL, f"{name}: need a contiguous CUDA tensor on the handle's device ({device}), of {dtype} with {n} elements")
    return t.data_ptr()


def _ck(device: int, c: Optional[Checkpoint]):
    if c is None:
        return None
    if c._q.data_ptr() != c._q_at or c._scale.data_ptr() != c._scale_at:
        c.__init__(c._q, c._scale)
    if c._device != device:
        raise TensileError(TENSILE_E_INVAL, f"checkpoint: it is on device {c._device}, the handle belongs to device {device}")
    return c._st


def _missing(**args) -> None:
    for name, value in args.items():
        if value is None:
            raise TensileError(TENSILE_E_INVAL, f"{name}: is None")


# the current stream, without a Stream object where that is possible (2.8 us)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream_ptr(stream, ops: OpsHandle) -> int:
    if getattr(stream, "device_index", ops.device) != ops.device:
        raise TensileError(TENSILE_E_INVAL, f"stream: it is of device {stream.device_index}, the handle belongs to device {ops.device}")
    return stream.cuda_stream


def tensile_ops_create() -> OpsHandle:
    """A handle for the current device."""
    out = ctypes.c_void_p()
    _check(_lib.tensile_ops_create(ctypes.byref(out)))
    return OpsHandle(out.value, torch.cuda.current_device())


def tensile_ops_free(ops: OpsHandle) -> None:
    ops.close()


def tensile_ckpt_pack(ops: OpsHandle, x: torch.Tensor, c: Checkpoint, stream=None) -> None:
    """c = x in 8 bits"""
    d = ops.device
    rc = _lib.tensile_ckpt_pack(ops._ptr or ops.ptr, _mat(d, x, "x"), _ck(d, c), _raw_stream(d) if stream is None else _stream_ptr(stream, ops))
    if rc:
        _check(rc)


def tensile_ckpt_unpack(ops: OpsHandle, c: Checkpoint, y: torch.Tensor, stream=None) -> None:
    """y = the values of c"""
    d = ops.device
    rc = _lib.tensile_ckpt_unpack(ops._ptr or ops.ptr, _ck(d, c), _mat(d, y, "y"), _raw_stream(d) if stream is None else _stream_ptr(stream, ops))
    if rc:
        _check(rc)


def tensile_layer_norm(ops: OpsHandle, x: torch.Tensor, gamma: torch.Tensor, beta: torch.Tensor, y: torch.Tensor, eps: float = 1e-5,
                       residual: Optional[torch.Tensor] = None, total: Optional[torch.Tensor] = None, xhat: Optional[Checkpoint] = None,
                       rstd: Optional[torch.Tensor] = None, stream=None) -> None:
    """y = layer norm of x (+ residual); total: the sum; xhat, rstd: what the backward pass reads"""
    if x is None or gamma is None:
        _missing(x=x, gamma=gamma)
    d = ops.device
    m = _mat(d, x, "x")
    rc = _lib.tensile_layer_norm(ops._ptr or ops.ptr, m, _mat(d, residual, "residual"), _vec(d, gamma, gamma.dtype, m.cols, "gamma"),
                                 _vec(d, beta, gamma.dtype, m.cols, "beta"), _TYPES.get(gamma.dtype, -1), eps, _mat(d, y, "y"), _mat(d, total, "total"),
                                 _ck(d, xhat), _vec(d, rstd, _F32, m.rows, "rstd"), _raw_stream(d) if stream is None else _stream_ptr(stream, ops))
    if rc:
        _check(rc)


def tensile_layer_norm_backward(ops: OpsHandle, dy: torch.Tensor, xhat: Checkpoint, rstd: torch.Tensor, gamma: torch.Tensor, dx: torch.Tensor,
                                dgamma: Optional[torch.Tensor] = None, dbeta: Optional[torch.Tensor] = None,
                                dresidual: Optional[torch.Tensor] = None, stream=None) -> None:
    """dx = gradient through the norm (+ dresidual); dgamma, dbeta: the parameters' gradients"""
    if dy is None or gamma is None:
        _missing(dy=dy, gamma=gamma)
    d = ops.device
    m = _mat(d, dy, "dy")
    rc = _lib.tensile_layer_norm_backward(ops._ptr or ops.ptr, m, _ck(d, xhat), _vec(d, rstd, _F32, m.rows, "rstd"),
                                          _vec(d, gamma, gamma.dtype, m.cols, "gamma"), _TYPES.get(gamma.dtype, -1), _mat(d, dresidual, "dresidual"),
                                          _mat(d, dx, "dx"), _vec(d, dgamma, gamma.dtype, m.cols, "dgamma"),
                                          _vec(d, dbeta, gamma.dtype, m.cols, "dbeta"), _raw_stream(d) if stream is None else _stream_ptr(stream, ops))
    if rc:
        _check(rc)


def tensile_gelu(ops: OpsHandle, x: torch.Tensor, y: torch.Tensor, ckpt: Optional[Checkpoint] = None, tanh: bool = False, stream=None) -> None:
    """y = gelu(x); ckpt: x in 8 bits"""
    d = ops.device
    rc = _lib.tensile_gelu(ops._ptr or ops.ptr, _mat(d, x, "x"), _mat(d, y, "y"), _ck(d, ckpt), 1 if tanh else 0, _raw_stream(d) if stream is None else _stream_ptr(stream, ops))
    if rc:
        _check(rc)


def tensile_gelu_backward(ops: OpsHandle, dy: torch.Tensor, ckpt: Checkpoint, dx: torch.Tensor, y_ckpt: Optional[Checkpoint] = None,
                          tanh: bool = False, stream=None) -> None:
    """dx = dy * gelu'(x) at the x that ckpt holds; y_ckpt: gelu(x) in 8 bits, for the next layer's weight gradient"""
    d = ops.device
    rc = _lib.tensile_gelu_backward(ops._ptr or ops.ptr, _mat(d, dy, "dy"), _ck(d, ckpt), _mat(d, dx, "dx"), _ck(d, y_ckpt), 1 if tanh else 0, _raw_stream(d) if stream is None else _stream_ptr(stream, ops))
    if rc:
        _check(rc)


def tensile_linear_grad(ops: OpsHandle, dy: torch.Tensor, ckpt: Checkpoint, dw: torch.Tensor, dbias: Optional[torch.Tensor] = None,
                        gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None, stream=None) -> None:
    """dw [N, K] = dy^T X, dbias [N] = column sums of dy; X is what ckpt holds, or that * gamma + beta"""
    if dy is None or ckpt is None or dw is None:
        _missing(dy=dy, ckpt=ckpt, dw=dw)
    d = ops.device
    m, c = _mat(d, dy, "dy"), _ck(d, ckpt)
    K = c.cols
    param = None if gamma is None else gamma.dtype
    rc = _lib.tensile_linear_grad(ops._ptr or ops.ptr, m, c, _vec(d, gamma, param, K, "gamma"), _vec(d, beta, param, K, "beta"), _TYPES.get(param, 0 if param is None else -1),
                                  _mat(d, dw, "dw"), _vec(d, dbias, dw.dtype, m.cols, "dbias"), _raw_stream(d) if stream is None else _stream_ptr(stream, ops))
    if rc:
        _check(rc)
