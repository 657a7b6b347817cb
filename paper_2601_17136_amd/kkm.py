"""Thin ctypes binding to libkkm.so: the C ABI of include/kkm.h under the same names.

Only argument marshalling happens here: device tensors become raw pointers
(after dtype/device/contiguity checks), host results come back as Python
values, and a non-zero status raises KKMError with the library's message.
Every step of the computation runs in the library's HIP kernels.  If the
library has not been built, loading it fails loudly; there is no fallback.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libkkm.so")

KKM_OK, KKM_ERR_ARG, KKM_ERR_OOM, KKM_ERR_HIP, KKM_ERR_STATE, KKM_ERR_DEVICE_DATA = 0, -1, -2, -3, -4, -5
KKM_LINEAR, KKM_POLY, KKM_GAUSS = 0, 1, 2
KKM_MODE_AUTO, KKM_MODE_RESIDENT, KKM_MODE_ONTHEFLY, KKM_MODE_PACKED = 0, 1, 2, 3
KKM_STORE_F32, KKM_STORE_F16 = 0, 1
KKM_F32, KKM_F16, KKM_BF16 = 0, 1, 2
KKM_MAX_TOP, KKM_MAX_FEATURES, KKM_MAX_ROWS = 256, 1 << 20, 1 << 21
KKM_MAX_RANK, KKM_MAX_ADAPTERS = 128, 1024
KKM_MAX_STEPS, KKM_MAX_GIVEN, KKM_MAX_BIASES = 32, (1 << 20) - 1, 1000
# Steps that bring singular values from 0.01 .. 1 to 0.7 .. 1.2 in five, and steps that bring them to 1 in the end.
KKM_QUINTIC, KKM_CUBIC = (3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0)
STORAGES = {"f32": KKM_STORE_F32, "f16": KKM_STORE_F16}
KKM_MAX_K = 1024
KKM_PACKED_MAX_K = 64
KKM_PACKED_FAST_K = 64
KKM_ABI_VERSION = 8
KKM_NOALLOC_SCRATCH_BYTES = 64 << 20
PHASES = ("stage", "gemm", "fixup", "labels", "scatter", "spmm", "assign", "onthefly", "reduce", "other",
          "seed")
KINDS = {"linear": KKM_LINEAR, "poly": KKM_POLY, "gauss": KKM_GAUSS}
MODES = {"auto": KKM_MODE_AUTO, "resident": KKM_MODE_RESIDENT, "onthefly": KKM_MODE_ONTHEFLY,
         "packed": KKM_MODE_PACKED}


class KKMError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"kkm error {code}: {msg}")
        self.code = code


class kkm_params(ctypes.Structure):
    _fields_ = [("gamma", ctypes.c_float), ("coef0", ctypes.c_float),
                ("degree", ctypes.c_int32), ("mode", ctypes.c_int32), ("storage", ctypes.c_int32),
                ("k_hint", ctypes.c_int32)]


class kkm_timing(ctypes.Structure):
    _fields_ = [("ms", ctypes.c_double * len(PHASES)), ("launches", ctypes.c_int64 * len(PHASES))]


class kkm_info(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64), ("d", ctypes.c_int32), ("d_pad", ctypes.c_int32),
                ("kind", ctypes.c_int32), ("mode", ctypes.c_int32), ("storage", ctypes.c_int32),
                ("ld", ctypes.c_int64),
                ("bytes_K", ctypes.c_size_t), ("bytes_total", ctypes.c_size_t),
                ("fixups", ctypes.c_int64), ("fixup_capacity", ctypes.c_int64),
                ("r0", ctypes.c_int64), ("r1", ctypes.c_int64), ("c0", ctypes.c_int64), ("c1", ctypes.c_int64)]


class kkm_head(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int32), ("d", ctypes.c_int32), ("n", ctypes.c_int64),
                ("classes", ctypes.c_int64), ("h", ctypes.c_void_p), ("ldh", ctypes.c_int64),
                ("w", ctypes.c_void_p), ("ldw", ctypes.c_int64), ("offset", ctypes.c_void_p),
                ("scale", ctypes.c_float)]


class kkm_teacher(ctypes.Structure):
    _fields_ = [("ids", ctypes.c_void_p), ("logits", ctypes.c_void_p), ("m", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class kkm_adapted(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int32), ("d", ctypes.c_int32), ("n", ctypes.c_int64), ("m", ctypes.c_int64),
                ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("w", ctypes.c_void_p), ("ldw", ctypes.c_int64),
                ("adapters", ctypes.c_int32), ("rank", ctypes.c_int32), ("down", ctypes.c_void_p),
                ("up", ctypes.c_void_p), ("ids", ctypes.c_void_p), ("factor", ctypes.c_void_p)]


class kkm_newton(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int32), ("coef", ctypes.POINTER(ctypes.c_double)), ("eps", ctypes.c_double)]


class kkm_choice(ctypes.Structure):
    _fields_ = [("type", ctypes.c_int32), ("classes", ctypes.c_int32), ("n", ctypes.c_int64), ("z", ctypes.c_void_p),
                ("ldz", ctypes.c_int64), ("scale", ctypes.c_float), ("offset", ctypes.c_void_p),
                ("given", ctypes.c_void_p), ("ngiven", ctypes.c_int32), ("repeat", ctypes.c_float),
                ("presence", ctypes.c_float), ("frequency", ctypes.c_float), ("bias_ids", ctypes.c_void_p),
                ("bias", ctypes.c_void_p), ("nbias", ctypes.c_int32), ("masks", ctypes.c_void_p),
                ("words", ctypes.c_int64), ("nmasks", ctypes.c_int32), ("mask_ids", ctypes.c_void_p)]


_lib = None
_vp, _i32, _i64, _f64, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double, ctypes.c_size_t
_f32, _headp, _teacherp = ctypes.c_float, ctypes.POINTER(kkm_head), ctypes.POINTER(kkm_teacher)
_adaptedp, _newtonp, _choicep = ctypes.POINTER(kkm_adapted), ctypes.POINTER(kkm_newton), ctypes.POINTER(kkm_choice)
_SIGS = {
    "kkm_abi_version": ([], _i32),
    "kkm_last_error": ([_vp], ctypes.c_char_p),
    "kkm_last_warning": ([_vp], ctypes.c_char_p),
    "kkm_create": ([ctypes.POINTER(_vp), _vp, _sz], _i32),
    "kkm_destroy": ([_vp], _i32),
    "kkm_plan": ([_i64, _i32, _i32, _i32, _sz, _i32, _i32, ctypes.POINTER(_i32), ctypes.POINTER(_sz)], _i32),
    "kkm_check_build_args": ([_i64, _i32, _i32, ctypes.POINTER(kkm_params)], _i32),
    "kkm_check_iterate_args": ([_i64, _i32, _i32], _i32),
    "kkm_build_kernel": ([_vp, _vp, _i64, _i32, _i32, ctypes.POINTER(kkm_params)], _i32),
    "kkm_iterate": ([_vp, _vp, _i32, _i32, _f64, ctypes.POINTER(_i32), _vp], _i32),
    "kkm_iterate_noalloc": ([_vp, _vp, _i32, _i32, _f64, ctypes.POINTER(_i32), _vp], _i32),
    "kkm_objective": ([_vp, _vp, _i32, ctypes.POINTER(_f64)], _i32),
    "kkm_step": ([_vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp, ctypes.POINTER(_f64)], _i32),
    "kkm_init_kmeanspp": ([_vp, _i32, _vp, _vp, _vp], _i32),
    "kkm_build_panel": ([_vp, _vp, _i64, _i32, _i32, ctypes.POINTER(kkm_params), _i64, _i64], _i32),
    "kkm_panel_spmm": ([_vp, _vp, _i32, _vp, _vp], _i32),
    "kkm_panel_assign": ([_vp, _i32, _vp, _vp, _vp, _vp], _i32),
    "kkm_build_block": ([_vp, _vp, _i64, _i32, _i32, ctypes.POINTER(kkm_params), _i64, _i64, _i64, _i64], _i32),
    "kkm_block_spmm": ([_vp, _vp, _i32, _vp], _i32),
    "kkm_block_zpart": ([_vp, _vp, _vp, _i64, _i64, _i32, _vp, _vp], _i32),
    "kkm_block_assign": ([_vp, _vp, _i64, _i64, _i32, _vp, _vp, _vp, _vp], _i32),
    "kkm_copy_kernel_rows": ([_vp, _i64, _i64, _vp], _i32),
    "kkm_copy_diag": ([_vp, _vp], _i32),
    "kkm_set_timing": ([_vp, _i32], _i32),
    "kkm_peak_read": ([_vp, _vp, _sz, _vp, _i32, ctypes.POINTER(ctypes.c_float)], _i32),
    "kkm_peak_read_rows": ([_vp, _vp, ctypes.c_int64, ctypes.c_int64, _vp, _i32, _i32, _vp, _i32,
                            ctypes.POINTER(ctypes.c_float)], _i32),
    "kkm_peak_write": ([_vp, _vp, _sz, ctypes.c_float, _i32, ctypes.POINTER(ctypes.c_float)], _i32),
    "kkm_peak_mfma": ([_vp, _i32, _vp, _i32, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(_f64)], _i32),
    "kkm_get_timing": ([_vp, ctypes.POINTER(kkm_timing)], _i32),
    "kkm_get_info": ([_vp, ctypes.POINTER(kkm_info)], _i32),
    "kkm_layer_norm": ([_vp, _i32, _i64, _i32, _vp, _i64, _i32, _vp, _vp, _f32, _vp, _i64, _vp, _vp], _i32),
    "kkm_layer_norm_grad": ([_vp, _i32, _i64, _i32, _vp, _i64, _i32, _vp, _vp, _vp, _vp, _i64, _vp, _i64, _vp, _vp],
                            _i32),
    "kkm_head_loss": ([_vp, _headp, _vp, _vp, _vp], _i32),
    "kkm_head_grad": ([_vp, _headp, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _i64], _i32),
    "kkm_distill_loss": ([_vp, _headp, _teacherp, _vp, _vp], _i32),
    "kkm_distill_grad": ([_vp, _headp, _teacherp, _vp, _vp, _vp, _vp, _i64, _vp, _i64], _i32),
    "kkm_check_norm_args": ([_i32, _i64, _i32, _i64, _i32, _f32], _i32),
    "kkm_check_head_args": ([_headp, _teacherp], _i32),
    "kkm_adapted_linear": ([_vp, _adaptedp, _vp, _i64], _i32),
    "kkm_adapted_linear_grad": ([_vp, _adaptedp, _vp, _i64, _vp, _i64, _vp, _vp], _i32),
    "kkm_orthogonalize": ([_vp, _newtonp, _i32, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64], _i32),
    "kkm_orthogonal_step": ([_vp, _newtonp, _i32, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _f32, _i32,
                             _f32, _f32], _i32),
    "kkm_choose": ([_vp, _choicep, _vp, _i64, _vp, _vp, _vp], _i32),
    "kkm_check_adapted_args": ([_adaptedp], _i32),
    "kkm_check_newton_args": ([_newtonp, _i32, _i64, _i64, _i64], _i32),
    "kkm_check_choice_args": ([_choicep], _i32),
    "kkm_get_stream": ([_vp, ctypes.POINTER(_vp)], _i32),
}


def lib():
    """Load libkkm.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python __graft_entry__.py build` "
                               "(hipcc --offload-arch=gfx950); the engine has no fallback")
        L = ctypes.CDLL(LIB_PATH)
        for name, (args, res) in _SIGS.items():
            f = getattr(L, name)
            f.argtypes, f.restype = args, res
        if L.kkm_abi_version() != KKM_ABI_VERSION:
            raise RuntimeError(f"{LIB_PATH} has ABI {L.kkm_abi_version()}, this binding {KKM_ABI_VERSION}: "
                               "rebuild it with `python __graft_entry__.py build`")
        _lib = L
    return _lib


def _check(rc: int, ctx=None):
    if rc != KKM_OK:
        msg = lib().kkm_last_error(ctx)
        raise KKMError(rc, msg.decode() if msg else "")


def _dev_ptr(t, dtype, name, numel=None):
    """Raw device address of a contiguous CUDA/HIP tensor, with its checks."""
    if t is None:
        return None
    try:  # (calls of a few microseconds are counted in these checks)
        if t.dtype is dtype and t.is_cuda and t.is_contiguous() and (numel is None or t.numel() == numel):
            return t.data_ptr()
    except AttributeError:
        pass
    if isinstance(t, int):
        return t
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{name} must have {numel} elements, got {t.numel()}")
    return t.data_ptr()


def _shaped(t, dtype, name, shape):
    """As _dev_ptr, of a tensor of this shape (dimensions of one aside) or of one dimension."""
    p = _dev_ptr(t, dtype, name, math.prod(shape))
    if t is None or isinstance(t, int) or t.shape == shape or t.dim() == 1:
        return p
    if [v for v in t.shape if v != 1] != [v for v in shape if v != 1]:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return p


def current_stream_handle():
    """hipStream_t of torch's current stream on the current device."""
    import torch
    return torch.cuda.current_stream().cuda_stream


# ------------------------------------------------------------------ the C ABI

def kkm_abi_version() -> int:
    return lib().kkm_abi_version()


def kkm_last_error(ctx=None) -> str:
    m = lib().kkm_last_error(ctx)
    return m.decode() if m else ""


def kkm_create(stream=None, mem_budget: int = 0):
    ctx = _vp()
    _check(lib().kkm_create(ctypes.byref(ctx), stream, int(mem_budget)))
    return ctx


def kkm_destroy(ctx) -> None:
    _check(lib().kkm_destroy(ctx))


def kkm_plan(n: int, d: int, k: int, kind: int, mem_budget: int, mode: int = KKM_MODE_AUTO,
             storage: int = KKM_STORE_F32):
    """(resolved mode, device bytes); raises KKMError(KKM_ERR_OOM) if it cannot fit."""
    m, b = _i32(), _sz()
    _check(lib().kkm_plan(int(n), int(d), int(k), int(kind), int(mem_budget), int(mode), int(storage),
                          ctypes.byref(m), ctypes.byref(b)))
    return m.value, b.value


def make_params(gamma=1.0, coef0=0.0, degree=1, mode=KKM_MODE_AUTO, storage=KKM_STORE_F32,
                k_hint=0) -> kkm_params:
    return kkm_params(float(gamma), float(coef0), int(degree), int(mode), int(storage), int(k_hint))


def kkm_last_warning(ctx=None) -> str:
    m = lib().kkm_last_warning(ctx)
    return m.decode() if m else ""


def _warn_if_any(ctx):
    msg = kkm_last_warning(ctx)
    if msg:
        import warnings
        warnings.warn(msg, RuntimeWarning, stacklevel=3)


def kkm_check_build_args(n, d, kind, params: kkm_params) -> int:
    return lib().kkm_check_build_args(int(n), int(d), int(kind), ctypes.byref(params))


def kkm_check_iterate_args(n, k, max_iter) -> int:
    return lib().kkm_check_iterate_args(int(n), int(k), int(max_iter))


def kkm_build_kernel(ctx, X, n: int, d: int, kind: int, params: kkm_params) -> None:
    import torch
    _check(lib().kkm_build_kernel(ctx, _dev_ptr(X, torch.float32, "X", int(n) * int(d)), int(n), int(d),
                                  int(kind), ctypes.byref(params)), ctx)
    _warn_if_any(ctx)


def kkm_iterate(ctx, V, k: int, max_iter: int, tol: float = -1.0):
    """Returns (iters_done, obj_hist[:iters_done] as numpy fp64)."""
    import torch
    it = _i32()
    hist = np.zeros(max(int(max_iter), 1), dtype=np.float64)
    _check(lib().kkm_iterate(ctx, _dev_ptr(V, torch.int32, "V"), int(k), int(max_iter), float(tol),
                             ctypes.byref(it), hist.ctypes.data), ctx)
    return it.value, hist[:it.value].copy()


def kkm_iterate_noalloc(ctx, V, k: int, max_iter: int, tol: float = -1.0):
    """kkm_iterate on the library's static device scratch (no device allocation
    in the call).  Returns (iters_done, obj_hist[:iters_done] as numpy fp64)."""
    import torch
    it = _i32()
    hist = np.zeros(max(int(max_iter), 1), dtype=np.float64)
    _check(lib().kkm_iterate_noalloc(ctx, _dev_ptr(V, torch.int32, "V"), int(k), int(max_iter), float(tol),
                                     ctypes.byref(it), hist.ctypes.data), ctx)
    return it.value, hist[:it.value].copy()


def kkm_objective(ctx, V, k: int) -> float:
    import torch
    J = _f64()
    _check(lib().kkm_objective(ctx, _dev_ptr(V, torch.int32, "V"), int(k), ctypes.byref(J)), ctx)
    return J.value


def kkm_step(ctx, cl_in, k: int, E=None, z=None, D=None, cl_out=None, counts_out=None) -> float:
    """One step with every intermediate; returns J(cl_in).  Outputs are device tensors or None."""
    import torch
    J = _f64()
    _check(lib().kkm_step(ctx, _dev_ptr(cl_in, torch.int32, "cl_in"), int(k),
                          _dev_ptr(E, torch.float32, "E"), _dev_ptr(z, torch.float32, "z", int(k)),
                          _dev_ptr(D, torch.float32, "D"), _dev_ptr(cl_out, torch.int32, "cl_out"),
                          _dev_ptr(counts_out, torch.int32, "counts_out", int(k)), ctypes.byref(J)), ctx)
    return J.value


def kkm_build_panel(ctx, X, n: int, d: int, kind: int, params: kkm_params, c0: int, c1: int) -> None:
    """One GPU's share: the column panel K[:, c0:c1] (c0 a multiple of 128)."""
    import torch
    _check(lib().kkm_build_panel(ctx, _dev_ptr(X, torch.float32, "X", int(n) * int(d)), int(n), int(d),
                                 int(kind), ctypes.byref(params), int(c0), int(c1)), ctx)
    _warn_if_any(ctx)


def _stored(ctx):
    """(r0, r1, c0, c1) of the K the context holds, or None before a build."""
    info = kkm_info()
    if lib().kkm_get_info(ctx, ctypes.byref(info)) != KKM_OK:
        return None
    return info.r0, info.r1, info.c0, info.c1


def kkm_panel_spmm(ctx, cl, k: int):
    """E for the panel's points (kept); returns (zpart as numpy fp64[k], sizes as numpy int32[k])."""
    import torch
    st = _stored(ctx)
    zpart = np.zeros(int(k), dtype=np.float64)
    counts = np.zeros(int(k), dtype=np.int32)
    _check(lib().kkm_panel_spmm(ctx, _dev_ptr(cl, torch.int32, "cl", st and st[1] - st[0]), int(k),
                                zpart.ctypes.data, counts.ctypes.data), ctx)
    return zpart, counts


def kkm_panel_assign(ctx, k: int, z, cl_out, E_out=None) -> np.ndarray:
    """New ids of the panel's points into cl_out from the global z; returns
    how many of them took each id (numpy int32[k])."""
    import torch
    z = np.ascontiguousarray(z, dtype=np.float64)
    if z.shape != (int(k),):
        raise KKMError(KKM_ERR_ARG, f"z must hold k={k} values, got shape {z.shape}")
    st = _stored(ctx)
    w = st and st[3] - st[2]
    counts = np.zeros(int(k), dtype=np.int32)
    _check(lib().kkm_panel_assign(ctx, int(k), z.ctypes.data, _dev_ptr(cl_out, torch.int32, "cl_out", w),
                                  _dev_ptr(E_out, torch.float32, "E_out", w and w * int(k)),
                                  counts.ctypes.data), ctx)
    return counts


def kkm_build_block(ctx, X, n: int, d: int, kind: int, params: kkm_params, r0: int, r1: int, c0: int,
                    c1: int) -> None:
    """One GPU's share of the 1.5D split: the block K[r0:r1, c0:c1] (r0, c0 multiples of 128)."""
    import torch
    _check(lib().kkm_build_block(ctx, _dev_ptr(X, torch.float32, "X", int(n) * int(d)), int(n), int(d),
                                 int(kind), ctypes.byref(params), int(r0), int(r1), int(c0), int(c1)), ctx)
    _warn_if_any(ctx)


def kkm_block_spmm(ctx, cl, k: int, E_out) -> None:
    """The block's partial E (its c1 - c0 columns x k, point-major) into
    E_out from the ids cl of its rows r0 .. r1-1."""
    import torch
    st = _stored(ctx)
    _check(lib().kkm_block_spmm(ctx, _dev_ptr(cl, torch.int32, "cl", st and st[1] - st[0]), int(k),
                                _dev_ptr(E_out, torch.float32, "E_out", st and (st[3] - st[2]) * int(k))), ctx)


def kkm_block_zpart(ctx, E, cl, a0: int, a1: int, k: int):
    """Self-term parts and sizes of the piece [a0, a1) of the block's columns
    from its rows of E (device, (a1-a0) x k) and its ids; returns (zpart as
    numpy fp64[k], sizes as numpy int32[k])."""
    import torch
    m = max(int(a1) - int(a0), 0)
    zpart = np.zeros(int(k), dtype=np.float64)
    counts = np.zeros(int(k), dtype=np.int32)
    _check(lib().kkm_block_zpart(ctx, _dev_ptr(E, torch.float32, "E", m * int(k)),
                                 _dev_ptr(cl, torch.int32, "cl", m), int(a0), int(a1), int(k),
                                 zpart.ctypes.data, counts.ctypes.data), ctx)
    return zpart, counts


def kkm_block_assign(ctx, E, a0: int, a1: int, k: int, z, counts, cl_out) -> np.ndarray:
    """New ids of the piece [a0, a1) into cl_out from its rows of E and the
    global z and sizes; returns how many of its points took each id."""
    import torch
    m = max(int(a1) - int(a0), 0)
    z = np.ascontiguousarray(z, dtype=np.float64)
    counts = np.ascontiguousarray(counts, dtype=np.int32)
    if z.shape != (int(k),) or counts.shape != (int(k),):
        raise KKMError(KKM_ERR_ARG, f"z and counts must hold k={k} values, got {z.shape}, {counts.shape}")
    took = np.zeros(int(k), dtype=np.int32)
    _check(lib().kkm_block_assign(ctx, _dev_ptr(E, torch.float32, "E", m * int(k)), int(a0), int(a1), int(k),
                                  z.ctypes.data, counts.ctypes.data, _dev_ptr(cl_out, torch.int32, "cl_out", m),
                                  took.ctypes.data), ctx)
    return took


def kkm_init_kmeanspp(ctx, k: int, u, V) -> np.ndarray:
    """K-means++ seeding from the uniforms u (k floats in [0, 1)); writes the
    initial ids into V (device int32[n]) and returns the chosen centers."""
    import torch
    u = np.ascontiguousarray(u, dtype=np.float64)
    if u.shape != (int(k),):
        raise KKMError(KKM_ERR_ARG, f"u must hold k={k} uniforms, got shape {u.shape}")
    centers = np.zeros(int(k), dtype=np.int32)
    _check(lib().kkm_init_kmeanspp(ctx, int(k), u.ctypes.data, centers.ctypes.data,
                                   _dev_ptr(V, torch.int32, "V")), ctx)
    return centers


def kkm_copy_kernel_rows(ctx, r0: int, r1: int, out) -> None:
    """Rows r0 .. r1-1 of the stored K (of a panel or block: its columns) into out."""
    import torch
    st = _stored(ctx)
    numel = (int(r1) - int(r0)) * (st[3] - st[2]) if st and r1 > r0 else None
    _check(lib().kkm_copy_kernel_rows(ctx, int(r0), int(r1), _dev_ptr(out, torch.float32, "out", numel)), ctx)


def kkm_copy_diag(ctx, out) -> None:
    import torch
    st = _stored(ctx)
    n = kkm_get_info(ctx)["n"] if st else None
    _check(lib().kkm_copy_diag(ctx, _dev_ptr(out, torch.float32, "out", n)), ctx)


PEAK_READ_GROUPS = 2040  # workgroups of the streaming read and write


def kkm_peak_read(ctx, buf, sums, reps: int = 1) -> float:
    """Streaming-read microbenchmark over the fp32 device tensor buf; the sum read by
    workgroup g goes to sums[g], g < PEAK_READ_GROUPS.  Returns ms per launch."""
    import torch
    if sums.numel() < PEAK_READ_GROUPS:
        raise KKMError(KKM_ERR_ARG, f"sums must hold at least {PEAK_READ_GROUPS} floats (one per workgroup)")
    ms = ctypes.c_float()
    _check(lib().kkm_peak_read(ctx, _dev_ptr(buf, torch.float32, "buf"), buf.numel() * 4,
                               _dev_ptr(sums, torch.float32, "sums"), int(reps), ctypes.byref(ms)), ctx)
    return ms.value


def kkm_peak_read_rows(ctx, buf, rows, seg: int, sums, reps: int = 1) -> float:
    """Streaming read of rows in the packed SpMM's load pattern over the 2-D fp32
    device tensor buf (nrows x ld): workgroup (c, s) reads rows[128c .. 128c + 127]
    (int32 device tensor, clamped into range) over columns [s*seg, (s+1)*seg) and
    writes its sum to sums[c * (ld // seg) + s].  Returns ms per launch."""
    import torch
    if buf.dim() != 2 or not buf.is_contiguous():
        raise KKMError(KKM_ERR_ARG, "buf must be a contiguous 2-D tensor")
    nrows, ld = buf.shape
    if rows.numel() % 128 or rows.numel() == 0:
        raise KKMError(KKM_ERR_ARG, "rows must hold a positive multiple of 128 indices")
    nchunks = rows.numel() // 128
    if seg > 0 and sums.numel() < nchunks * (ld // seg):
        raise KKMError(KKM_ERR_ARG, f"sums must hold at least {nchunks * (ld // seg)} floats")
    ms = ctypes.c_float()
    _check(lib().kkm_peak_read_rows(ctx, _dev_ptr(buf, torch.float32, "buf"), nrows, ld,
                                    _dev_ptr(rows, torch.int32, "rows"), nchunks, int(seg),
                                    _dev_ptr(sums, torch.float32, "sums"), int(reps), ctypes.byref(ms)), ctx)
    return ms.value


def kkm_peak_write(ctx, buf, value: float, reps: int = 1) -> float:
    """Streaming-write microbenchmark: value into every element of buf.  Returns ms per launch."""
    import torch
    ms = ctypes.c_float()
    _check(lib().kkm_peak_write(ctx, _dev_ptr(buf, torch.float32, "buf"), buf.numel() * 4, float(value),
                                int(reps), ctypes.byref(ms)), ctx)
    return ms.value


def kkm_peak_mfma(ctx, iters: int, out, reps: int = 1):
    """fp32 MFMA register loop; out >= 4096 floats.  Returns (ms per launch, flop per launch)."""
    import torch
    if out.numel() < 4096:
        raise KKMError(KKM_ERR_ARG, "out must hold at least 4096 floats (one per wavefront)")
    ms, fl = ctypes.c_float(), _f64()
    _check(lib().kkm_peak_mfma(ctx, int(iters), _dev_ptr(out, torch.float32, "out"), int(reps),
                               ctypes.byref(ms), ctypes.byref(fl)), ctx)
    return ms.value, fl.value


KKM_TIME_ALL = (1 << len(PHASES)) - 1


def phase_mask(*names) -> int:
    """Bit mask of the named phases for kkm_set_timing."""
    return sum(1 << PHASES.index(n) for n in names)


def kkm_set_timing(ctx, phase_mask_: int) -> None:
    """phase_mask_: phases to bracket with HIP events (KKM_TIME_ALL, 0 = off)."""
    _check(lib().kkm_set_timing(ctx, int(phase_mask_)), ctx)


def kkm_get_timing(ctx) -> dict:
    t = kkm_timing()
    _check(lib().kkm_get_timing(ctx, ctypes.byref(t)), ctx)
    return {p: (t.ms[i], t.launches[i]) for i, p in enumerate(PHASES)}


def kkm_get_info(ctx) -> dict:
    i = kkm_info()
    _check(lib().kkm_get_info(ctx, ctypes.byref(i)), ctx)
    return {f: getattr(i, f) for f, _ in kkm_info._fields_}


# ------------------------------------------------------------------ a model that learns from a clustering

_TYPE_CODES = {}


def _type_code(dtype, name):
    if not _TYPE_CODES:
        import torch
        _TYPE_CODES.update({torch.float32: KKM_F32, torch.float16: KKM_F16, torch.bfloat16: KKM_BF16})
    code = _TYPE_CODES.get(dtype)
    if code is None:
        raise TypeError(f"{name} must have dtype float32, float16 or bfloat16, got {dtype}")
    return code


def _rows(t, name, dtype=None, shape=None):
    """(address, row stride in elements) of a device matrix whose rows are contiguous."""
    if not getattr(t, "is_cuda", False):
        raise TypeError(f"{name} must be a device tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    size = t.shape
    if len(size) != 2:
        raise ValueError(f"{name} must be a matrix, got {len(size)} dimensions")
    if shape is not None and size != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(size)}")
    n, d = size
    ld, step = t.stride()
    if d > 1 and step != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    if ld < d:
        if n > 1:
            raise ValueError(f"{name}'s rows overlap (stride {ld}, width {d})")
        ld = d
    return t.data_ptr(), ld


class _Elsewhere:
    """Work on the context's stream while torch's current stream of the tensors'
    device is another: it waits for what that stream has enqueued, that stream
    waits for it, and the tensors' memory is held until then (memory given as an
    address is the caller's to keep)."""

    def __init__(self, handle, tensors):
        import torch
        device = tensors[0].device
        self.here = torch.cuda.current_stream(device)
        self.there = (torch.cuda.ExternalStream(handle, device=device) if handle
                      else torch.cuda.default_stream(device))
        self.tensors = [t for t in tensors if t is not None and not isinstance(t, int)]

    def __enter__(self):
        self.there.wait_stream(self.here)

    def __exit__(self, *exc):
        self.here.wait_stream(self.there)
        for t in self.tensors:
            t.record_stream(self.there)


_HERE = contextlib.nullcontext()


def _ordered(ctx, *tensors):
    """The context's stream as the place of the call's work."""
    import torch
    handle = kkm_get_stream(ctx)
    if handle == torch._C._cuda_getCurrentRawStream(tensors[0].device.index):
        return _HERE
    return _Elsewhere(handle, tensors)


def kkm_layer_norm(ctx, x, weight, bias, eps: float, y, mean=None, rstd=None) -> None:
    """Layer norm of the rows of x (n x d) into y; weight and bias (fp32 or x's
    dtype) may be None.  mean and rstd (fp32[n]) take the statistics that the
    gradient needs.  y may be x."""
    import torch
    px, ldx = _rows(x, "x")
    n, d = x.shape
    py, ldy = _rows(y, "y", x.dtype, (n, d))
    wdt = _weight_dtype(x, weight, bias)
    with _ordered(ctx, x, weight, bias, y, mean, rstd):
        _check(lib().kkm_layer_norm(ctx, _type_code(x.dtype, "x"), n, d, px, ldx, _type_code(wdt, "weight"),
                                    _dev_ptr(weight, wdt, "weight", d), _dev_ptr(bias, wdt, "bias", d), float(eps),
                                    py, ldy, _dev_ptr(mean, torch.float32, "mean", n),
                                    _dev_ptr(rstd, torch.float32, "rstd", n)), ctx)


def _weight_dtype(x, *vectors):
    import torch
    for v in vectors:
        if v is not None:
            return v.dtype
    return torch.float32


def kkm_layer_norm_grad(ctx, x, weight, dy, mean, rstd, dx=None, dweight=None, dbias=None) -> None:
    """The gradient of kkm_layer_norm from dy into dx, dweight and dbias (each
    may be None; the last two have weight's dtype)."""
    import torch
    px, ldx = _rows(x, "x")
    n, d = x.shape
    pdy, lddy = _rows(dy, "dy", x.dtype, (n, d))
    pdx, lddx = _rows(dx, "dx", x.dtype, (n, d)) if dx is not None else (None, d)
    wdt = _weight_dtype(x, weight, dweight, dbias)
    with _ordered(ctx, x, weight, dy, mean, rstd, dx, dweight, dbias):
        _check(lib().kkm_layer_norm_grad(ctx, _type_code(x.dtype, "x"), n, d, px, ldx, _type_code(wdt, "weight"),
                                         _dev_ptr(weight, wdt, "weight", d), _dev_ptr(mean, torch.float32, "mean", n),
                                         _dev_ptr(rstd, torch.float32, "rstd", n), pdy, lddy, pdx, lddx,
                                         _dev_ptr(dweight, wdt, "dweight", d), _dev_ptr(dbias, wdt, "dbias", d)), ctx)


def _head_args(h, w, scale, offset):
    import torch
    ph, ldh = _rows(h, "h")
    pw, ldw = _rows(w, "w", h.dtype)
    n, d = h.shape
    if w.shape[1] != d:
        raise ValueError(f"w must be as wide as h ({d}), got {w.shape[1]}")
    return kkm_head(_type_code(h.dtype, "h"), d, n, w.shape[0], ph, ldh, pw, ldw,
                    _dev_ptr(offset, torch.float32, "offset", w.shape[0]), float(scale))


def _teacher_args(n, top_ids, top_logits, teacher_scale):
    import torch
    if top_ids.dim() != 2 or top_ids.shape[0] != n:
        raise ValueError(f"top_ids must be a matrix of {n} rows, got shape {tuple(top_ids.shape)}")
    m = top_ids.shape[1]
    return kkm_teacher(_dev_ptr(top_ids, torch.int32, "top_ids"),
                       _dev_ptr(top_logits, torch.float32, "top_logits", n * m), m, float(teacher_scale))


def _head_grads(h, w, dh, dw):
    pdh, lddh = _rows(dh, "dh", h.dtype, h.shape) if dh is not None else (None, 0)
    pdw, lddw = _rows(dw, "dw", h.dtype, w.shape) if dw is not None else (None, 0)
    return pdh, lddh, pdw, lddw


def kkm_head_loss(ctx, h, w, ids, loss, lse, scale: float = 1.0, offset=None) -> None:
    """Softmax cross entropy of the logits scale * h w^T + offset with ids
    (int32[n]; negative: no label) into loss and lse (fp32[n])."""
    import torch
    a, n, f32 = _head_args(h, w, scale, offset), h.shape[0], torch.float32
    with _ordered(ctx, h, w, offset, ids, loss, lse):
        _check(lib().kkm_head_loss(ctx, ctypes.byref(a), _dev_ptr(ids, torch.int32, "ids", n),
                                   _dev_ptr(loss, f32, "loss", n), _dev_ptr(lse, f32, "lse", n)), ctx)


def kkm_head_grad(ctx, h, w, ids, dloss, loss, lse, dh=None, dw=None, scale: float = 1.0, offset=None) -> None:
    """kkm_head_loss, and the gradient of sum(dloss * loss) by h and w into dh and dw (each may be None)."""
    import torch
    a, n, f32 = _head_args(h, w, scale, offset), h.shape[0], torch.float32
    g = _head_grads(h, w, dh, dw)
    with _ordered(ctx, h, w, offset, ids, dloss, loss, lse, dh, dw):
        _check(lib().kkm_head_grad(ctx, ctypes.byref(a), _dev_ptr(ids, torch.int32, "ids", n),
                                   _dev_ptr(dloss, f32, "dloss", n), _dev_ptr(loss, f32, "loss", n),
                                   _dev_ptr(lse, f32, "lse", n), *g), ctx)


def kkm_distill_loss(ctx, h, w, top_ids, top_logits, loss, lse, scale: float = 1.0, offset=None,
                     teacher_scale: float = 1.0) -> None:
    """Divergence of softmax(scale * h w^T + offset) from the teacher's
    softmax(teacher_scale * top_logits) over the classes top_ids (int32, n x m)."""
    import torch
    a, n, f32 = _head_args(h, w, scale, offset), h.shape[0], torch.float32
    t = _teacher_args(n, top_ids, top_logits, teacher_scale)
    with _ordered(ctx, h, w, offset, top_ids, top_logits, loss, lse):
        _check(lib().kkm_distill_loss(ctx, ctypes.byref(a), ctypes.byref(t), _dev_ptr(loss, f32, "loss", n),
                                      _dev_ptr(lse, f32, "lse", n)), ctx)


def kkm_distill_grad(ctx, h, w, top_ids, top_logits, dloss, loss, lse, dh=None, dw=None, scale: float = 1.0,
                     offset=None, teacher_scale: float = 1.0) -> None:
    """kkm_distill_loss, and the gradient of sum(dloss * loss) by h and w into dh and dw (each may be None)."""
    import torch
    a, n, f32 = _head_args(h, w, scale, offset), h.shape[0], torch.float32
    t = _teacher_args(n, top_ids, top_logits, teacher_scale)
    g = _head_grads(h, w, dh, dw)
    with _ordered(ctx, h, w, offset, top_ids, top_logits, dloss, loss, lse, dh, dw):
        _check(lib().kkm_distill_grad(ctx, ctypes.byref(a), ctypes.byref(t), _dev_ptr(dloss, f32, "dloss", n),
                                      _dev_ptr(loss, f32, "loss", n), _dev_ptr(lse, f32, "lse", n), *g), ctx)


def _adapted_args(x, w, down, up, ids, factor):
    import torch
    px, ldx = _rows(x, "x")
    pw, ldw = _rows(w, "w", x.dtype)
    n, d = x.shape
    m = w.shape[0]
    if w.shape[1] != d:
        raise ValueError(f"w must be as wide as x ({d}), got {w.shape[1]}")
    if down.dim() != 3 or down.shape[2] != d:
        raise ValueError(f"down must have shape (adapters, rank, {d}), got {tuple(down.shape)}")
    s, rank, _ = down.shape
    if up.shape != (s, m, rank):
        raise ValueError(f"up must have shape {(s, m, rank)}, got {tuple(up.shape)}")
    return kkm_adapted(_type_code(x.dtype, "x"), d, n, m, px, ldx, pw, ldw, s, rank, _dev_ptr(down, x.dtype, "down"),
                       _dev_ptr(up, x.dtype, "up"), _dev_ptr(ids, torch.int32, "ids", n),
                       _dev_ptr(factor, torch.float32, "factor", s))


def kkm_adapted_linear(ctx, x, w, down, up, ids, y, factor=None) -> None:
    """y = x w^T, and for a row i of adapter g = ids[i] (int32[n]; negative: none)
    factor[g] up[g] (down[g] x_i) added, into y (n x m).  down: adapters x rank x d,
    up: adapters x m x rank, contiguous, of x's dtype; factor: fp32[adapters] or None."""
    a = _adapted_args(x, w, down, up, ids, factor)
    py, ldy = _rows(y, "y", x.dtype, (x.shape[0], w.shape[0]))
    with _ordered(ctx, x, w, down, up, ids, y, factor):
        _check(lib().kkm_adapted_linear(ctx, ctypes.byref(a), py, ldy), ctx)


def kkm_adapted_linear_grad(ctx, x, w, down, up, ids, dy, dx=None, ddown=None, dup=None, factor=None) -> None:
    """The gradient of kkm_adapted_linear from dy (n x m) by x, down and up, into dx,
    ddown and dup (each may be None); w is held."""
    a = _adapted_args(x, w, down, up, ids, factor)
    pdy, lddy = _rows(dy, "dy", x.dtype, (x.shape[0], w.shape[0]))
    pdx, lddx = _rows(dx, "dx", x.dtype, x.shape) if dx is not None else (None, 0)
    with _ordered(ctx, x, w, down, up, ids, dy, dx, ddown, dup, factor):
        _check(lib().kkm_adapted_linear_grad(ctx, ctypes.byref(a), pdy, lddy, pdx, lddx,
                                             _shaped(ddown, x.dtype, "ddown", down.shape),
                                             _shaped(dup, x.dtype, "dup", up.shape)), ctx)


def _matrices(t, name, dtype=None, shape=None):
    """(address, row stride, matrix stride) of a device matrix, or of a batch of them, with contiguous rows."""
    if not getattr(t, "is_cuda", False):
        raise TypeError(f"{name} must be a device tensor")
    if t.dim() not in (2, 3):
        raise ValueError(f"{name} must be a matrix or a batch of them, got {t.dim()} dimensions")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dim() == 2:
        p, ld = _rows(t, name, dtype)
        return p, ld, 0
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    batch, m, n = t.shape
    stride, ld, step = t.stride()
    if n > 1 and step != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    if m <= 1:
        ld = n
    if ld < n:
        raise ValueError(f"{name}'s rows overlap (stride {ld}, width {n})")
    if batch > 1 and stride < (m - 1) * ld + n:
        raise ValueError(f"{name}'s matrices overlap (stride {stride})")
    return t.data_ptr(), ld, stride


def _newton_args(coef, eps):
    if any(len(step) != 3 for step in coef):
        raise ValueError("coef must hold three numbers a step")
    flat = [float(v) for step in coef for v in step]
    return kkm_newton(len(coef), (ctypes.c_double * max(len(flat), 1))(*flat), float(eps))


def _batch_shape(t):
    return (1, *t.shape) if t.dim() == 2 else tuple(t.shape)


def kkm_orthogonalize(ctx, x, y, coef=(KKM_QUINTIC,) * 5, eps: float = 1e-7) -> None:
    """Each matrix of x (m x n, or batch x m x n) divided by the root of its sum of
    squares + eps and taken through Newton-Schulz steps, into y.  coef: (a, b, c)
    of each step, X <- a X + (b A + c A A) X with A = X X^T.  y may be x."""
    px, ldx, sx = _matrices(x, "x")
    py, ldy, sy = _matrices(y, "y", x.dtype, x.shape)
    w = _newton_args(coef, eps)
    with _ordered(ctx, x, y):
        _check(lib().kkm_orthogonalize(ctx, ctypes.byref(w), _type_code(x.dtype, "x"), *_batch_shape(x), px, ldx, sx,
                                       py, ldy, sy), ctx)


def kkm_orthogonal_step(ctx, w, g, v, rate: float, momentum: float = 0.95, nesterov: bool = True, keep: float = 1.0,
                        coef=(KKM_QUINTIC,) * 5, eps: float = 1e-7) -> None:
    """v = momentum v + g, u = g + momentum v (nesterov) or v, w = keep w - rate X with
    X from u as in kkm_orthogonalize.  w and g (m x n, or batch x m x n) of one dtype,
    v fp32, contiguous, of w's shape."""
    import torch
    pw, ldw, sw = _matrices(w, "w")
    pg, ldg, sg = _matrices(g, "g", w.dtype, w.shape)
    a = _newton_args(coef, eps)
    with _ordered(ctx, w, g, v):
        _check(lib().kkm_orthogonal_step(ctx, ctypes.byref(a), _type_code(w.dtype, "w"), *_batch_shape(w), pw, ldw, sw,
                                         pg, ldg, sg, _shaped(v, torch.float32, "v", w.shape), float(momentum),
                                         int(nesterov), float(rate), float(keep)), ctx)


def _list_width(t, n, name):
    """Entries a row of a list matrix (0 of None)."""
    if t is None:
        return 0
    if t.dim() != 2 or t.shape[0] != n:
        raise ValueError(f"{name} must be a matrix of {n} rows, got shape {tuple(t.shape)}")
    return t.shape[1]


def kkm_choose(ctx, z, out=None, ids=None, logp=None, lse=None, scale: float = 1.0, offset=None, given=None,
               repeat: float = 1.0, presence: float = 0.0, frequency: float = 0.0, bias_ids=None, bias=None, masks=None,
               mask_ids=None) -> None:
    """Answers from logits z (n x classes): penalties for the ids in given (int32, n x
    any; negative: none), offset (fp32[classes]) and biases (bias of bias_ids, n x any)
    added, scale, and the bit masks (int32, masks x words) that mask_ids (int32[n];
    negative: none) names; into out (may be z), the first of the largest ids (int32[n]),
    logp and lse (fp32[n]); each may be None."""
    import torch
    pz, ldz = _rows(z, "z")
    n, classes = z.shape
    pout, ldo = _rows(out, "out", z.dtype, z.shape) if out is not None else (None, 0)
    i32, f32 = torch.int32, torch.float32
    h, b = _list_width(given, n, "given"), _list_width(bias_ids, n, "bias_ids")
    if b and bias is None:
        raise ValueError("bias_ids need bias")
    if bias is not None and bias_ids is None:
        raise ValueError("bias needs bias_ids")
    if masks is not None and masks.dim() != 2:
        raise ValueError(f"masks must be a matrix, got {masks.dim()} dimensions")
    a = kkm_choice(_type_code(z.dtype, "z"), classes, n, pz, ldz, float(scale),
                   _dev_ptr(offset, f32, "offset", classes), _dev_ptr(given, i32, "given") if h else None, h,
                   float(repeat), float(presence), float(frequency),
                   _dev_ptr(bias_ids, i32, "bias_ids") if b else None,
                   _shaped(bias, f32, "bias", (n, b)) if b else None, b, _dev_ptr(masks, i32, "masks"),
                   masks.shape[1] if masks is not None else 0, masks.shape[0] if masks is not None else 0,
                   _dev_ptr(mask_ids, i32, "mask_ids", n))
    with _ordered(ctx, z, out, ids, logp, lse, offset, given, bias_ids, bias, masks, mask_ids):
        _check(lib().kkm_choose(ctx, ctypes.byref(a), pout, ldo, _dev_ptr(ids, i32, "ids", n),
                                _dev_ptr(logp, f32, "logp", n), _dev_ptr(lse, f32, "lse", n)), ctx)


def kkm_check_adapted_args(adapted: kkm_adapted) -> int:
    return lib().kkm_check_adapted_args(ctypes.byref(adapted))


def kkm_check_newton_args(newton: kkm_newton, type_: int, batch: int, m: int, n: int) -> int:
    return lib().kkm_check_newton_args(ctypes.byref(newton), int(type_), int(batch), int(m), int(n))


def kkm_check_choice_args(choice: kkm_choice) -> int:
    return lib().kkm_check_choice_args(ctypes.byref(choice))


def kkm_check_norm_args(type_: int, n: int, d: int, ldx: int, wtype: int, eps: float) -> int:
    return lib().kkm_check_norm_args(int(type_), int(n), int(d), int(ldx), int(wtype), float(eps))


def kkm_check_head_args(head: kkm_head, teacher=None) -> int:
    return lib().kkm_check_head_args(ctypes.byref(head), ctypes.byref(teacher) if teacher is not None else None)


def kkm_get_stream(ctx) -> int:
    """hipStream_t of the context (0: the default stream)."""
    h = _vp()
    _check(lib().kkm_get_stream(ctx, ctypes.byref(h)), ctx)
    return h.value or 0
