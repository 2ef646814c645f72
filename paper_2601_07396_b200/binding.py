"""Thin ctypes binding of ``libsvdcache.so``: same names as ``include/svdcache.h``,
argument marshalling only (tensor -> raw pointer, current stream -> void*; for the 8-bit calls
and those for queries and keys by the extension ``_calls.*.so``).  Every step
of the path runs in the library's CUDA kernels; nothing here computes, and there is no
fallback: a missing library or a failing call raises.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os
from typing import NamedTuple, Optional, Tuple

import torch

from .build import calls_path

F32, BF16, FP8 = 0, 1, 2
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}

_HERE = os.path.dirname(os.path.abspath(__file__))
# SVDCACHE_LIBRARY names another build of the same library (e.g. one made with different
# compiler flags); by default the in-tree build next to this file is loaded.
LIB_PATH = os.environ.get("SVDCACHE_LIBRARY") or os.path.join(_HERE, "libsvdcache.so")
_lib = None

_vp, _i64, _ci, _sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
_szp = ctypes.POINTER(ctypes.c_size_t)

# name -> (restype, argtypes); mirrors include/svdcache.h declaration by declaration
SIGNATURES = {
    "svdcache_status_string": (ctypes.c_char_p, [_ci]),
    "svdcache_last_cuda_error": (ctypes.c_char_p, []),
    "svdcache_calibrate_workspace_bytes": (_ci, [_ci, _ci, _szp]),
    "svdcache_calibrate_begin": (_ci, [_ci, _ci, _vp, _sz, _vp]),
    "svdcache_calibrate_accumulate": (_ci, [_vp, _i64, _ci, _i64, _ci, _vp, _sz, _vp]),
    "svdcache_calibrate_finish": (_ci, [_ci, _ci, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "svdcache_calibrate": (_ci, [_vp, _i64, _ci, _i64, _ci, _ci, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "svdcache_calibrate_noalloc": (_ci, [_vp, _i64, _ci, _i64, _ci, _ci, _vp, _vp, _vp, _vp, _vp]),
    "svdcache_rank_for_energy": (_ci, [_vp, _ci, ctypes.c_double, ctypes.c_double, ctypes.POINTER(_ci)]),
    "svdcache_basis_bytes": (_ci, [_ci, _ci, _ci, _szp]),
    "svdcache_basis_layout": (_ci, [_ci, _ci, _ci, _szp, _szp, _szp, _szp]),
    "svdcache_basis_prepare": (_ci, [_vp, _ci, _ci, _ci, _vp, _sz, _vp]),
    "svdcache_state_bytes": (_ci, [_i64, _ci, _ci, _ci, _szp]),
    "svdcache_state_layout": (_ci, [_i64, _ci, _ci, _ci, _szp, _szp]),
    "svdcache_state_reset": (_ci, [_vp, _i64, _ci, _ci, _ci, _vp]),
    "svdcache_state_query": (_ci, [_vp, _vp, ctypes.POINTER(_i64), ctypes.POINTER(_ci)]),
    "svdcache_full_step": (_ci, [_vp, _i64, _vp, _vp, _vp, _i64, _ci, _ci, _ci, ctypes.c_float, _vp]),
    "svdcache_cached_step": (_ci, [_vp, _vp, _vp, _i64, _i64, _ci, _ci, _ci, _ci, _vp]),
    "svdcache_full_step_batched": (_ci, [_ci, _vp, _i64, _sz, _vp, _sz, _vp, _sz, _vp, _sz, _i64, _ci, _ci,
                                         _ci, ctypes.c_float, _vp]),
    "svdcache_cached_step_batched": (_ci, [_ci, _vp, _sz, _vp, _sz, _vp, _i64, _sz, _i64, _ci, _ci, _ci,
                                           _ci, _vp]),
    "svdcache_kernel_launches": (ctypes.c_uint64, []),
    "svdcache_set_path": (_ci, [_ci]),
    "svdcache_last_path": (_ci, []),
    "svdcache_selftest_wait_timeout": (_ci, [_vp, _i64, _vp]),
    "svdcache_full_step_ranked_batched": (_ci, [_ci, _vp, _i64, _sz, _vp, _sz, _vp, _sz, _vp, _sz, _i64, _ci,
                                                ctypes.POINTER(_ci), _ci, ctypes.c_float, _vp]),
    "svdcache_cached_step_ranked_batched": (_ci, [_ci, _vp, _sz, _vp, _sz, _vp, _i64, _sz, _i64, _ci,
                                                  ctypes.POINTER(_ci), _ci, _ci, _vp]),
    "svdcache_forecast_weights": (_ci, [_ci, _ci, _ci, _ci, ctypes.POINTER(ctypes.c_double)]),
    "svdcache_forecast_bytes": (_ci, [_i64, _ci, _szp]),
    "svdcache_cached_step_forecast_batched": (_ci, [_ci, _vp, _sz, _vp, _sz, _vp, _i64, _sz, _i64, _ci, _ci, _ci,
                                                    ctypes.POINTER(_vp), _sz, _ci, _ci, _ci, _ci, _vp, _sz, _vp]),
    "svdcache_full_step_residual_ema_batched": (_ci, [_ci, _vp, _i64, _sz, _vp, _sz, _vp, _sz, _vp, _sz, _i64, _ci,
                                                      _ci, _ci, ctypes.c_float, ctypes.c_float, _vp]),
    "svdcache_calibrate_gram_region": (_ci, [_ci, _szp, _szp]),
    "svdcache_basis_similarity": (_ci, [_vp, _vp, _vp, _vp, _ci, _ci, _vp, ctypes.POINTER(ctypes.c_double), _vp]),
    "svdcache_singular_values": (_ci, [_vp, _ci, _vp, _vp]),
    "svdcache_left_factors": (_ci, [_vp, _vp, _i64, _ci, _vp, _vp]),
    "svdcache_fp8_scale_bytes": (_ci, [_i64, _ci, _szp]),
    "svdcache_quantize_fp8": (_ci, [_vp, _i64, _ci, _i64, _ci, _ci, _vp, _i64, _vp, _vp]),
    "svdcache_residual_rmsnorm_fp8": (_ci, [_vp, _i64, _vp, _i64, _vp, _i64, _vp, ctypes.c_float, _vp, _i64, _vp, _i64,
                                            _ci, _ci, _vp]),
    "svdcache_gemm_fp8_status_word": (_ci, [ctypes.POINTER(_vp)]),
    "svdcache_gemm_fp8_status_query": (_ci, [ctypes.POINTER(ctypes.c_int32)]),
    "svdcache_gemm_fp8": (_ci, [_vp, _i64, _vp, _vp, _i64, _vp, _vp, _ci, _vp, _i64, _ci, _vp, _i64, _ci, _ci, _vp, _vp]),
    "svdcache_gemm_fp8_plan": (_ci, [_i64, _ci, _ci, _i64, _i64, _ci, _vp]),
    "svdcache_selftest_gemm_fp8": (_ci, [_vp, _i64, _vp, _vp, _i64, _vp, _vp, _ci, _vp, _i64, _ci, _vp, _i64, _ci, _ci, _vp, _vp, _i64, _vp]),
    "svdcache_adapters_workspace_bytes": (_ci, [_i64, _ci, _ci, _szp]),
    "svdcache_gemm_fp8_adapters": (_ci, [_vp, _i64, _vp, _vp, _i64, _vp, _vp, _ci, _vp, _i64, _ci, _vp, _i64, _ci, _ci, _vp, _vp, _vp, _ci, _vp, _sz,
                                         _vp, _vp]),
    "svdcache_selftest_gemm_fp8_adapters": (_ci, [_vp, _i64, _vp, _vp, _i64, _vp, _vp, _ci, _vp, _i64, _ci, _vp, _i64, _ci, _ci, _vp, _vp, _vp, _ci,
                                                  _vp, _sz, _vp, _vp, _i64, _vp]),
    "svdcache_selftest_adapters_sizes": (_ci, [_i64, _ci, _ci, _ci, _ci, _ci, _vp, _ci, _ci, _vp]),
    "svdcache_selftest_adapters_slots": (_ci, [_vp, _vp, _ci, _i64, _i64, _ci, _ci, _vp, _vp, _vp, _vp]),
    "svdcache_adapter_load": (_ci, [_vp, _ci, _vp, _i64, _vp, _i64, _ci, ctypes.c_float, _ci, _ci, _ci, _vp]),
    "svdcache_rotary_table": (_ci, [_vp, _i64, _i64, _ci, _ci, _vp, _vp, _vp, _i64, _vp]),
    "svdcache_rotary": (_ci, [_vp, _vp, _i64, _i64, _ci, _ci, _vp, _vp]),
    "svdcache_qk_rmsnorm_rotary": (_ci, [_vp, _vp, _vp, _vp, _vp, _vp, ctypes.c_float, _i64, _i64, _ci, _ci, _vp, _vp]),
}


class SvdCacheError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        text = lib().svdcache_status_string(code).decode()
        extra = ""
        if code == -7:
            extra = " [" + lib().svdcache_last_cuda_error().decode() + "]"
        super().__init__(f"{where}: {text} ({code}){extra}")


def lib():
    """Load the CUDA library (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2601_07396_b200.build` "
                "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(code: int, where: str) -> None:
    if code != 0:
        raise SvdCacheError(code, where)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _dt(t_or_dtype) -> int:
    d = t_or_dtype.dtype if isinstance(t_or_dtype, torch.Tensor) else t_or_dtype
    return _DTYPES[d]


def _bytes_buffer(nbytes: int, device) -> torch.Tensor:
    # torch's caching allocator hands out 512-byte aligned blocks
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


# ------------------------------------------------------------------ size queries ---

def svdcache_calibrate_workspace_bytes(D: int, k: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().svdcache_calibrate_workspace_bytes(D, k, ctypes.byref(out)), "calibrate_workspace_bytes")
    return out.value


def svdcache_basis_bytes(D: int, k: int, dtype: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().svdcache_basis_bytes(D, k, dtype, ctypes.byref(out)), "basis_bytes")
    return out.value


def svdcache_basis_layout(D: int, k: int, dtype: int) -> Tuple[int, int, int, int]:
    o = [ctypes.c_size_t(0) for _ in range(4)]
    _check(lib().svdcache_basis_layout(D, k, dtype, *[ctypes.byref(x) for x in o]), "basis_layout")
    return tuple(x.value for x in o)


def svdcache_state_bytes(N: int, D: int, k: int, dtype: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().svdcache_state_bytes(N, D, k, dtype, ctypes.byref(out)), "state_bytes")
    return out.value


def svdcache_state_layout(N: int, D: int, k: int, dtype: int) -> Tuple[int, int]:
    a, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(lib().svdcache_state_layout(N, D, k, dtype, ctypes.byref(a), ctypes.byref(b)), "state_layout")
    return a.value, b.value


# ------------------------------------------------------------------- calibration ---

def svdcache_calibrate_begin(D: int, k: int, workspace: torch.Tensor, stream=None) -> None:
    _check(lib().svdcache_calibrate_begin(D, k, _ptr(workspace), workspace.numel(), _stream(stream)),
           "calibrate_begin")


def svdcache_calibrate_accumulate(F: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    M, D = F.shape
    assert F.stride(1) == 1
    _check(lib().svdcache_calibrate_accumulate(_ptr(F), M, D, F.stride(0), _dt(F), _ptr(workspace),
                                               workspace.numel(), _stream(stream)), "calibrate_accumulate")


def svdcache_calibrate_finish(D: int, k: int, workspace: torch.Tensor, stream=None, strict: bool = True):
    """Returns (Vk [D x k] fp32, lambda [k] fp64, trace [1] fp64, info list) on the device."""
    dev = workspace.device
    Vk = torch.empty(D, k, dtype=torch.float32, device=dev)
    lam = torch.empty(k, dtype=torch.float64, device=dev)
    tr = torch.empty(1, dtype=torch.float64, device=dev)
    info = (ctypes.c_double * 4)()
    rc = lib().svdcache_calibrate_finish(D, k, _ptr(Vk), _ptr(lam), _ptr(tr), ctypes.cast(info, _vp),
                                         _ptr(workspace), workspace.numel(), _stream(stream))
    if rc != 0 and (strict or rc != -8):
        raise SvdCacheError(rc, "calibrate_finish")
    return Vk, lam, tr, list(info)


def svdcache_calibrate(Fstack: torch.Tensor, k: int, workspace: Optional[torch.Tensor] = None,
                       stream=None, strict: bool = True):
    """One-shot calibration of a device stack (M x D).  Returns (Vk, lambda, trace, info)."""
    M, D = Fstack.shape
    assert Fstack.stride(1) == 1
    if workspace is None:
        workspace = _bytes_buffer(svdcache_calibrate_workspace_bytes(D, k), Fstack.device)
    dev = Fstack.device
    Vk = torch.empty(D, k, dtype=torch.float32, device=dev)
    lam = torch.empty(k, dtype=torch.float64, device=dev)
    tr = torch.empty(1, dtype=torch.float64, device=dev)
    info = (ctypes.c_double * 4)()
    rc = lib().svdcache_calibrate(_ptr(Fstack), M, D, Fstack.stride(0), _dt(Fstack), k, _ptr(Vk), _ptr(lam),
                                  _ptr(tr), ctypes.cast(info, _vp), _ptr(workspace), workspace.numel(),
                                  _stream(stream))
    if rc != 0 and (strict or rc != -8):
        raise SvdCacheError(rc, "calibrate")
    return Vk, lam, tr, list(info)


BUILTIN_SCRATCH_BYTES = 4 << 20


def svdcache_calibrate_noalloc(Fstack: torch.Tensor, k: int, Vk: torch.Tensor, lam: torch.Tensor,
                               tr: torch.Tensor, stream=None, strict: bool = True):
    """Calibration on the library's built-in scratch, for callers that may not allocate
    device memory: the outputs (Vk [D x k] fp32, lam [k] fp64, tr [1] fp64) are passed in,
    and neither this wrapper nor the call behind it allocates anything on the device.
    Returns the info list."""
    M, D = Fstack.shape
    assert Fstack.stride(1) == 1 and Vk.shape == (D, k) and Vk.dtype == torch.float32 and Vk.is_contiguous()
    info = (ctypes.c_double * 4)()
    rc = lib().svdcache_calibrate_noalloc(_ptr(Fstack), M, D, Fstack.stride(0), _dt(Fstack), k, _ptr(Vk),
                                          _ptr(lam), _ptr(tr), ctypes.cast(info, _vp), _stream(stream))
    if rc != 0 and (strict or rc != -8):
        raise SvdCacheError(rc, "calibrate_noalloc")
    return list(info)


def svdcache_rank_for_energy(lam, trace: float, tau: float) -> int:
    arr = (ctypes.c_double * len(lam))(*[float(x) for x in lam])
    out = ctypes.c_int(0)
    _check(lib().svdcache_rank_for_energy(ctypes.cast(arr, _vp), len(lam), float(trace), float(tau),
                                          ctypes.byref(out)), "rank_for_energy")
    return out.value


# ------------------------------------------------------------------ basis, state ---

def svdcache_basis_prepare(Vk: torch.Tensor, dtype: int, basis: Optional[torch.Tensor] = None,
                           stream=None) -> torch.Tensor:
    D, k = Vk.shape
    assert Vk.dtype == torch.float32 and Vk.is_contiguous()
    if basis is None:
        basis = _bytes_buffer(svdcache_basis_bytes(D, k, dtype), Vk.device)
    _check(lib().svdcache_basis_prepare(_ptr(Vk), D, k, dtype, _ptr(basis), basis.numel(), _stream(stream)),
           "basis_prepare")
    return basis


def svdcache_state_reset(state: torch.Tensor, N: int, D: int, k: int, dtype: int, stream=None) -> None:
    _check(lib().svdcache_state_reset(_ptr(state), N, D, k, dtype, _stream(stream)), "state_reset")


def svdcache_state_query(state: torch.Tensor, stream=None) -> Tuple[int, int]:
    steps, status = ctypes.c_int64(0), ctypes.c_int(0)
    _check(lib().svdcache_state_query(_ptr(state), _stream(stream), ctypes.byref(steps), ctypes.byref(status)),
           "state_query")
    return steps.value, status.value


# ------------------------------------------------------------------------- steps ---

def svdcache_full_step(F: torch.Tensor, basis: torch.Tensor, state: torch.Tensor, k: int, beta: float,
                       C_out: Optional[torch.Tensor] = None, stream=None) -> None:
    N, D = F.shape
    assert F.stride(1) == 1
    _check(lib().svdcache_full_step(_ptr(F), F.stride(0), _ptr(basis), _ptr(state), _ptr(C_out), N, D, k,
                                    _dt(F), float(beta), _stream(stream)), "full_step")


def svdcache_cached_step(state: torch.Tensor, basis: torch.Tensor, Fhat: torch.Tensor, k: int,
                         steps_since_full: int = 1, stream=None) -> None:
    N, D = Fhat.shape
    assert Fhat.stride(1) == 1
    _check(lib().svdcache_cached_step(_ptr(state), _ptr(basis), _ptr(Fhat), Fhat.stride(0), N, D, k,
                                      _dt(Fhat), int(steps_since_full), _stream(stream)), "cached_step")


def svdcache_full_step_batched(F: torch.Tensor, basis: torch.Tensor, state: torch.Tensor, k: int,
                               beta: float, C_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """F: [blocks, N, D]; basis, state: [blocks, bytes] uint8; C_out: [blocks, N, k] or None."""
    nb, N, D = F.shape
    assert F.stride(2) == 1
    eb = F.element_size()
    _check(lib().svdcache_full_step_batched(
        nb, _ptr(F), F.stride(1), F.stride(0) * eb, _ptr(basis), basis.stride(0), _ptr(state),
        state.stride(0), _ptr(C_out), 0 if C_out is None else C_out.stride(0) * 4, N, D, k, _dt(F),
        float(beta), _stream(stream)), "full_step_batched")


def svdcache_cached_step_batched(state: torch.Tensor, basis: torch.Tensor, Fhat: torch.Tensor, k: int,
                                 steps_since_full: int = 1, stream=None) -> None:
    nb, N, D = Fhat.shape
    assert Fhat.stride(2) == 1
    eb = Fhat.element_size()
    _check(lib().svdcache_cached_step_batched(
        nb, _ptr(state), state.stride(0), _ptr(basis), basis.stride(0), _ptr(Fhat), Fhat.stride(1),
        Fhat.stride(0) * eb, N, D, k, _dt(Fhat), int(steps_since_full), _stream(stream)), "cached_step_batched")


def svdcache_kernel_launches() -> int:
    return int(lib().svdcache_kernel_launches())


def svdcache_set_path(path: int) -> int:
    return int(lib().svdcache_set_path(path))


def svdcache_last_path() -> int:
    return int(lib().svdcache_last_path())


def svdcache_selftest_wait_timeout(state: torch.Tensor, limit_cycles: int, stream=None) -> None:
    _check(lib().svdcache_selftest_wait_timeout(_ptr(state), int(limit_cycles), _stream(stream)), "selftest_wait_timeout")


PREDICT_EMA, PREDICT_TAYLOR, PREDICT_NEWTON = 0, 1, 2


def svdcache_forecast_weights(predictor: int, order: int, steps_since_full: int, interval: int):
    w = (ctypes.c_double * (order + 1))()
    _check(lib().svdcache_forecast_weights(predictor, order, steps_since_full, interval, w), "forecast_weights")
    return list(w)


def svdcache_forecast_bytes(N: int, k: int) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().svdcache_forecast_bytes(N, k, ctypes.byref(out)), "forecast_bytes")
    return int(out.value)


def svdcache_cached_step_forecast_batched(state: torch.Tensor, basis: torch.Tensor, Fhat: torch.Tensor, k: int, history,
                                  predictor: int, steps_since_full: int, interval: int, forecast=None, stream=None):
    """Cached step with the coefficients forecast from `history` (list of N x k fp32 device tensors --
    or [blocks, N, k] for a batched Fhat [blocks, N, D] -- newest first; its length - 1 is the order).
    Returns the forecast buffer (allocated here unless given)."""
    batched = Fhat.dim() == 3
    nb = Fhat.shape[0] if batched else 1
    N, D = Fhat.shape[-2:]
    assert Fhat.stride(-1) == 1
    order = len(history) - 1
    fbytes = svdcache_forecast_bytes(N, k)
    if forecast is None:
        forecast = torch.empty(nb, fbytes, dtype=torch.uint8, device=Fhat.device) if batched else _bytes_buffer(fbytes, Fhat.device)
    ptrs = (_vp * (order + 1))(*[_ptr(h) for h in history])
    eb = Fhat.element_size()
    _check(lib().svdcache_cached_step_forecast_batched(
        nb, _ptr(state), state.stride(0) if batched else 0, _ptr(basis), basis.stride(0) if batched else 0, _ptr(Fhat),
        Fhat.stride(-2), Fhat.stride(0) * eb if batched else 0, N, D, k, _dt(Fhat), ptrs,
        history[0].stride(0) * 4 if batched else 0, predictor, order, int(steps_since_full), int(interval), _ptr(forecast),
        forecast.stride(0) if batched else 0, _stream(stream)), "cached_step_forecast")
    return forecast


def svdcache_full_step_residual_ema_batched(F: torch.Tensor, basis: torch.Tensor, state: torch.Tensor, k: int, beta: float,
                                    beta_r: float, C_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """Full step whose stored residual is an EMA of the residuals (ablation); F is [N, D] or [blocks, N, D]."""
    batched = F.dim() == 3
    nb = F.shape[0] if batched else 1
    N, D = F.shape[-2:]
    eb = F.element_size()
    _check(lib().svdcache_full_step_residual_ema_batched(
        nb, _ptr(F), F.stride(-2), F.stride(0) * eb if batched else 0, _ptr(basis), basis.stride(0) if batched else 0,
        _ptr(state), state.stride(0) if batched else 0, _ptr(C_out) if C_out is not None else None,
        C_out.stride(0) * 4 if (batched and C_out is not None) else 0, N, D, k, _dt(F), float(beta), float(beta_r),
        _stream(stream)), "full_step_residual_ema")


def svdcache_full_step_ranked_batched(F: torch.Tensor, bases: torch.Tensor, states: torch.Tensor, ranks, beta: float,
                              C_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """Batched full step over blocks of different rank: F [blocks, N, D], bases / states [blocks, bytes]
    (each block's buffer laid out for its own rank), C_out [blocks, N, kmax] (row b*... holds N x k_b dense)."""
    nb, N, D = F.shape
    arr = (_ci * nb)(*[int(r) for r in ranks])
    _check(lib().svdcache_full_step_ranked_batched(
        nb, _ptr(F), F.stride(1), F.stride(0) * F.element_size(), _ptr(bases), bases.stride(0), _ptr(states),
        states.stride(0), _ptr(C_out) if C_out is not None else None, C_out.stride(0) * 4 if C_out is not None else 0,
        N, D, arr, _dt(F), float(beta), _stream(stream)), "full_step_ranked")


def svdcache_cached_step_ranked_batched(states: torch.Tensor, bases: torch.Tensor, Fhat: torch.Tensor, ranks,
                                steps_since_full: int = 1, stream=None) -> None:
    nb, N, D = Fhat.shape
    arr = (_ci * nb)(*[int(r) for r in ranks])
    _check(lib().svdcache_cached_step_ranked_batched(
        nb, _ptr(states), states.stride(0), _ptr(bases), bases.stride(0), _ptr(Fhat), Fhat.stride(1),
        Fhat.stride(0) * Fhat.element_size(), N, D, arr, _dt(Fhat), int(steps_since_full), _stream(stream)),
        "cached_step_ranked")


def svdcache_calibrate_gram_region(D: int):
    off, nbytes = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(lib().svdcache_calibrate_gram_region(D, ctypes.byref(off), ctypes.byref(nbytes)), "calibrate_gram_region")
    return int(off.value), int(nbytes.value)


def svdcache_basis_similarity(VkA: torch.Tensor, lamA: torch.Tensor, VkB: torch.Tensor, lamB: torch.Tensor, stream=None):
    """(similarity of the singular values, mean similarity of the right singular vectors, per-column |cos|)."""
    D, k = VkA.shape
    assert VkB.shape == (D, k) and VkA.is_contiguous() and VkB.is_contiguous()
    cols = torch.empty(k, dtype=torch.float64, device=VkA.device)
    out = (ctypes.c_double * 2)()
    _check(lib().svdcache_basis_similarity(_ptr(VkA), _ptr(lamA), _ptr(VkB), _ptr(lamB), D, k, _ptr(cols), out,
                                           _stream(stream)), "basis_similarity")
    return float(out[0]), float(out[1]), cols


def svdcache_singular_values(lam: torch.Tensor, stream=None) -> torch.Tensor:
    sigma = torch.empty_like(lam)
    _check(lib().svdcache_singular_values(_ptr(lam), lam.numel(), _ptr(sigma), _stream(stream)), "singular_values")
    return sigma


def svdcache_left_factors(C: torch.Tensor, sigma: torch.Tensor, stream=None) -> torch.Tensor:
    N, k = C.shape
    assert C.is_contiguous() and C.dtype == torch.float32 and sigma.dtype == torch.float64
    U = torch.empty_like(C)
    _check(lib().svdcache_left_factors(_ptr(C), _ptr(sigma), N, k, _ptr(U), _stream(stream)), "left_factors")
    return U


# ------------------------------------------------------------- 8-bit linear path ---

ACT_NONE, ACT_GELU = 0, 1


def svdcache_fp8_scale_bytes(rows: int, cols: int) -> int:
    out = ctypes.c_size_t(0)
    if not (0 <= rows < 1 << 31 and 0 <= cols < 1 << 31):   # ctypes would cut them to their low bits
        raise SvdCacheError(-2, "fp8_scale_bytes")
    _check(lib().svdcache_fp8_scale_bytes(rows, cols, ctypes.byref(out)), "fp8_scale_bytes")
    return out.value


# The calls below can be shorter on the GPU than a binding in Python is on the host, so their arguments are read and
# checked by a small extension (csrc/calls.cpp), which calls the same C entry points.  It raises ValueError for
# arguments that the C ABI cannot see to be wrong (types, shapes against one another, device, contiguity).  The values of an
# 8-bit matrix are uint8 or float8_e4m3fn tensors, its scales uint8 or float8_e8m0fnu.
_calls = None


def calls():
    """Load the extension (once) and bind it to the library.  Raises if it has not been built."""
    global _calls
    if _calls is None:
        path = calls_path()
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with `python -m paper_2601_07396_b200.build`")
        loader = importlib.machinery.ExtensionFileLoader("_calls", path)
        module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_calls", loader))
        loader.exec_module(module)
        L = lib()
        module.bind(*[ctypes.cast(f, _vp).value for f in (L.svdcache_quantize_fp8, L.svdcache_residual_rmsnorm_fp8, L.svdcache_gemm_fp8,
                                                            L.svdcache_gemm_fp8_status_word, L.svdcache_rotary_table, L.svdcache_rotary,
                                                            L.svdcache_qk_rmsnorm_rotary, L.svdcache_gemm_fp8_adapters,
                                                            L.svdcache_adapter_load)])
        _calls = module
    return _calls


def svdcache_quantize_fp8(X: torch.Tensor, Q: torch.Tensor, S: torch.Tensor, tile_rows: int = 1, stream=None) -> None:
    """X [rows, cols] fp32 or bf16 -> e4m3 bytes Q [rows, >= cols] and their scales S (see new_fp8); one scale per
    1 x 128 group, or with tile_rows = 128 per 128 x 128 tile."""
    rc = (_calls or calls()).quantize(X, Q, S, tile_rows, None if stream is None else stream.cuda_stream)
    if rc:
        raise SvdCacheError(rc, "quantize_fp8")


def svdcache_residual_rmsnorm_fp8(H: torch.Tensor, X: Optional[torch.Tensor], H_out: Optional[torch.Tensor],
                                  weight: Optional[torch.Tensor], eps: float, Q: torch.Tensor, S: torch.Tensor,
                                  stream=None) -> None:
    """h = H + X (X None: h = H) -> H_out (None: not kept; H itself: in place); RMS norm of h times weight [D] fp32
    (None: ones) as an 8-bit matrix Q, S."""
    rc = (_calls or calls()).norm(H, X, H_out, weight, eps, Q, S, None if stream is None else stream.cuda_stream)
    if rc:
        raise SvdCacheError(rc, "residual_rmsnorm_fp8")


def svdcache_gemm_fp8(A: torch.Tensor, SA: torch.Tensor, B: torch.Tensor, SB: torch.Tensor, K: int, C: torch.Tensor,
                      S_out: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, act: int = ACT_NONE,
                      status: Optional[torch.Tensor] = None, stream=None) -> None:
    """C [M, N] = act(A B^T + bias) of the 8-bit matrices A [M, >= K] and B [N, >= K].  C is fp32 or bf16, or bytes
    (uint8, float8_e4m3fn) with scales S_out.  `status`: an int32 tensor on the device, whose first element
    receives a time-out; by default the library's own on that device, which gemm_status() reads."""
    rc = (_calls or calls()).gemm(A, SA, B, SB, K, C, S_out, bias, act, status, None if stream is None else stream.cuda_stream)
    if rc:
        raise SvdCacheError(rc, "gemm_fp8")


def svdcache_gemm_fp8_plan(M: int, N: int, K: int, out: int, lda: Optional[int] = None, ldb: Optional[int] = None) -> Tuple[int, int, int, int]:
    """How a product into the type `out` is taken on the current device: (pairs, size of the tiles, CTAs per tile, tiles that
    follow one another on an SM at most).  lda, ldb: pitches, by default K up to a multiple of 16."""
    plan = (ctypes.c_int32 * 4)()
    pitch = -(-K // 16) * 16
    _check(lib().svdcache_gemm_fp8_plan(M, N, K, lda or pitch, ldb or pitch, out, plan), "gemm_fp8_plan")
    return tuple(plan)


def svdcache_selftest_gemm_fp8(A: torch.Tensor, SA: torch.Tensor, B: torch.Tensor, SB: torch.Tensor, K: int, C: torch.Tensor, plan,
                               S_out: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, act: int = ACT_NONE,
                               status: Optional[torch.Tensor] = None, limit_cycles: int = 0, stream=None) -> None:
    """svdcache_gemm_fp8 by the given plan (pairs, size of the tiles, CTAs per tile), which has to be one that the product may
    be taken by.  limit_cycles > 0: nothing is loaded and the kernel's waits run out after so many cycles.  For tests: of the
    tensors only what the C ABI sees is checked."""
    (M, N), out = C.shape, _DTYPES.get(C.dtype, FP8)
    words = (ctypes.c_int32 * 3)(*plan[:3])
    pitch = lambda t: t.stride(0) if t.shape[0] > 1 else -(-t.shape[1] // 16) * 16  # noqa: E731
    with torch.cuda.device(C.device):
        word = _ptr(status) if status is not None else svdcache_gemm_fp8_status_word()
        _check(lib().svdcache_selftest_gemm_fp8(_ptr(A), pitch(A), _ptr(SA), _ptr(B), pitch(B), _ptr(SB), _ptr(bias), act, _ptr(C), pitch(C), out,
                                                _ptr(S_out), M, N, K, word, words, limit_cycles, _stream(stream)),
               "selftest_gemm_fp8")


def svdcache_gemm_fp8_status_word() -> int:
    """The address of the current device's default status word."""
    out = _vp()
    _check(lib().svdcache_gemm_fp8_status_word(ctypes.byref(out)), "gemm_fp8_status_word")
    return out.value


def svdcache_gemm_fp8_status_query() -> int:
    """The current device's default status word, once all work of the device is done."""
    out = ctypes.c_int32(0)
    _check(lib().svdcache_gemm_fp8_status_query(ctypes.byref(out)), "gemm_fp8_status_query")
    return out.value


def gemm_status(device="cuda") -> int:
    """The sticky status of the products on `device` that were given no status word (synchronises): 0, or -6 if a
    bounded wait ran out in one of them."""
    with torch.cuda.device(device):
        return svdcache_gemm_fp8_status_query()


def new_fp8(rows: int, cols: int, device="cuda"):
    """Allocate (torch) an 8-bit matrix: bytes [rows, cols up to a multiple of 16] and its scale buffer, zeroed."""
    q = torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.uint8, device=device)
    return q, torch.zeros(svdcache_fp8_scale_bytes(rows, cols), dtype=torch.uint8, device=device)


def fp8_scale_exponents(S: torch.Tensor, rows: int, cols: int) -> torch.Tensor:
    """The scale bytes of a buffer as [rows, groups of 128 columns] (a copy); scale = 2^(byte - 127)."""
    i, j, g = -(-rows // 128), -(-cols // 512), -(-cols // 128)
    pieces = S.view(torch.uint8).reshape(-1)[:i * j * 512].view(i, j, 32, 4, 4)
    return pieces.permute(0, 3, 2, 1, 4).reshape(128 * i, 4 * j)[:rows, :g]


# ------------------------------------------------- adapters beside a projection ---

class Adapters(NamedTuple):
    """A pool of low-rank adapters for one projection of K columns to N (new_adapters): adapter a adds
    factor[a] * (x down[a]^T) up[a]^T to the rows of the requests that use it."""
    down: torch.Tensor          # [count, rank, K up to a multiple of 16] e4m3 bytes, rank a multiple of 8 up to 128
    down_scales: torch.Tensor   # [count, bytes] the scales of each
    up: torch.Tensor            # [count, N, rank] bf16, every value finite
    factor: torch.Tensor        # [count] fp32


def new_adapters(count: int, rank: int, N: int, K: int, device="cuda") -> Adapters:
    """Allocate (torch) a pool for adapters up to the given rank, all of them zero."""
    rank = -(-rank // 8) * 8
    return Adapters(torch.zeros(count, rank, -(-K // 16) * 16, dtype=torch.uint8, device=device),
                    torch.zeros(count, svdcache_fp8_scale_bytes(rank, K), dtype=torch.uint8, device=device),
                    torch.zeros(count, N, rank, dtype=torch.bfloat16, device=device), torch.zeros(count, device=device))


def svdcache_adapter_load(adapters: Adapters, index: int, down: torch.Tensor, up: torch.Tensor, factor: float = 1.0, stream=None) -> None:
    """Puts an adapter, down [r, K] and up [N, r] both fp32 or both bf16, into place `index` of a pool of rank r or more: down in 8 bits with
    a scale per 1 x 128 group (e4m3: x down^T is off by about 2.6 % of its norm), up in bf16.  If a value of up is not finite there, the factor becomes NaN, and with it every row
    that uses the adapter."""
    rc = (_calls or calls()).adapter_load(*adapters, index, down, up, factor, None if stream is None else stream.cuda_stream)
    if rc:
        raise SvdCacheError(rc, "adapter_load")


def svdcache_adapters_workspace_bytes(M: int, rank: int, requests: int) -> int:
    out = ctypes.c_size_t(0)
    if not (0 <= M < 1 << 31 and 0 <= rank < 1 << 31 and 0 <= requests < 1 << 31):   # ctypes would cut them to their low bits
        raise SvdCacheError(-2, "adapters_workspace_bytes")
    _check(lib().svdcache_adapters_workspace_bytes(M, rank, requests, ctypes.byref(out)), "adapters_workspace_bytes")
    return out.value


def new_adapters_workspace(M: int, rank: int, requests: int, device="cuda") -> torch.Tensor:
    """Allocate (torch) the workspace of calls up to these sizes.  Calls that may run at the same time need one each."""
    return _bytes_buffer(svdcache_adapters_workspace_bytes(M, -(-rank // 8) * 8, requests), device)


def svdcache_gemm_fp8_adapters(A: torch.Tensor, SA: torch.Tensor, B: torch.Tensor, SB: torch.Tensor, K: int, C: torch.Tensor, adapters: Adapters,
                               row_start: torch.Tensor, adapter: torch.Tensor, workspace: torch.Tensor, S_out: Optional[torch.Tensor] = None,
                               bias: Optional[torch.Tensor] = None, act: int = ACT_NONE, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """svdcache_gemm_fp8 with the adapters' term under the activation: C = act(A B^T + bias + factor_a (A down_a^T) up_a^T).  Request i is
    the rows row_start[i] .. row_start[i + 1] - 1 with adapter[i] (-1: none); both are int32 on the device and are read when the
    call runs.  `workspace`: new_adapters_workspace(M, rank, requests)."""
    rc = (_calls or calls()).gemm_adapters(A, SA, B, SB, K, C, S_out, bias, act, status, None if stream is None else stream.cuda_stream, *adapters,
                                           row_start, adapter, workspace)
    if rc:
        raise SvdCacheError(rc, "gemm_fp8_adapters")


class _AdaptersStruct(ctypes.Structure):
    _fields_ = [("down", _vp), ("down_ld", _i64), ("down_stride", _i64), ("down_scales", _vp), ("scales_stride", _i64), ("up", _vp), ("up_ld", _i64),
                ("up_stride", _i64), ("factor", _vp), ("count", _ci), ("rank", _ci)]


def svdcache_selftest_gemm_fp8_adapters(A: torch.Tensor, SA: torch.Tensor, B: torch.Tensor, SB: torch.Tensor, K: int, C: torch.Tensor, adapters: Adapters,
                                        row_start: torch.Tensor, adapter: torch.Tensor, workspace: torch.Tensor, plan, S_out: Optional[torch.Tensor] = None,
                                        bias: Optional[torch.Tensor] = None, act: int = ACT_NONE, status: Optional[torch.Tensor] = None,
                                        limit_cycles: int = 0, stream=None) -> None:
    """svdcache_gemm_fp8_adapters with its projection by the given plan, as svdcache_selftest_gemm_fp8.  For tests: of the tensors only
    what the C ABI sees is checked."""
    (M, N), out = C.shape, _DTYPES.get(C.dtype, FP8)
    words = (ctypes.c_int32 * 3)(*plan[:3])
    pitch = lambda t: t.stride(0) if t.shape[0] > 1 else -(-t.shape[1] // 16) * 16  # noqa: E731
    d, s, u, f = adapters
    count, rank = d.shape[:2]
    up_ld = u.stride(1) if N > 1 else rank
    pool = _AdaptersStruct(d.data_ptr(), d.stride(1), d.stride(0) if count > 1 else d.stride(1) * rank, s.data_ptr(), s.stride(0) if count > 1 else -(-s.shape[1] // 16) * 16,
                           u.data_ptr(), up_ld, u.stride(0) if count > 1 else up_ld * N, f.data_ptr(), count, rank)
    with torch.cuda.device(C.device):
        word = _ptr(status) if status is not None else svdcache_gemm_fp8_status_word()
        _check(lib().svdcache_selftest_gemm_fp8_adapters(_ptr(A), pitch(A), _ptr(SA), _ptr(B), pitch(B), _ptr(SB), _ptr(bias), act, _ptr(C), pitch(C), out,
                                                         _ptr(S_out), M, N, K, ctypes.byref(pool), _ptr(row_start), _ptr(adapter), adapter.numel(),
                                                         _ptr(workspace), workspace.numel() * workspace.element_size(), word, words, limit_cycles,
                                                         _stream(stream)), "selftest_gemm_fp8_adapters")


def svdcache_selftest_adapters_sizes(M: int, N: int, K: int, rank: int, requests: int, out: int, plan, brief: bool, sms: int = 148):
    """(CTAs, CTAs of a cluster, columns of tensor memory, bytes of shared memory) of the narrow product's kernel and of the projection's."""
    out_words = (ctypes.c_int64 * 8)()
    _check(lib().svdcache_selftest_adapters_sizes(M, N, K, rank, requests, out, (ctypes.c_int32 * 3)(*plan[:3]), int(brief), sms, out_words), "selftest_adapters_sizes")
    return tuple(out_words[:4]), tuple(out_words[4:])


def svdcache_selftest_adapters_slots(row_start: torch.Tensor, adapter: torch.Tensor, M: int, count: int, tile_rows: int, first: int = 0):
    """(tasks, tiles, list, tile_list) that the kernels find for requests given as int32 tensors on the host; what they leave is -9."""
    n = adapter.numel()
    if row_start.dtype != torch.int32 or adapter.dtype != torch.int32 or row_start.is_cuda or adapter.is_cuda or row_start.numel() != n + 1:
        raise ValueError("row_start and adapter: int32 on the host, one row more than there are adapters")
    tiles = -(-M // tile_rows)
    out = [torch.full(shape, -9, dtype=torch.int32) for shape in ((tiles + n, 4), (tiles, 4), (tiles + n, 2), (tiles, 1 + 2 * tile_rows))]
    row_start, adapter = row_start.contiguous(), adapter.contiguous()
    _check(lib().svdcache_selftest_adapters_slots(row_start.data_ptr(), adapter.data_ptr(), n, first, M, count, tile_rows, *[t.data_ptr() for t in out]),
           "selftest_adapters_slots")
    return tuple(out)


# --------------------------------------------------------------- queries and keys ---
#
# Heads are tensors [tokens, heads, dim] or [batch, tokens, heads, dim], fp32 or bf16, with any strides but the last: views of a
# packed projection as they are, and for heads before tokens the transposed view.  Arguments are read as above.

def svdcache_rotary_table(positions: torch.Tensor, dims, bases, table: torch.Tensor, stream=None) -> None:
    """(cos, sin) of positions [tokens, axes] (int32, int64 or fp32) -> table [tokens, sum(dims) / 2, 2] fp32; axis a has dims[a]
    elements of a head, whose pair j turns by position * bases[a] ** (-2 j / dims[a])."""
    rc = (_calls or calls()).rotary_table(positions, dims, bases, table, None if stream is None else stream.cuda_stream)
    if rc:
        raise SvdCacheError(rc, "rotary_table")


def svdcache_rotary(X: torch.Tensor, table: torch.Tensor, out: torch.Tensor, first: int = 0, halves: bool = False, inverse: bool = False,
                    stream=None) -> None:
    """X -> out (X itself: in place), the pairs of the first r elements of each head turned by table [rows, r / 2, 2] (or one for
    each batch), whose rows belong to the tokens from `first` on; other tokens and elements pass.  Pairs are neighbours, or with
    `halves` elements i and i + r / 2.  `inverse` turns back: the gradient with respect to X of what was turned."""
    rc = (_calls or calls()).rotary(X, table, out, first, halves, inverse, None if stream is None else stream.cuda_stream)
    if rc:
        raise SvdCacheError(rc, "rotary")


def svdcache_qk_rmsnorm_rotary(Q: torch.Tensor, K: Optional[torch.Tensor], q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor],
                               eps: float, table: Optional[torch.Tensor], Q_out: torch.Tensor, K_out: Optional[torch.Tensor], first: int = 0,
                               halves: bool = False, stream=None) -> None:
    """RMS norm of each head of Q and K (their numbers of heads may differ; K None: Q alone) times a weight [dim] fp32 (None: ones),
    then the rotation of svdcache_rotary (table None: none) -> Q_out, K_out (the inputs themselves: in place)."""
    rc = (_calls or calls()).qk(Q, K, q_weight, k_weight, eps, table, Q_out, K_out, first, halves, None if stream is None else stream.cuda_stream)
    if rc:
        raise SvdCacheError(rc, "qk_rmsnorm_rotary")


# ---------------------------------------------------------- views for tests/tools ---

def new_state(N: int, D: int, k: int, dtype: int, device="cuda", blocks: int = 0) -> torch.Tensor:
    """Allocate (torch) and reset a state buffer; ``blocks`` > 0 gives [blocks, bytes]."""
    nbytes = svdcache_state_bytes(N, D, k, dtype)
    if blocks:
        st = torch.empty(blocks, nbytes, dtype=torch.uint8, device=device)
        for b in range(blocks):
            svdcache_state_reset(st[b], N, D, k, dtype)
        return st
    st = _bytes_buffer(nbytes, device)
    svdcache_state_reset(st, N, D, k, dtype)
    return st


def state_views(state: torch.Tensor, N: int, D: int, k: int, dtype: int):
    """(Chat [N x k] fp32, R [N x D]) views into one block's state buffer."""
    co, ro = svdcache_state_layout(N, D, k, dtype)
    tdt = torch.float32 if dtype == F32 else torch.bfloat16
    eb = 4 if dtype == F32 else 2
    chat = state[co:co + N * k * 4].view(torch.float32).view(N, k)
    r = state[ro:ro + N * D * eb].view(tdt).view(N, D)
    return chat, r


def basis_views(basis: torch.Tensor, D: int, k: int, dtype: int):
    """(V fp32, V^T fp32, V bf16 | None, V^T bf16 | None) views into a basis buffer."""
    a, b, c, d = svdcache_basis_layout(D, k, dtype)
    v32 = basis[a:a + D * k * 4].view(torch.float32).view(D, k)
    vt32 = basis[b:b + D * k * 4].view(torch.float32).view(k, D)
    if dtype == BF16:
        v16 = basis[c:c + D * k * 2].view(torch.bfloat16).view(D, k)
        vt16 = basis[d:d + D * k * 2].view(torch.bfloat16).view(k, D)
        return v32, vt32, v16, vt16
    return v32, vt32, None, None
