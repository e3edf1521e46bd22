"""Binding of libdab_hip.so: argument marshalling only.

Every function here has the name of the C entry point it calls (see
``include/dab.h``) and does nothing but check tensor dtype / device /
contiguity, allocate the output tensors with ``torch.empty`` and pass raw
device pointers plus the current HIP stream.  The calls of single layers do that
in native code (``csrc/binding_call.cpp``, the module ``_dab_call``), plain ones whole,
others from the Python below on; the grouped
calls, whose jobs are marshalled once and kept, go through ctypes.  All arithmetic
of the path runs in the HIP kernels.  There is no CPU fallback: if the library is
not built, or a tensor is not on the GPU, the call raises.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import c_char_p, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_uint64, c_void_p

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdab_hip.so")

DAB_OK = 0
DAB_ERR_NULL, DAB_ERR_SHAPE, DAB_ERR_ALIGN, DAB_ERR_WORKSPACE, DAB_ERR_UNSUPPORTED, DAB_ERR_HIP = 1, 2, 3, 4, 5, 6
DAB_LAYOUT_NHWC = 0
DAB_LAYOUT_NCHW = 1
DAB_F32, DAB_BF16, DAB_F16 = 0, 1, 2


class DabError(RuntimeError):
    def __init__(self, name, status, text):
        super().__init__(f"{name} failed: status {status} ({text})")
        self.status = status


class dab_adamw_job(ctypes.Structure):
    _fields_ = [("P", c_void_p), ("G", c_void_p), ("M", c_void_p), ("V", c_void_p), ("MS", c_void_p), ("VS", c_void_p), ("copy", c_void_p),
                ("n", c_int64), ("place", c_uint64), ("grad_dtype", c_int32), ("copy_dtype", c_int32), ("bits", c_int32), ("weight_decay", c_float)]


class dab_adamw_plan(ctypes.Structure):
    _fields_ = [("n_jobs", c_int32), ("turns", c_int32), ("workgroups", c_int32), ("table_bytes", c_int64)]


class dab_adamw_step(ctypes.Structure):
    _fields_ = [("lr", c_double), ("beta1", c_double), ("beta2", c_double), ("eps", c_double), ("step", c_int64), ("seed", c_uint64),
                ("lr_dev", c_void_p), ("step_dev", c_void_p), ("grad_scale", c_void_p)]


class dab_conv_desc(ctypes.Structure):
    _fields_ = [(k, c_int32) for k in
                ("B", "C", "H", "W", "F", "kh", "kw", "pad_h", "pad_w", "stride_h", "stride_w")]

    @property
    def Ho(self):
        return (self.H + 2 * self.pad_h - self.kh) // self.stride_h + 1

    @property
    def Wo(self):
        return (self.W + 2 * self.pad_w - self.kw) // self.stride_w + 1


_SIGNATURES = {
    "dab_strerror": (c_char_p, [c_int]),
    "dab_last_hip_error": (c_int, []),
    "dab_init": (c_int, []),
    "dab_probe_popcount": (c_int, [c_int, c_int, c_int, c_void_p, c_void_p, ctypes.POINTER(ctypes.c_int64),
                                   ctypes.POINTER(c_int32), c_void_p]),
    "dab_estimate_alpha_beta": (c_int, [c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                                        c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "dab_estimate_alpha_beta_bounded": (c_int, [c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_int32, c_void_p,
                                                c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_size_t,
                                                c_void_p]),
    "dab_estimate_sign_split": (c_int, [c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                                        c_void_p, c_void_p, c_void_p]),
    "dab_estimate_alpha_beta_noalloc": (c_int, [c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                                                c_void_p, c_void_p, c_void_p]),
    "dab_estimate_noalloc_max_filters": (c_int32, []),
    "dab_estimate_workspace_bytes": (c_size_t, [c_int32, c_int32]),
    "dab_estimate_max_n": (c_int32, []),
    "dab_pack_weights": (c_int, [c_void_p, c_int32, c_int32, c_int32, c_int32, c_void_p, c_void_p, c_void_p,
                                 c_void_p, c_void_p, c_void_p]),
    "dab_pack_activations": (c_int, [c_void_p, c_int32, c_int32, c_int32, c_int32, c_int32, c_void_p, c_void_p,
                                     c_void_p]),
    "dab_pack_activations_multi": (c_int, [c_void_p, c_int32, c_void_p]),
    "dab_binarize_weights_multi": (c_int, [c_void_p, c_int32, c_void_p, c_size_t, c_void_p]),
    "dab_binarize_weights_multi_workspace_bytes": (c_size_t, [c_void_p, c_int32]),
    "dab_prepare_layers": (c_int, [c_void_p, c_int32, c_void_p, c_int32, c_void_p, c_size_t, c_void_p]),
    "dab_binconv2d": (c_int, [ctypes.POINTER(dab_conv_desc), c_void_p, c_void_p, c_void_p, c_void_p,
                              c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "dab_binconv2d_workspace_bytes": (c_size_t, [ctypes.POINTER(dab_conv_desc)]),
    "dab_binfc": (c_int, [c_int32, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                          c_void_p, c_void_p, c_size_t, c_void_p]),
    "dab_binfc_workspace_bytes": (c_size_t, [c_int32, c_int32, c_int32]),
    "dab_binconv2d_bits": (c_int, [ctypes.POINTER(dab_conv_desc), c_void_p, c_void_p, c_void_p, c_void_p,
                                   c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "dab_binfc_bits": (c_int, [c_int32, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                               c_void_p, c_void_p, c_size_t, c_void_p]),
    "dab_pool_bits": (c_int, [c_void_p, c_int32, c_int32, c_int32, c_int32, c_int32, c_int32, c_int32, c_int32,
                              c_void_p, c_void_p]),
    "dab_wbin_conv2d_workspace_bytes": (c_size_t, [ctypes.POINTER(dab_conv_desc)]),
    "dab_wbin_fc_workspace_bytes": (c_size_t, [c_int32, c_int32, c_int32]),
    "dab_wbin_conv2d": (c_int, [ctypes.POINTER(dab_conv_desc), c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                c_void_p, c_size_t, c_void_p]),
    "dab_wbin_fc": (c_int, [c_int32, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                            c_size_t, c_void_p]),
    "dab_mean_center_clamp": (c_int, [c_void_p, c_int32, c_int32, c_int32, c_int32, c_float, c_float, c_void_p,
                                      c_void_p]),
    "dab_binarized_weights": (c_int, [c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                      c_void_p, c_void_p]),
    "dab_weight_gradient": (c_int, [c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                    c_void_p]),
    "dab_ckpt8_save": (c_int, [c_void_p, c_int32, c_int32, c_int32, c_int64, c_void_p, c_void_p, c_void_p]),
    "dab_ckpt8_restore": (c_int, [c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_int32, c_int64, c_void_p]),
    "dab_ckpt8_weight_gradient_workspace_bytes": (c_size_t, [c_int32, c_int32, c_int32, c_int32, c_int64]),
    "dab_ckpt8_weight_gradient": (c_int, [c_void_p, c_int32, c_int64, c_void_p, c_void_p, c_int32, c_int32, c_int32,
                                          c_void_p, c_void_p, c_size_t, c_void_p]),
    "dab_head_loss_workspace_bytes": (c_size_t, [c_int32, c_int32, c_int32, c_int32, c_int64, c_int64]),
    "dab_head_loss": (c_int, [c_void_p, c_int64, c_void_p, c_int64, c_int32, c_void_p, c_int64, c_int32, c_int32, c_int32,
                              c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "dab_head_loss_gradient_workspace_bytes": (c_size_t, [c_int32, c_int32, c_int32, c_int32, c_int64, c_int64]),
    "dab_head_loss_gradient": (c_int, [c_void_p, c_int64, c_void_p, c_int64, c_int32, c_void_p, c_int64, c_void_p, c_void_p,
                                       c_int32, c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "dab_w4_pack": (c_int, [c_void_p, c_int32, c_int32, c_int32, c_int64, c_void_p, c_void_p, c_void_p]),
    "dab_w4_unpack": (c_int, [c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_void_p]),
    "dab_w4_matvec_workspace_bytes": (c_size_t, [c_int32, c_int32, c_int32, c_int32, c_int64]),
    "dab_w4_matvec": (c_int, [c_void_p, c_int32, c_int64, c_void_p, c_void_p, c_int32, c_int32, c_int32, c_void_p, c_void_p,
                              c_size_t, c_void_p]),
    "dab_rms_norm": (c_int, [c_void_p, c_int32, c_int64, c_void_p, c_int64, c_void_p, c_float, c_int32, c_int32, c_void_p, c_void_p, c_void_p,
                             c_void_p, c_void_p, c_void_p]),
    "dab_rms_norm_gradient_workspace_bytes": (c_size_t, [c_int32, c_int32]),
    "dab_rms_norm_gradient": (c_int, [c_void_p, c_int64, c_void_p, c_int64, c_int32, c_void_p, c_void_p, c_void_p, c_int64, c_int32, c_int32,
                                      c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "dab_adamw_plan_of": (c_int, [ctypes.POINTER(dab_adamw_job), c_int32, ctypes.POINTER(dab_adamw_plan)]),
    "dab_adamw_table": (c_int, [ctypes.POINTER(dab_adamw_job), ctypes.POINTER(dab_adamw_plan), c_void_p, c_size_t, c_void_p]),
    "dab_adamw": (c_int, [c_void_p, c_size_t, ctypes.POINTER(dab_adamw_plan), ctypes.POINTER(dab_adamw_step), c_void_p]),
    "dab_state8_restore": (c_int, [c_void_p, c_void_p, c_int64, c_int32, c_void_p, c_int32, c_void_p]),
    "dab_state8_save": (c_int, [c_void_p, c_int64, c_int32, c_void_p, c_void_p, c_void_p]),
    "dab_adapters": (c_int, [c_void_p, c_int32, c_int64, c_void_p, c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_int32, c_int32, c_int32,
                             c_void_p, c_int32, c_int64, c_void_p, c_void_p, c_void_p]),
    "dab_adapters_gradient_workspace_bytes": (c_size_t, [c_int32, c_int32, c_int32, c_int32, c_int32]),
    "dab_adapters_gradient": (c_int, [c_void_p, c_int64, c_void_p, c_int32, c_int64, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int32,
                                      c_int32, c_int32, c_int32, c_int32, c_void_p, c_int32, c_int64, c_void_p, c_void_p, c_void_p, c_void_p,
                                      c_size_t, c_void_p]),
    "dab_w4_adapters_workspace_bytes": (c_size_t, [c_int32, c_int32, c_int32, c_int32, c_int32, c_int64]),
    "dab_w4_adapters": (c_int, [c_void_p, c_int32, c_int64, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_int32,
                                c_int32, c_int32, c_void_p, c_void_p, c_size_t, c_void_p]),
}

_lib = None
_native = None


def lib() -> ctypes.CDLL:
    """The loaded shared library (opened on first use; raises if it was never built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_1804_02941_amd.build` first")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype, fn.argtypes = res, args
        _lib = handle
    return _lib


def native():
    """The module of the native calls (imported on first use; raises if it was never built).

    Its functions are named like the entry points, take their arguments without the stream, check the tensors as
    _ptr() does and raise like _check().  Measured over the nine calls of one sketch, launches included: 4.1 us of
    host time a call, 6.9 through ctypes."""
    global _native
    if _native is None:
        lib()
        try:
            from . import _dab_call
        except ImportError as e:
            raise RuntimeError(f"_dab_call.so is missing or unusable ({e}): run `python -m paper_1804_02941_amd.build` first") from e
        _dab_call.setup(_pointer, _check, _number, dab_conv_desc, ctypes.ArgumentError)
        _native = _dab_call
    return _native


def _check(name, status):
    if status != DAB_OK:
        raise DabError(name, status, lib().dab_strerror(status).decode())


def _ptr(t, dtype, name):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a tensor on the GPU")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: tensor must be contiguous")
    return t.data_ptr()


_KINDS = {"f": torch.float32, "i": torch.int32, "b": torch.uint8}


def _pointer(t, kind, name):
    """What native code does not take at a glance: the address of tensor t (kind "v", or no name: unchecked)."""
    return t.data_ptr() if name is None or kind == "v" else _ptr(t, _KINDS[kind], name)


_NUMBERS = {"i": c_int32, "z": c_size_t, "f": ctypes.c_float}


def _number(value, kind):
    """What native code takes for no number at a glance, as ctypes converts it for a C argument."""
    ctype = _NUMBERS[kind]
    try:
        ctype.from_param(value)                                     # (its result does not show the number)
    except (TypeError, AttributeError) as e:
        raise ctypes.ArgumentError(str(e)) from None
    while True:
        if isinstance(value, ctype):
            return value.value
        try:
            return ctype(value).value
        except TypeError:
            value = value._as_parameter_


def _stream():
    # the raw handle of the current device's current stream; torch.cuda.current_stream() builds a Stream
    # object around it first (measured: 2.7 us a call against 0.2, of the 7.4 us of a small call)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def words_per_pixel(C):
    return (C + 31) // 32


def padded_filters(F):
    return 64 * ((F + 63) // 64)


def _workspace(nbytes, dev, ws):
    """A caller-supplied workspace tensor if it is large enough, else a fresh one (None when none is needed)."""
    if nbytes == 0:
        return None
    if ws is not None and ws.numel() * ws.element_size() >= nbytes:
        return ws
    return torch.empty(nbytes, dtype=torch.uint8, device=dev)


def estimate_outputs(F, dev):
    """Empty output tensors of dab_estimate_alpha_beta for F filters."""
    return dict(
        alpha=torch.empty(F, dtype=torch.float32, device=dev), beta=torch.empty(F, dtype=torch.float32, device=dev),
        K=torch.empty(F, dtype=torch.int32, device=dev), thr_val=torch.empty(F, dtype=torch.float32, device=dev),
        thr_idx=torch.empty(F, dtype=torch.int32, device=dev),
        alpha_is_upper=torch.empty(F, dtype=torch.uint8, device=dev))


def dab_estimate_alpha_beta(W, out=None, ws=None):
    """W [F, n] fp32 -> dict(alpha, beta, K, thr_val, thr_idx, alpha_is_upper), each [F].

    out: a dict from estimate_outputs() to write into instead of fresh tensors."""
    F, n = W.shape
    dev = W.device
    if out is None:
        out = estimate_outputs(F, dev)
    call = _native or native()
    nbytes = call.dab_estimate_workspace_bytes(F, n)
    ws = _workspace(nbytes, dev, ws)
    call.dab_estimate_alpha_beta(W, F, n, out["alpha"], out["beta"], out["K"], out["thr_val"], out["thr_idx"],
                                 out["alpha_is_upper"], ws, nbytes)
    return out


def dab_estimate_alpha_beta_noalloc(W, out):
    """dab_estimate_alpha_beta into the tensors of `out` (from estimate_outputs()), with the hand-over flags in
    the library's own device array: the call allocates nothing."""
    F, n = W.shape
    _check("dab_estimate_alpha_beta_noalloc", lib().dab_estimate_alpha_beta_noalloc(
        _ptr(W, torch.float32, "W"), F, n, out["alpha"].data_ptr(), out["beta"].data_ptr(), out["K"].data_ptr(),
        out["thr_val"].data_ptr(), out["thr_idx"].data_ptr(), out["alpha_is_upper"].data_ptr(), _stream()))
    return out


def dab_estimate_sign_split(W, out=None):
    """W [F, n] fp32 -> the same dict as dab_estimate_alpha_beta for e = [w >= 0], alpha = mean|w|, beta = -alpha."""
    F, n = W.shape
    if out is None:
        out = estimate_outputs(F, W.device)
    call = _native or native()
    call.dab_estimate_sign_split(W, F, n, out["alpha"], out["beta"], out["K"], out["thr_val"], out["thr_idx"],
                                 out["alpha_is_upper"])
    return out


def pack_weights_outputs(F, C, kh, kw, dev):
    """Empty (E_packed, ecnt) of dab_pack_weights."""
    R, Fp = kh * kw * words_per_pixel(C), padded_filters(F)
    return (torch.empty((R, Fp), dtype=torch.int32, device=dev),
            torch.empty((F, kh * kw), dtype=torch.int32, device=dev))


def dab_pack_weights(W, thr_val, thr_idx, alpha_is_upper, out=None):
    """W [F, C, kh, kw] fp32 + split descriptor -> (E_packed uint32-as-int32 [R, Fp], ecnt int32 [F, kh*kw]).

    out: an (E_packed, ecnt) pair from pack_weights_outputs() to write into."""
    F, C, kh, kw = W.shape
    E, ecnt = out if out is not None else pack_weights_outputs(F, C, kh, kw, W.device)
    call = _native or native()
    call.dab_pack_weights(W, F, C, kh, kw, thr_val, thr_idx, alpha_is_upper, E, ecnt)
    return E, ecnt


def dab_pack_activations(X, layout=DAB_LAYOUT_NHWC, tau=None, out=None):
    """X fp32 NHWC [B,H,W,C] (or NCHW [B,C,H,W]; a 2-D [B,C] is H=W=1) -> int32 [B,H,W,Cw]."""
    A = (_native or native()).pack_activations(X, layout, tau, out)
    if A is not None:
        return A
    if X.dim() == 2:
        B, C = X.shape
        H = W = 1
    elif layout == DAB_LAYOUT_NHWC:
        B, H, W, C = X.shape
    else:
        B, C, H, W = X.shape
    A = out if out is not None else torch.empty((B, H, W, words_per_pixel(C)), dtype=torch.int32, device=X.device)
    call = _native or native()
    call.dab_pack_activations(X, layout, B, C, H, W, tau, A)
    return A


def dab_init():
    """One-time set-up of the current device (every entry point does it on first use as well)."""
    _check("dab_init", lib().dab_init())


def dab_probe_popcount(pair, iters, grid, out, clocks):
    """One launch of the popcount-rate probe; returns (lane-popcounts issued, constant-rate clock in kHz)."""
    ops, khz = ctypes.c_int64(0), c_int32(0)
    _check("dab_probe_popcount", lib().dab_probe_popcount(
        int(bool(pair)), iters, grid, _ptr(out, torch.int32, "out"), _ptr(clocks, torch.int64, "clocks"),
        ctypes.byref(ops), ctypes.byref(khz), _stream()))
    return ops.value, khz.value


class dab_weight_job(ctypes.Structure):
    _fields_ = [("W", c_void_p), ("F", c_int32), ("C", c_int32), ("kh", c_int32), ("kw", c_int32),
                ("alpha", c_void_p), ("beta", c_void_p), ("K", c_void_p), ("thr_val", c_void_p), ("thr_idx", c_void_p),
                ("alpha_is_upper", c_void_p), ("E_packed", c_void_p), ("ecnt", c_void_p),
                ("K_prev", c_void_p), ("alpha_is_upper_prev", c_void_p), ("max_change", c_int32)]


def weight_jobs(items):
    """A host array of dab_weight_job from dicts(W=[F,C,kh,kw], est=estimate_outputs(), packed=(E, ecnt) or None,
    prev=(K_prev, alpha_is_upper_prev, max_change) or None); built once, reused per call."""
    arr = (dab_weight_job * len(items))()
    for k, it in enumerate(items):
        W, est = it["W"], it["est"]
        F, C, kh, kw = W.shape
        E, ecnt = it.get("packed") or (None, None)
        Kp, up, mc = it.get("prev") or (None, None, 0)
        arr[k] = dab_weight_job(
            _ptr(W, torch.float32, "W"), F, C, kh, kw, _ptr(est["alpha"], torch.float32, "alpha"),
            _ptr(est["beta"], torch.float32, "beta"), _ptr(est["K"], torch.int32, "K"),
            _ptr(est["thr_val"], torch.float32, "thr_val"), _ptr(est["thr_idx"], torch.int32, "thr_idx"),
            _ptr(est["alpha_is_upper"], torch.uint8, "alpha_is_upper"), _ptr(E, torch.int32, "E_packed"),
            _ptr(ecnt, torch.int32, "ecnt"), _ptr(Kp, torch.int32, "K_prev"), _ptr(up, torch.uint8, "alpha_is_upper_prev"), mc)
    return arr


def dab_binarize_weights_multi(jobs, ws=None):
    """Estimation and weight packing of every job of weight_jobs() in two or three launches."""
    nbytes = lib().dab_binarize_weights_multi_workspace_bytes(jobs, len(jobs))
    if nbytes and (ws is None or ws.numel() * ws.element_size() < nbytes):
        ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    _check("dab_binarize_weights_multi", lib().dab_binarize_weights_multi(
        jobs, len(jobs), ws.data_ptr() if nbytes else None, nbytes, _stream()))


class dab_pack_job(ctypes.Structure):
    _fields_ = [("X", c_void_p), ("tau", c_void_p), ("A_packed", c_void_p),
                ("B", c_int32), ("C", c_int32), ("H", c_int32), ("W", c_int32)]


def pack_jobs(items):
    """A host array of dab_pack_job from (X NHWC or [B,C], tau or None, A_packed) triples (built once, reused per call)."""
    arr = (dab_pack_job * len(items))()
    for k, (X, tau, A) in enumerate(items):
        if X.dim() == 2:
            B, C = X.shape
            H = W = 1
        else:
            B, H, W, C = X.shape
        arr[k] = dab_pack_job(_ptr(X, torch.float32, "X"), _ptr(tau, torch.float32, "tau"), _ptr(A, torch.int32, "A_packed"),
                              B, C, H, W)
    return arr


def dab_pack_activations_multi(jobs):
    """dab_pack_activations for every job of pack_jobs() in one launch."""
    _check("dab_pack_activations_multi", lib().dab_pack_activations_multi(jobs, len(jobs), _stream()))


def dab_prepare_layers(wjobs, pjobs, ws=None):
    """dab_binarize_weights_multi(wjobs) and dab_pack_activations_multi(pjobs) in the same launches."""
    nbytes = lib().dab_binarize_weights_multi_workspace_bytes(wjobs, len(wjobs))
    if nbytes and (ws is None or ws.numel() * ws.element_size() < nbytes):
        ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    _check("dab_prepare_layers", lib().dab_prepare_layers(
        wjobs, len(wjobs), pjobs, len(pjobs), ws.data_ptr() if nbytes else None, nbytes, _stream()))


def dab_binconv2d(desc, A_packed, E_packed, alpha, beta, want_s1=False, out=None, ws=None):
    """Binarized convolution; returns Y fp32 [B,Ho,Wo,F] (and int32 s1 of the same shape if asked)."""
    if not want_s1:
        Y = (_native or native()).binconv2d(desc, A_packed, E_packed, alpha, beta, out, ws)
        if Y is not None:
            return Y
    dev = A_packed.device
    shape = (desc.B, desc.Ho, desc.Wo, desc.F) if out is None or want_s1 else None
    Y = out if out is not None else torch.empty(shape, dtype=torch.float32, device=dev)
    s1 = torch.empty(shape, dtype=torch.int32, device=dev) if want_s1 else None
    call = _native or native()
    nbytes = call.dab_binconv2d_workspace_bytes(desc)
    ws = _workspace(nbytes, dev, ws)
    call.dab_binconv2d(desc, A_packed, E_packed, alpha, beta, Y, s1, ws, nbytes)
    return (Y, s1) if want_s1 else Y


def dab_binfc(A_packed, E_packed, alpha, beta, Kin, want_s1=False, out=None, ws=None):
    """Binarized fully-connected layer; A_packed [B, Kw], returns Y fp32 [B, F]."""
    if not want_s1:
        Y = (_native or native()).binfc(A_packed, E_packed, alpha, beta, Kin, out, ws)
        if Y is not None:
            return Y
    dev = A_packed.device
    B = A_packed.shape[0]
    F = alpha.shape[0]
    Y = out if out is not None else torch.empty((B, F), dtype=torch.float32, device=dev)
    s1 = torch.empty((B, F), dtype=torch.int32, device=dev) if want_s1 else None
    call = _native or native()
    nbytes = call.dab_binfc_workspace_bytes(B, Kin, F)
    ws = _workspace(nbytes, dev, ws)
    call.dab_binfc(B, Kin, F, A_packed, E_packed, alpha, beta, Y, s1, ws, nbytes)
    return (Y, s1) if want_s1 else Y


def dab_binconv2d_bits(desc, A_packed, E_packed, alpha, beta, tau_out=None, out=None, ws=None):
    """Binarized convolution with the re-binarizing epilogue; returns int32 [B,Ho,Wo,ceil(F/32)]."""
    A_next = (_native or native()).binconv2d_bits(desc, A_packed, E_packed, alpha, beta, tau_out, out, ws)
    if A_next is not None:
        return A_next
    dev = A_packed.device
    A_next = out if out is not None else torch.empty((desc.B, desc.Ho, desc.Wo, words_per_pixel(desc.F)), dtype=torch.int32,
                                                     device=dev)
    call = _native or native()
    nbytes = call.dab_binconv2d_workspace_bytes(desc)
    ws = _workspace(nbytes, dev, ws)
    call.dab_binconv2d_bits(desc, A_packed, E_packed, alpha, beta, tau_out, A_next, ws, nbytes)
    return A_next


def dab_binfc_bits(A_packed, E_packed, alpha, beta, Kin, tau_out=None, out=None, ws=None):
    """Binarized fully-connected layer with the re-binarizing epilogue; returns int32 [B, ceil(F/32)]."""
    dev = A_packed.device
    B, F = A_packed.shape[0], alpha.shape[0]
    A_next = out if out is not None else torch.empty((B, words_per_pixel(F)), dtype=torch.int32, device=dev)
    call = _native or native()
    nbytes = call.dab_binfc_workspace_bytes(B, Kin, F)
    ws = _workspace(nbytes, dev, ws)
    call.dab_binfc_bits(B, Kin, F, A_packed, E_packed, alpha, beta, tau_out, A_next, ws, nbytes)
    return A_next


def dab_pool_bits(A_packed, C, kh, kw, stride_h, stride_w, out=None):
    """OR-pooling of packed signs: int32 [B,H,W,Cw] -> [B,Ho,Wo,Cw] (windows inside the image)."""
    A_pooled = (_native or native()).pool_bits(A_packed, C, kh, kw, stride_h, stride_w, out)
    if A_pooled is not None:
        return A_pooled
    B, H, W, Cw = A_packed.shape
    Ho, Wo = (H - kh) // stride_h + 1, (W - kw) // stride_w + 1
    A_pooled = out if out is not None else torch.empty((B, max(Ho, 0), max(Wo, 0), Cw), dtype=torch.int32,
                                                        device=A_packed.device)
    call = _native or native()
    call.dab_pool_bits(A_packed, B, C, H, W, kh, kw, stride_h, stride_w, A_pooled)
    return A_pooled


DAB_CENTER_FILTER, DAB_CENTER_CHANNEL = 0, 1


def dab_mean_center_clamp(W, axis=DAB_CENTER_FILTER, lo=-1.0, hi=1.0, out=None):
    """MeanCenter + Clamp of W[F,C,kh,kw] (fp32); out may be W itself."""
    F, C = W.shape[0], W.shape[1]
    T = W.shape[2] * W.shape[3]
    W_out = out if out is not None else torch.empty_like(W)
    call = _native or native()
    call.dab_mean_center_clamp(W, F, C, T, axis, lo, hi, W_out)
    return W_out


def dab_binarized_weights(W, alpha, beta, thr_val, thr_idx, alpha_is_upper, out=None):
    """W~ = alpha e + beta (1 - e) as fp32 [F,n] from W[F,n] and the estimator's outputs."""
    F, n = W.shape
    Wt = out if out is not None else torch.empty_like(W)
    call = _native or native()
    call.dab_binarized_weights(W, F, n, alpha, beta, thr_val, thr_idx, alpha_is_upper, Wt)
    return Wt


def dab_weight_gradient(W, thr_val, thr_idx, alpha_is_upper, upstream=None, out=None):
    """Theorem 4's element-wise factor G~ for W[F,n] (times `upstream` when given)."""
    F, n = W.shape
    G = out if out is not None else torch.empty_like(W)
    call = _native or native()
    call.dab_weight_gradient(W, F, n, thr_val, thr_idx, alpha_is_upper, upstream, G)
    return G


def dab_estimate_alpha_beta_bounded(W, K_prev, alpha_is_upper_prev, max_change, out=None, ws=None):
    """dab_estimate_alpha_beta with the split at most `max_change` elements from the previous one
    (K_prev int32 [F], alpha_is_upper_prev uint8 [F]: the previous call's outputs; `out` may hold them)."""
    F, n = W.shape
    o = out if out is not None else estimate_outputs(F, W.device)
    call = _native or native()
    nbytes = call.dab_estimate_workspace_bytes(F, n)
    ws = _workspace(nbytes, W.device, ws)
    call.dab_estimate_alpha_beta_bounded(W, F, n, K_prev, alpha_is_upper_prev, max_change, o["alpha"], o["beta"],
                                         o["K"], o["thr_val"], o["thr_idx"], o["alpha_is_upper"], ws, nbytes)
    return o


def dab_wbin_conv2d(desc, X, E_packed, alpha, beta, out=None, ws=None):
    """Weights-only binarized convolution: X fp32 NHWC [B,H,W,C] -> Y fp32 [B,Ho,Wo,F]."""
    Y = (_native or native()).wbin_conv2d(desc, X, E_packed, alpha, beta, out, ws)
    if Y is not None:
        return Y
    dev = X.device
    Y = out if out is not None else torch.empty((desc.B, desc.Ho, desc.Wo, desc.F), dtype=torch.float32, device=dev)
    call = _native or native()
    nbytes = call.dab_wbin_conv2d_workspace_bytes(desc)
    ws = _workspace(nbytes, dev, ws)
    call.dab_wbin_conv2d(desc, X, E_packed, alpha, beta, Y, ws, nbytes)
    return Y


def dab_wbin_fc(X, E_packed, alpha, beta, out=None, ws=None):
    """Weights-only binarized fully-connected layer: X fp32 [B,Kin] -> Y fp32 [B,F]."""
    Y = (_native or native()).wbin_fc(X, E_packed, alpha, beta, out, ws)
    if Y is not None:
        return Y
    dev = X.device
    B, Kin = X.shape
    F = alpha.shape[0]
    Y = out if out is not None else torch.empty((B, F), dtype=torch.float32, device=dev)
    call = _native or native()
    nbytes = call.dab_wbin_fc_workspace_bytes(B, Kin, F)
    ws = _workspace(nbytes, dev, ws)
    call.dab_wbin_fc(B, Kin, F, X, E_packed, alpha, beta, Y, ws, nbytes)
    return Y


# ------------------------------------------------------------------ the real-valued ends of a network
_REAL = {torch.float32: DAB_F32, torch.bfloat16: DAB_BF16, torch.float16: DAB_F16}


def _counted(t, name):
    """t, a matrix whose rows and columns the C calls' 32-bit sizes count (ctypes would pass the lower bits of larger ones)."""
    if max(t.shape) > 2 ** 31 - 1:
        raise ValueError(f"{name}: expected at most {2 ** 31 - 1} rows and columns, got {tuple(t.shape)}")
    return t


def _matrix(t, name):
    """(address, element type, distance of the rows) of a matrix on the GPU whose rows are contiguous."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a tensor on the GPU")
    if t.dtype not in _REAL:
        raise TypeError(f"{name}: expected torch.float32, torch.bfloat16 or torch.float16, got {t.dtype}")
    if t.dim() != 2:
        raise ValueError(f"{name}: expected two dimensions, got {t.dim()}")
    rows, cols = t.shape
    if cols > 1 and t.stride(1) != 1 or rows > 1 and t.stride(0) < cols:
        raise ValueError(f"{name}: the elements of a row must be contiguous and rows apart")
    _counted(t, name)
    return t.data_ptr(), _REAL[t.dtype], t.stride(0) if rows > 1 else cols


def _shaped(t, shape, name):
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    return t


def _result(out, shape, dtype, dev, name):
    """The caller's output tensor, checked, or a new one."""
    if out is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    _ptr(out, dtype, name)
    return _shaped(out, shape, name)


def _scratch(nbytes, dev, ws):
    """(tensor, address, bytes) of a caller's workspace that is large enough, else of a new one."""
    ws = _workspace(nbytes, dev, ws)
    return ws, ws.data_ptr() if ws is not None else None, nbytes


def ckpt8_outputs(rows, cols, dev):
    """Empty (Q, S) of dab_ckpt8_save."""
    groups = (cols + 31) // 32
    return (torch.empty((rows, 32 * groups), dtype=torch.int8, device=dev), torch.empty((rows, groups), dtype=torch.uint8, device=dev))


def _saved(Q, S, cols):
    rows, groups = Q.shape[0], (cols + 31) // 32
    _counted(_shaped(Q, (rows, 32 * groups), "Q"), "Q"), _shaped(S, (rows, groups), "S")
    return _ptr(Q, torch.int8, "Q"), _ptr(S, torch.uint8, "S"), rows


def dab_ckpt8_save(X, out=None):
    """X [rows, cols] fp32, bf16 or f16 -> (Q int8 [rows, 32 ceil(cols/32)], S uint8 [rows, ceil(cols/32)])."""
    done = (_native or native()).ckpt8_save(X, out)
    if done is not None:
        return done
    ptr, dtype, ld = _matrix(X, "X")
    rows, cols = X.shape
    Q, S = out if out is not None else ckpt8_outputs(rows, cols, X.device)
    q, s, n = _saved(Q, S, cols)
    if n != rows:
        raise ValueError(f"Q: expected {rows} rows, got {n}")
    _check("dab_ckpt8_save", lib().dab_ckpt8_save(ptr, dtype, rows, cols, ld, q, s, _stream()))
    return Q, S


def dab_ckpt8_restore(Q, S, cols, dtype=torch.float32, out=None):
    """What dab_ckpt8_save() kept of `cols` channels, as a tensor [rows, cols] of dtype (or into `out`)."""
    if out is None:
        done = (_native or native()).ckpt8_restore(Q, S, cols, dtype)
        if done is not None:
            return done
    q, s, rows = _saved(Q, S, cols)
    X = out if out is not None else torch.empty((rows, cols), dtype=dtype, device=Q.device)
    ptr, code, ld = _matrix(_shaped(X, (rows, cols), "out"), "out")
    _check("dab_ckpt8_restore", lib().dab_ckpt8_restore(q, s, rows, cols, ptr, code, ld, _stream()))
    return X


def dab_ckpt8_weight_gradient(dY, Q, S, cols, out=None, ws=None):
    """dW = dY^T X fp32 [F, cols] from dY [rows, F] (fp32, bf16 or f16) and what dab_ckpt8_save() kept of X [rows, cols]."""
    done = (_native or native()).ckpt8_weight_gradient(dY, Q, S, cols, out, ws)
    if done is not None:
        return done
    ptr, dtype, ld = _matrix(dY, "dY")
    q, s, rows = _saved(Q, S, cols)
    F = _shaped(dY, (rows, dY.shape[1]), "dY").shape[1]
    dW = _result(out, (F, cols), torch.float32, dY.device, "out")
    nbytes = lib().dab_ckpt8_weight_gradient_workspace_bytes(rows, cols, F, dtype, ld)
    ws, at, nbytes = _scratch(nbytes, dY.device, ws)
    _check("dab_ckpt8_weight_gradient", lib().dab_ckpt8_weight_gradient(ptr, dtype, ld, q, s, rows, cols, F, dW.data_ptr(), at, nbytes,
                                                                        _stream()))
    return dW


def _head(H, W, targets):
    h, dtype, ldh = _matrix(H, "H")
    w, dtype_w, ldw = _matrix(W, "W")
    if dtype != dtype_w:
        raise TypeError(f"W: expected {H.dtype}, got {W.dtype}")
    T, D = H.shape
    _shaped(W, (W.shape[0], D), "W")
    return h, ldh, w, ldw, dtype, _ptr(_shaped(targets, (T,), "targets"), torch.int64, "targets"), T, D, W.shape[0]


def dab_head_loss(H, W, targets, ignore_index=-100, out=None, ws=None):
    """Softmax cross entropy of H [T, D] W [V, D]^T (bf16 or fp32) with targets int64 [T] -> (loss fp32 [T], lse fp32 [T])."""
    done = (_native or native()).head_loss(H, W, targets, ignore_index, out, ws)
    if done is not None:
        return done
    h, ldh, w, ldw, dtype, t, T, D, V = _head(H, W, targets)
    loss, lse = out if out is not None else (None, None)
    loss, lse = _result(loss, (T,), torch.float32, H.device, "loss"), _result(lse, (T,), torch.float32, H.device, "lse")
    ws, at, nbytes = _scratch(lib().dab_head_loss_workspace_bytes(T, D, V, dtype, ldh, ldw), H.device, ws)
    _check("dab_head_loss", lib().dab_head_loss(h, ldh, w, ldw, dtype, t, ignore_index, T, D, V, loss.data_ptr(), lse.data_ptr(), at, nbytes,
                                                _stream()))
    return loss, lse


def dab_head_loss_gradient(H, W, targets, lse, g=None, ignore_index=-100, out=None, ws=None):
    """(dH, dW) of sum_t g_t loss_t (g fp32 [T], or None for ones), with lse from dab_head_loss() for the same H, W and targets."""
    done = (_native or native()).head_loss_gradient(H, W, targets, lse, g, ignore_index, out, ws)
    if done is not None:
        return done
    h, ldh, w, ldw, dtype, t, T, D, V = _head(H, W, targets)
    dH, dW = out if out is not None else (None, None)
    dH, dW = _result(dH, (T, D), H.dtype, H.device, "dH"), _result(dW, (V, D), H.dtype, H.device, "dW")
    l = _ptr(_shaped(lse, (T,), "lse"), torch.float32, "lse")
    gp = None if g is None else _ptr(_shaped(g, (T,), "g"), torch.float32, "g")
    ws, at, nbytes = _scratch(lib().dab_head_loss_gradient_workspace_bytes(T, D, V, dtype, ldh, ldw), H.device, ws)
    _check("dab_head_loss_gradient", lib().dab_head_loss_gradient(h, ldh, w, ldw, dtype, t, ignore_index, l, gp, T, D, V, dH.data_ptr(),
                                                                  dW.data_ptr(), at, nbytes, _stream()))
    return dH, dW


def w4_outputs(F, K, dev):
    """Empty (Q, S) of dab_w4_pack."""
    return (torch.empty(((F + 15) // 16, (K + 127) // 128, 64, 16), dtype=torch.uint8, device=dev),
            torch.empty(((F + 15) // 16, (K + 511) // 512, 64, 4), dtype=torch.uint8, device=dev))


def _packed(Q, S, F, K):
    _shaped(Q, ((F + 15) // 16, (K + 127) // 128, 64, 16), "Q"), _shaped(S, ((F + 15) // 16, (K + 511) // 512, 64, 4), "S")
    return _ptr(Q, torch.uint8, "Q"), _ptr(S, torch.uint8, "S")


def dab_w4_pack(W, out=None):
    """W [F, K] fp32, bf16 or f16 -> (Q, S): 4-bit codes and scale bytes in the layout of include/dab.h."""
    done = (_native or native()).w4_pack(W, out)
    if done is not None:
        return done
    ptr, dtype, ld = _matrix(W, "W")
    F, K = W.shape
    Q, S = out if out is not None else w4_outputs(F, K, W.device)
    q, s = _packed(Q, S, F, K)
    _check("dab_w4_pack", lib().dab_w4_pack(ptr, dtype, F, K, ld, q, s, _stream()))
    return Q, S


def dab_w4_unpack(Q, S, F, K, out=None):
    """The weights that dab_w4_pack()'s (Q, S) stand for, fp32 [F, K]."""
    done = (_native or native()).w4_unpack(Q, S, F, K, out)
    if done is not None:
        return done
    q, s = _packed(Q, S, F, K)
    W = _result(out, (F, K), torch.float32, Q.device, "out")
    _check("dab_w4_unpack", lib().dab_w4_unpack(q, s, F, K, W.data_ptr(), _stream()))
    return W


def dab_w4_matvec(X, Q, S, F, out=None, ws=None):
    """X [B, K] (fp32, bf16 or f16) times the F packed rows -> Y [B, F] of X's type."""
    done = (_native or native()).w4_matvec(X, Q, S, F, out, ws)
    if done is not None:
        return done
    ptr, dtype, ld = _matrix(X, "X")
    B, K = X.shape
    q, s = _packed(Q, S, F, K)
    Y = _result(out, (B, F), X.dtype, X.device, "out")
    ws, at, nbytes = _scratch(lib().dab_w4_matvec_workspace_bytes(B, K, F, dtype, ld), X.device, ws)
    _check("dab_w4_matvec", lib().dab_w4_matvec(ptr, dtype, ld, q, s, B, K, F, Y.data_ptr(), at, nbytes, _stream()))
    return Y


# ------------------------------------------------------------------ what stands around the layers: norms, steps, adapters
def _here(*tensors):
    """Refuses tensors of another device than the current one, whose stream the calls take."""
    now = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and t.is_cuda and t.device.index != now:
            raise ValueError(f"a tensor lies on {t.device}, the current device is cuda:{now}")


def _beside(t, shape, dtypes, name):
    """(address, element type, distance of the rows) of a matrix of this shape and one of these types, or of none."""
    if t is None:
        return None, DAB_F32, 0
    ptr, code, ld = _matrix(t, name)
    if t.dtype not in dtypes:
        raise TypeError(f"{name}: expected {' or '.join(map(str, dtypes))}, got {t.dtype}")
    _shaped(t, shape, name)
    return ptr, code, ld


def dab_rms_norm(X, gain, residual=None, eps=1e-5, save=False, out=None):
    """The root-mean-square norm of X + residual (fp32, bf16 or f16 [rows, cols]) times gain (fp32 [cols]) -> (Y, H, rstd, saved).

    H is the sum (X itself without a residual), rstd fp32 [rows] what the gradient takes.  save: Y as dab_ckpt8_save() keeps it too, saved = (Q, S), or
    only so (save="only": Y is None); else saved is None.  out: (Y, H, rstd, saved) to write into, None where a tensor is to be new; H may be
    X or the residual, Y may be X."""
    done = (_native or native()).rms_norm(X, gain, residual, eps, save, out)
    if done is not None:
        return done
    ptr, dtype, ld = _matrix(X, "X")
    rows, cols = X.shape
    r, _, ldr = _beside(residual, X.shape, (X.dtype,), "residual")
    g = _ptr(_shaped(gain, (cols,), "gain"), torch.float32, "gain")
    Y, H, rstd, saved = out if out is not None else (None, None, None, None)
    _here(X, residual, gain, Y, H, rstd, *(saved or ()))
    H = _result(H, X.shape, X.dtype, X.device, "H") if residual is not None else X
    Y = _result(Y, X.shape, X.dtype, X.device, "Y") if save != "only" else None
    rstd = _result(rstd, (rows,), torch.float32, X.device, "rstd")
    q = s = None
    if save:
        saved = saved if saved is not None else ckpt8_outputs(rows, cols, X.device)
        q, s, n = _saved(*saved, cols)
        if n != rows:
            raise ValueError(f"Q: expected {rows} rows, got {n}")
    _check("dab_rms_norm", lib().dab_rms_norm(ptr, dtype, ld, r, ldr, g, eps, rows, cols, H.data_ptr() if residual is not None else None,
                                              Y.data_ptr() if Y is not None else None, q, s, rstd.data_ptr(), _stream()))
    return Y, H, rstd, saved if save else None


def dab_rms_norm_gradient(dY, H, gain, rstd, dH=None, out=None, ws=None):
    """(dX [rows, cols] of H's type, dgain fp32 [cols]) from dY, dab_rms_norm()'s H and rstd, and what arrives at H beside the norm (dH)."""
    done = (_native or native()).rms_norm_gradient(dY, H, gain, rstd, dH, out, ws)
    if done is not None:
        return done
    h, dtype, ldh = _matrix(H, "H")
    rows, cols = H.shape
    dy, _, lddy = _beside(dY, H.shape, (H.dtype,), "dY")
    if dy is None:
        raise TypeError("dY: expected a tensor on the GPU")
    d, _, ldd = _beside(dH, H.shape, (H.dtype,), "dH")
    g, s = _ptr(_shaped(gain, (cols,), "gain"), torch.float32, "gain"), _ptr(_shaped(rstd, (rows,), "rstd"), torch.float32, "rstd")
    dX, dgain = out if out is not None else (None, None)
    _here(dY, H, gain, rstd, dH, dX, dgain)
    dX, dgain = _result(dX, H.shape, H.dtype, H.device, "dX"), _result(dgain, (cols,), torch.float32, H.device, "dgain")
    ws, at, nbytes = _scratch(lib().dab_rms_norm_gradient_workspace_bytes(rows, cols), H.device, ws)
    _check("dab_rms_norm_gradient", lib().dab_rms_norm_gradient(dy, lddy, h, ldh, dtype, g, s, d, ldd, rows, cols, dX.data_ptr(), dgain.data_ptr(), at,
                                                                nbytes, _stream()))
    return dX, dgain


def _flat(t, n, dtypes, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a tensor on the GPU")
    if t.dtype not in dtypes:
        raise TypeError(f"{name}: expected {' or '.join(map(str, dtypes))}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: tensor must be contiguous")
    if t.numel() != n:
        raise ValueError(f"{name}: expected {n} elements, got {t.numel()}")
    return t.data_ptr()


def adamw_states(P, bits=32):
    """The two states of a tensor before its first step: zeros, fp32 like P (bits=32) or pairs of codes and scale bytes (bits=8)."""
    if bits == 32:
        return torch.zeros_like(P, dtype=torch.float32), torch.zeros_like(P, dtype=torch.float32)
    groups = (P.numel() + 31) // 32
    return tuple((torch.zeros(32 * groups, dtype=torch.uint8, device=P.device), torch.full((groups,), 27, dtype=torch.uint8, device=P.device))
                 for _ in range(2))


class _AdamwJobs:
    """What adamw_jobs() makes: the table in device memory, and the tensors that it points into."""

    def __init__(self, table, plan, tensors):
        self.table, self.plan, self.tensors = table, plan, tensors

    def __len__(self):
        return self.plan.n_jobs


def adamw_jobs(items):
    """The table of a step's tensors from dicts(P, G, M, V, copy=None, weight_decay=0.0, place=None), built once and reused per step.

    It holds addresses: as long as all tensors stay where they are, the gradients among them (write each step's into the same tensors), it serves every step.
    Building it costs far more than a step does (96 small tensors: 0.5 to 0.6 ms, the step's call 5 us).

    P: fp32; G: a gradient of as many elements (fp32, bf16 or f16); M, V: from adamw_states(); copy: a bf16 or f16 tensor that takes the new P
    too; place: of the tensor in the sequence of random numbers (behind the tensor before it unless given).  The tensors are kept alive.  The
    table is written on the current stream and waited for (in a graph that is being captured, it is written at every replay)."""
    if not items:
        raise ValueError("expected one tensor at least")
    arr, written, kept, place = (dab_adamw_job * len(items))(), [], [], 0
    device = None
    for k, it in enumerate(items):
        P, G, M, V, copy = it["P"], it["G"], it["M"], it["V"], it.get("copy")
        n = P.numel() if isinstance(P, torch.Tensor) else 0
        p = _flat(P, n, (torch.float32,), "P")
        device = P.device if device is None else device
        g = _flat(G, n, tuple(_REAL), "G")
        c = _flat(copy, n, (torch.bfloat16, torch.float16), "copy") if copy is not None else None
        bits = 8 if isinstance(M, (tuple, list)) else 32
        if bits == 8:
            if not isinstance(V, (tuple, list)):
                raise TypeError("V: expected codes and scale bytes, as for M")
            groups = (n + 31) // 32
            m, ms = _flat(M[0], 32 * groups, (torch.uint8,), "M"), _flat(M[1], groups, (torch.uint8,), "M's scales")
            v, vs = _flat(V[0], 32 * groups, (torch.uint8,), "V"), _flat(V[1], groups, (torch.uint8,), "V's scales")
            states = [*M, *V]
        else:
            m, v, ms, vs = _flat(M, n, (torch.float32,), "M"), _flat(V, n, (torch.float32,), "V"), None, None
            states = [M, V]
        tensors = [P, *states] + ([copy] if copy is not None else [])
        for t in [G, *tensors]:
            if t.device != device:
                raise ValueError(f"all tensors are on one device: {t.device} and {device}")
        if it.get("place") is not None:
            place = it["place"]
        arr[k] = dab_adamw_job(p, g, m, v, ms, vs, c, n, place, _REAL[G.dtype], _REAL[copy.dtype] if copy is not None else 0, bits,
                               it.get("weight_decay", 0.0))
        place += 32 * ((n + 31) // 32)
        written += [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), True) for t in tensors]
        written.append((g, g + n * G.element_size(), False))
        kept += [G, *tensors]
    written.sort()
    last_in = last_out = 0
    for a, b, out in written:
        if a < last_out or (out and a < last_in):
            raise ValueError("two tensors of the step overlap")
        if out:
            last_out = max(last_out, b)
        else:
            last_in = max(last_in, b)
    _here(*kept)
    plan = dab_adamw_plan()
    _check("dab_adamw_plan_of", lib().dab_adamw_plan_of(arr, len(arr), ctypes.byref(plan)))
    table = torch.empty(plan.table_bytes, dtype=torch.uint8, device=device)
    _check("dab_adamw_table", lib().dab_adamw_table(arr, ctypes.byref(plan), table.data_ptr(), table.numel(), _stream()))
    if not torch.cuda.is_current_stream_capturing():
        torch.cuda.current_stream().synchronize()
    return _AdamwJobs(table, plan, kept)


def dab_adamw(jobs, lr, step, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=None, seed=0):
    """A step of AdamW for every job of adamw_jobs(), in place.

    lr, step (from 1 on): numbers, or tensors of one element on the GPU (fp32, int64) that a captured graph reads anew at every replay; grad_scale: an
    fp32 tensor of one element that multiplies all gradients (infinite or a NaN: nothing is changed).  seed: of the random numbers that 8-bit states
    are rounded by, with the step."""
    if (_native or native()).adamw(jobs.table, jobs.plan, lr, step, beta1, beta2, eps, grad_scale, seed):
        return
    lr_dev = _flat(lr, 1, (torch.float32,), "lr") if isinstance(lr, torch.Tensor) else None
    step_dev = _flat(step, 1, (torch.int64,), "step") if isinstance(step, torch.Tensor) else None
    scale = _flat(grad_scale, 1, (torch.float32,), "grad_scale") if grad_scale is not None else None
    _here(jobs.table, grad_scale, *(t for t in (lr, step) if isinstance(t, torch.Tensor)))
    s = dab_adamw_step(0.0 if lr_dev else lr, beta1, beta2, eps, 1 if step_dev else step, seed, lr_dev, step_dev, scale)
    _check("dab_adamw", lib().dab_adamw(jobs.table.data_ptr(), jobs.table.numel(), ctypes.byref(jobs.plan), ctypes.byref(s), _stream()))


def _state8(Q, S, name):
    groups = S.numel() if isinstance(S, torch.Tensor) else 0
    return _flat(Q, 32 * groups, (torch.uint8,), name), _flat(S, groups, (torch.uint8,), f"{name}'s scales"), 32 * groups


def dab_state8_restore(Q, S, is_signed, dtype=torch.float32, n=None, out=None):
    """What an 8-bit state stands for (is_signed: a first moment, else the root of a second one), of its first n elements (all unless given)."""
    if n is None and out is None:
        done = (_native or native()).state8_restore(Q, S, is_signed, dtype)
        if done is not None:
            return done
    q, s, most = _state8(Q, S, "Q")
    n = most if n is None else n
    if not most - 32 < n <= most:
        raise ValueError(f"n: expected {most - 31} .. {most}, got {n}")
    if dtype not in _REAL:
        raise TypeError(f"dtype: expected torch.float32, torch.bfloat16 or torch.float16, got {dtype}")
    X = _result(out, (n,), dtype, Q.device, "out")
    _here(Q, S, X)
    _check("dab_state8_restore", lib().dab_state8_restore(q, s, n, int(bool(is_signed)), X.data_ptr(), _REAL[dtype], _stream()))
    return X


def dab_state8_save(X, is_signed, out=None):
    """Numbers (fp32, any shape) as an 8-bit state, to the nearest code -> (Q uint8 [32 groups], S uint8 [groups])."""
    n = X.numel()
    x = _flat(X, n, (torch.float32,), "X")
    groups = (n + 31) // 32
    Q, S = out if out is not None else (None, None)
    Q, S = _result(Q, (32 * groups,), torch.uint8, X.device, "Q"), _result(S, (groups,), torch.uint8, X.device, "S")
    _here(X, Q, S)
    _check("dab_state8_save", lib().dab_state8_save(x, n, int(bool(is_signed)), Q.data_ptr(), S.data_ptr(), _stream()))
    return Q, S


def _adapters(X, ids, A, B, scale, F):
    """The arguments that the calls with adapters share, checked: (address, type, distance of X's rows), ids, A, B, scale, n, r."""
    x, dtype, ld = _matrix(X, "X")
    T, K = X.shape
    if not isinstance(A, torch.Tensor) or A.dim() != 3:
        raise ValueError("A: expected three dimensions")
    n, r = A.shape[0], A.shape[1]
    if F is None:
        if not isinstance(B, torch.Tensor) or B.dim() != 3:
            raise ValueError("B: expected three dimensions")
        F = B.shape[2]
    a, b = _ptr(_shaped(A, (n, r, K), "A"), X.dtype, "A"), _ptr(_shaped(B, (n, r, F), "B"), X.dtype, "B")
    i = _ptr(_shaped(ids, (T,), "ids"), torch.int32, "ids")
    s = None if scale is None else _ptr(_shaped(scale, (n,), "scale"), torch.float32, "scale")
    if None in (a, b, i):
        raise TypeError("A, B and ids: expected tensors on the GPU")
    for t, name in ((A, "A"), (B, "B")):
        _counted(t, name)
    _here(X, ids, A, B, scale)
    return (x, dtype, ld), i, a, b, s, T, K, F, n, r


def dab_adapters(X, ids, A, B, scale=None, base=None, out=None):
    """base + scale_i (X A_i^T) B_i for every token's adapter i = ids[t] (none unless 0 <= i < n) -> (Y [T, F] of X's type, U fp32 [T, r]).

    X [T, K]; ids int32 [T]; A [n, r, K] and B [n, r, F] of X's type; scale fp32 [n] or None for ones; base [T, F] of X's type or fp32, or None for
    zeros.  out: (Y, U) to write into, None where a tensor is to be new; Y may be base."""
    done = (_native or native()).adapters(X, ids, A, B, scale, base, out)
    if done is not None:
        return done
    (x, dtype, ld), i, a, b, s, T, K, F, n, r = _adapters(X, ids, A, B, scale, None)
    p, base_dtype, ldb = _beside(base, (T, F), (X.dtype, torch.float32), "base")
    Y, U = out if out is not None else (None, None)
    _here(base, Y, U)
    Y, U = _result(Y, (T, F), X.dtype, X.device, "Y"), _result(U, (T, r), torch.float32, X.device, "U")
    _check("dab_adapters", lib().dab_adapters(x, dtype, ld, i, a, b, s, T, K, F, n, r, p, base_dtype, ldb, Y.data_ptr(), U.data_ptr(), _stream()))
    return Y, U


def dab_adapters_gradient(dY, X, U, ids, A, B, scale=None, base=None, want_dX=True, out=None, ws=None):
    """(dX [T, K] of X's type, dA fp32 [n, r, K], dB fp32 [n, r, F]) of dab_adapters(), with U from it.

    base [T, K] of X's type or fp32: what dX is added to (the shared projection's gradient), or None.  want_dX=False: dX is None.  out: (dX, dA, dB) to
    write into, None where a tensor is to be new; dX may be base."""
    done = (_native or native()).adapters_gradient(dY, X, U, ids, A, B, scale, base, want_dX, out, ws)
    if done is not None:
        return done
    (x, dtype, ld), i, a, b, s, T, K, F, n, r = _adapters(X, ids, A, B, scale, None)
    dy, _, lddy = _beside(dY, (T, F), (X.dtype,), "dY")
    if dy is None:
        raise TypeError("dY: expected a tensor on the GPU")
    u = _ptr(_shaped(U, (T, r), "U"), torch.float32, "U")
    p, base_dtype, ldb = _beside(base, (T, K), (X.dtype, torch.float32), "base")
    if base is not None and not want_dX:
        raise ValueError("base: there is no dX to add it to")
    dX, dA, dB = out if out is not None else (None, None, None)
    _here(dY, U, base, dX, dA, dB)
    dX = _result(dX, (T, K), X.dtype, X.device, "dX") if want_dX else None
    dA, dB = _result(dA, (n, r, K), torch.float32, X.device, "dA"), _result(dB, (n, r, F), torch.float32, X.device, "dB")
    ws, at, nbytes = _scratch(lib().dab_adapters_gradient_workspace_bytes(T, K, F, n, r), X.device, ws)
    _check("dab_adapters_gradient", lib().dab_adapters_gradient(dy, lddy, x, dtype, ld, u, i, a, b, s, T, K, F, n, r, p, base_dtype, ldb,
                                                                dX.data_ptr() if want_dX else None, dA.data_ptr(), dB.data_ptr(), at, nbytes,
                                                                _stream()))
    return dX, dA, dB


def dab_w4_adapters(X, Q, S, F, ids, A, B, scale=None, out=None, ws=None):
    """X [T, K] times the F packed rows, plus every token's adapter (arguments as of dab_w4_matvec() and dab_adapters()) -> Y [T, F] of X's type."""
    done = (_native or native()).w4_adapters(X, Q, S, F, ids, A, B, scale, out, ws)
    if done is not None:
        return done
    (x, dtype, ld), i, a, b, s, T, K, F, n, r = _adapters(X, ids, A, B, scale, F)
    q, sc = _packed(Q, S, F, K)
    _here(Q, S, out)
    Y = _result(out, (T, F), X.dtype, X.device, "out")
    ws, at, nbytes = _scratch(lib().dab_w4_adapters_workspace_bytes(T, K, F, r, dtype, ld), X.device, ws)
    _check("dab_w4_adapters", lib().dab_w4_adapters(x, dtype, ld, q, sc, i, a, b, s, T, K, F, n, r, Y.data_ptr(), at, nbytes, _stream()))
    return Y
