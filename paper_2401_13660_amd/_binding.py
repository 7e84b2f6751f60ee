"""Python binding of libmbscan.so: argument marshalling only.

Every step of the scan runs in the HIP kernels behind the C ABI declared in
``include/mbscan.h``; this module checks torch tensors, allocates outputs with
torch (device memory and streams are all PyTorch is used for) and passes raw
device pointers plus the current HIP stream.  There is no fallback: without the
built library every call raises ``MBScanError``.
"""
from __future__ import annotations

import contextlib
import ctypes
import math
import os
import warnings

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libmbscan.so")

MB_F32, MB_BF16, MB_FP8 = 0, 1, 2
_STATUS_OK = 0


class MBScanError(RuntimeError):
    pass


class ScanDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("dim", ctypes.c_int64), ("seqlen", ctypes.c_int64),
                ("dstate", ctypes.c_int64), ("in_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32),
                ("delta_softplus", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class ConvDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("dim", ctypes.c_int64), ("seqlen", ctypes.c_int64),
                ("width", ctypes.c_int32), ("in_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32),
                ("apply_silu", ctypes.c_int32), ("reserved", ctypes.c_int32), ("reserved2", ctypes.c_int32)]


class MatmulDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("m", ctypes.c_int64), ("n", ctypes.c_int64), ("k", ctypes.c_int64),
                ("a_batched", ctypes.c_int32), ("b_batched", ctypes.c_int32), ("a_tile", ctypes.c_int32),
                ("b_tile", ctypes.c_int32), ("out_dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


_lib = None
_fast = None            # the native entry points for well-formed calls (csrc/fastcall.cpp)
_VP = ctypes.c_void_p


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load (once) and return the HIP library; raise loudly if it is not built."""
    global _lib, _fast
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise MBScanError(f"{path} is not built; run `python -m paper_2401_13660_amd.build` "
                          "(or __graft_entry__.build()) first")
    lib = ctypes.CDLL(path)
    lib.mb_scan_fwd.restype = ctypes.c_int
    lib.mb_scan_fwd.argtypes = [ctypes.POINTER(ScanDesc)] + [_VP] * 12
    lib.mb_scan_fwd_noalloc.restype = ctypes.c_int
    lib.mb_scan_fwd_noalloc.argtypes = [ctypes.POINTER(ScanDesc)] + [_VP] * 12
    lib.mb_scan_fwd_states.restype = ctypes.c_int
    lib.mb_scan_fwd_states.argtypes = [ctypes.POINTER(ScanDesc)] + [_VP] * 11 + [_VP, ctypes.c_int64, _VP, _VP]
    lib.mb_scan_step.restype = ctypes.c_int
    lib.mb_scan_step.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int32] * 3 + [_VP] * 11
    lib.mb_conv1d_fwd.restype = ctypes.c_int
    lib.mb_conv1d_fwd.argtypes = [ctypes.POINTER(ConvDesc)] + [_VP] * 7
    lib.mb_conv1d_step.restype = ctypes.c_int
    lib.mb_conv1d_step.argtypes = [ctypes.c_int64] * 2 + [ctypes.c_int32] * 4 + [_VP] * 6
    lib.mb_scan_bwd.restype = ctypes.c_int
    lib.mb_scan_bwd.argtypes = [ctypes.POINTER(ScanDesc)] + [_VP] * 22
    lib.mb_scan_fwd_ckpt.restype = ctypes.c_int
    lib.mb_scan_fwd_ckpt.argtypes = [ctypes.POINTER(ScanDesc)] + [_VP] * 13
    lib.mb_verify_rank.restype = ctypes.c_int
    lib.mb_verify_rank.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int32] * 2 + [_VP] * 6
    i64, i32, f32 = ctypes.c_int64, ctypes.c_int32, ctypes.c_float
    lib.mb_embedding_fwd.restype = ctypes.c_int
    lib.mb_embedding_fwd.argtypes = [i64] * 3 + [i32] * 3 + [f32] + [_VP] * 4
    lib.mb_embedding_bwd.restype = ctypes.c_int
    lib.mb_embedding_bwd.argtypes = [i64] * 3 + [i32] * 3 + [f32] + [_VP] * 5
    lib.mb_conv1d_bwd.restype = ctypes.c_int
    lib.mb_conv1d_bwd.argtypes = [ctypes.POINTER(ConvDesc)] + [_VP] * 12
    lib.mb_grad_norm.restype = ctypes.c_int
    lib.mb_grad_norm.argtypes = [i64] + [_VP] * 6
    lib.mb_clip_grad_norm.restype = ctypes.c_int
    lib.mb_clip_grad_norm.argtypes = [i64] + [_VP] * 4 + [f32] * 2 + [_VP] * 3
    for size, args in ((lib.mb_embedding_bwd_workspace, [i64] * 3), (lib.mb_grad_norm_workspace, [i64]), (lib.mb_verify_sample_workspace, [i64] * 3),
                       (lib.mb_conv1d_bwd_workspace, [ctypes.POINTER(ConvDesc)])):
        size.restype, size.argtypes = i64, args
    lib.mb_verify_sample.restype = ctypes.c_int
    lib.mb_verify_sample.argtypes = [i64] * 3 + [i32, f32] + [_VP] * 12
    lib.mb_rms_norm_fwd.restype = ctypes.c_int
    lib.mb_rms_norm_fwd.argtypes = [i64] * 2 + [i32] * 3 + [f32] + [_VP] * 8
    lib.mb_rms_norm_bwd.restype = ctypes.c_int
    lib.mb_rms_norm_bwd.argtypes = [i64] * 2 + [i32] * 3 + [_VP] * 10
    lib.mb_rms_norm_bwd_workspace.restype = i64
    lib.mb_rms_norm_bwd_workspace.argtypes = [i64] * 2
    lib.mb_quantize_fp8.restype = ctypes.c_int
    lib.mb_quantize_fp8.argtypes = [i64] * 3 + [i32] * 3 + [_VP] * 4
    lib.mb_matmul_fp8.restype = ctypes.c_int
    lib.mb_matmul_fp8.argtypes = [ctypes.POINTER(MatmulDesc)] + [_VP] * 6
    lib.mb_sample.restype = ctypes.c_int
    lib.mb_sample.argtypes = [i64] * 2 + [i32, f32, i32, f32, f32] + [_VP] * 9
    lib.mb_status_string.restype = ctypes.c_char_p
    lib.mb_status_string.argtypes = [ctypes.c_int]
    lib.mb_abi_version.restype = ctypes.c_int
    _fast = _load_fast(lib)
    _lib = lib
    return lib


def _load_fast(lib):
    """The module built from csrc/fastcall.cpp, calling the functions of ``lib``.  It takes
    the calls whose tensors are plain, dense, of the expected shapes and on the current
    device, does what the functions below do with them, and returns None for any other.
    Where it is not built, or against another torch, the Python code takes every call."""
    if _raw_stream is None or _cur_device is None:
        return None
    try:
        from . import _fastcall
    except ImportError as e:
        why = str(e)
    else:
        built_for = getattr(_fastcall, "torch_version", None)
        why = None if built_for == torch.__version__ else f"built for torch {built_for}, not {torch.__version__}"
    if why is not None:
        warnings.warn(f"the native entry points of the binding are not used ({why}): calls are marshalled in Python. "
                      "`python -m paper_2401_13660_amd.build` builds them.", RuntimeWarning, stacklevel=3)
        return None
    at = [ctypes.cast(fn, _VP).value for fn in (lib.mb_scan_fwd, lib.mb_scan_fwd_states, lib.mb_scan_fwd_ckpt,
                                                lib.mb_scan_step, lib.mb_conv1d_fwd, lib.mb_conv1d_step,
                                                lib.mb_verify_rank, lib.mb_embedding_fwd, lib.mb_embedding_bwd,
                                                lib.mb_embedding_bwd_workspace, lib.mb_conv1d_bwd,
                                                lib.mb_conv1d_bwd_workspace, lib.mb_grad_norm,
                                                lib.mb_grad_norm_workspace, lib.mb_clip_grad_norm,
                                                lib.mb_verify_sample, lib.mb_verify_sample_workspace,
                                                lib.mb_rms_norm_fwd, lib.mb_rms_norm_bwd, lib.mb_rms_norm_bwd_workspace,
                                                lib.mb_quantize_fp8, lib.mb_matmul_fp8, lib.mb_sample)]
    _fastcall.setup(*at, _cur_device, _raw_stream, torch.nn.Parameter)
    return _fastcall


def _done(res, what):
    """The result of a native entry point: what it returned, or the library's refusal."""
    if type(res) is int:
        _check(res, what)
    return res


def _check(status: int, what: str):
    if status != _STATUS_OK:
        msg = load_library().mb_status_string(status).decode()
        raise MBScanError(f"{what} failed with status {status}: {msg}")


def _dt(t: torch.dtype) -> int:
    if t == torch.float32:
        return MB_F32
    if t == torch.bfloat16:
        return MB_BF16
    raise MBScanError(f"unsupported element type {t}; use float32 or bfloat16")


def _ptr(t):
    return None if t is None else t.data_ptr()


# Per-call host work bounds a decode step called from Python (the kernel of a
# one-byte step takes a few microseconds): well-formed calls go through _fastcall.
# What it does not take comes here, and the stream and device lookups use torch's raw
# accessors where it has them.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_cur_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(dev):
    """The raw HIP stream torch currently uses on device ``dev``."""
    if _raw_stream is not None and dev.index is not None:
        return _raw_stream(dev.index)
    return torch.cuda.current_stream(dev).cuda_stream


def _on_device(dev):
    """A context making ``dev`` current for the call; nothing if it already is."""
    cur = _cur_device() if _cur_device is not None else torch.cuda.current_device()
    return contextlib.nullcontext() if dev.index == cur else torch.cuda.device(dev)


def _need(t, name, shape, dtype=None, device=None):
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.shape == shape and (dtype is None or t.dtype == dtype)
            and (device is None or t.device == device) and t.is_contiguous()):
        return
    if not isinstance(t, torch.Tensor):
        raise MBScanError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise MBScanError(f"{name} must be a GPU tensor")
    if device is not None and t.device != device:
        raise MBScanError(f"{name} is on {t.device}, expected {device}")
    if tuple(t.shape) != tuple(shape):
        raise MBScanError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if dtype is not None and t.dtype != dtype:
        raise MBScanError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if not t.is_contiguous():
        raise MBScanError(f"{name} must be contiguous")


def scan_fwd(u, delta, A, B, C, D=None, dt_bias=None, z=None, h0=None, *, delta_softplus=True,
             out_dtype=torch.float32, return_last_state=False, out=None, h_last=None,
             positions=None, h_at=None, return_ckpt=False, ck=None):
    """Selective scan over (batch, dim, L) inputs; returns y or (y, h_last).

    u, delta, z: (batch, dim, L); B, C: (batch, N, L), all of one dtype (fp32 or bf16);
    A: (dim, N) fp32; D, dt_bias: (dim,) fp32; h0: (batch, dim, N) fp32.

    ``positions``: int32 (npos, batch) on the GPU; position k of batch element b is a
    timestep in [0, L) or -1 (the initial state).  The states there are returned as a
    last extra element ``h_at`` of shape (npos, batch, dim, N) (NaN for a position
    outside [-1, L-1]); ``h_at[k]`` can be passed back as ``h0`` to resume.

    ``return_ckpt`` (or a given ``ck``): also store the backward's checkpoints, the
    state before every 16th timestep, as a last extra element of shape
    (L // 16, batch, dim, N) (mb_scan_fwd_ckpt; not combined with positions).
    """
    lib = load_library()
    if _fast is not None:
        res = _fast.scan_fwd(u, delta, A, B, C, D, dt_bias, z, h0, delta_softplus, out_dtype, return_last_state, out,
                             h_last, positions, h_at, return_ckpt, ck)
        if res is not None:
            return _done(res, "mb_scan_fwd_ckpt" if return_ckpt or ck is not None
                         else "mb_scan_fwd" if positions is None else "mb_scan_fwd_states")
    if not isinstance(u, torch.Tensor) or u.dim() != 3:
        raise MBScanError("u must be a (batch, dim, L) tensor")
    nb, dim, L = u.shape
    if not isinstance(A, torch.Tensor) or A.dim() != 2:
        raise MBScanError("A must be a (dim, N) tensor")
    N = A.shape[1]
    dev, act = u.device, u.dtype
    _need(u, "u", (nb, dim, L), act, dev)
    _need(delta, "delta", (nb, dim, L), act, dev)
    _need(A, "A", (dim, N), torch.float32, dev)
    _need(B, "B", (nb, N, L), act, dev)
    _need(C, "C", (nb, N, L), act, dev)
    if z is not None:
        _need(z, "z", (nb, dim, L), act, dev)
    if D is not None:
        _need(D, "D", (dim,), torch.float32, dev)
    if dt_bias is not None:
        _need(dt_bias, "dt_bias", (dim,), torch.float32, dev)
    if h0 is not None:
        _need(h0, "h0", (nb, dim, N), torch.float32, dev)
    if out is None:
        out = torch.empty((nb, dim, L), dtype=out_dtype, device=dev)
    else:
        _need(out, "out", (nb, dim, L), None, dev)
    if return_last_state and h_last is None:
        h_last = torch.empty((nb, dim, N), dtype=torch.float32, device=dev)
    elif h_last is not None:
        _need(h_last, "h_last", (nb, dim, N), torch.float32, dev)
    npos = 0
    if positions is not None:
        if not isinstance(positions, torch.Tensor) or positions.dim() != 2:
            raise MBScanError("positions must be an int32 (npos, batch) tensor")
        npos = positions.shape[0]
        _need(positions, "positions", (npos, nb), torch.int32, dev)
        if h_at is None:
            h_at = torch.empty((npos, nb, dim, N), dtype=torch.float32, device=dev)
        else:
            _need(h_at, "h_at", (npos, nb, dim, N), torch.float32, dev)
    elif h_at is not None:
        raise MBScanError("h_at given without positions")
    want_ck = return_ckpt or ck is not None
    if want_ck:
        if positions is not None:
            raise MBScanError("checkpoints and positions are not recorded by the same call")
        if ck is None:
            ck = torch.empty((L // 16, nb, dim, N), dtype=torch.float32, device=dev)
        else:
            _need(ck, "ck", (L // 16, nb, dim, N), torch.float32, dev)
    desc = ScanDesc(nb, dim, L, N, _dt(act), _dt(out.dtype), 1 if delta_softplus else 0, 0)
    stream = _stream(dev)
    with _on_device(dev):
        if want_ck:
            st = lib.mb_scan_fwd_ckpt(ctypes.byref(desc), _ptr(u), _ptr(delta), _ptr(A), _ptr(B), _ptr(C),
                                      _ptr(D), _ptr(dt_bias), _ptr(z), _ptr(h0), _ptr(out), _ptr(h_last),
                                      _ptr(ck), stream)
        elif positions is None:
            st = lib.mb_scan_fwd(ctypes.byref(desc), _ptr(u), _ptr(delta), _ptr(A), _ptr(B), _ptr(C),
                                 _ptr(D), _ptr(dt_bias), _ptr(z), _ptr(h0), _ptr(out), _ptr(h_last),
                                 stream)
        else:
            st = lib.mb_scan_fwd_states(ctypes.byref(desc), _ptr(u), _ptr(delta), _ptr(A), _ptr(B),
                                        _ptr(C), _ptr(D), _ptr(dt_bias), _ptr(z), _ptr(h0), _ptr(out),
                                        _ptr(h_last), _ptr(positions), npos, _ptr(h_at), stream)
    _check(st, "mb_scan_fwd_ckpt" if want_ck else "mb_scan_fwd" if positions is None else "mb_scan_fwd_states")
    res = (out,)
    if return_last_state or h_last is not None:
        res += (h_last,)
    if positions is not None:
        res += (h_at,)
    if want_ck:
        res += (ck,)
    return res[0] if len(res) == 1 else res


def scan_fwd_noalloc(u, delta, A, B, C, D=None, dt_bias=None, z=None, h0=None, *, out, h_last=None,
                     delta_softplus=True):
    """scan_fwd through mb_scan_fwd_noalloc: nothing is allocated, so the output y
    (``out``) and, if wanted, ``h_last`` are given by the caller (h_last may be h0).
    Returns y or (y, h_last)."""
    lib = load_library()
    if not isinstance(u, torch.Tensor) or u.dim() != 3 or not isinstance(A, torch.Tensor) or A.dim() != 2:
        raise MBScanError("u must be a (batch, dim, L) tensor and A a (dim, N) tensor")
    nb, dim, L = u.shape
    N = A.shape[1]
    dev, act = u.device, u.dtype
    for t, name, shape, dt in ((u, "u", (nb, dim, L), act), (delta, "delta", (nb, dim, L), act),
                               (A, "A", (dim, N), torch.float32), (B, "B", (nb, N, L), act),
                               (C, "C", (nb, N, L), act)):
        _need(t, name, shape, dt, dev)
    for t, name, shape, dt in ((z, "z", (nb, dim, L), act), (D, "D", (dim,), torch.float32),
                               (dt_bias, "dt_bias", (dim,), torch.float32),
                               (h0, "h0", (nb, dim, N), torch.float32),
                               (h_last, "h_last", (nb, dim, N), torch.float32)):
        if t is not None:
            _need(t, name, shape, dt, dev)
    if not isinstance(out, torch.Tensor) or out.dtype not in (torch.float32, torch.bfloat16):
        raise MBScanError("out must be a float32 or bfloat16 tensor")
    _need(out, "out", (nb, dim, L), out.dtype, dev)
    desc = ScanDesc(nb, dim, L, N, _dt(act), _dt(out.dtype), 1 if delta_softplus else 0, 0)
    with _on_device(dev):
        st = lib.mb_scan_fwd_noalloc(ctypes.byref(desc), _ptr(u), _ptr(delta), _ptr(A), _ptr(B), _ptr(C),
                                     _ptr(D), _ptr(dt_bias), _ptr(z), _ptr(h0), _ptr(out), _ptr(h_last),
                                     _stream(dev))
    _check(st, "mb_scan_fwd_noalloc")
    return out if h_last is None else (out, h_last)


def scan_step(h, u_t, delta_t, A, B_t, C_t, D=None, dt_bias=None, z_t=None, *, delta_softplus=True,
              out_dtype=torch.float32, out=None):
    """One recurrent step; h (batch, dim, N) fp32 is updated in place.  Returns y_t (batch, dim)."""
    lib = load_library()
    if _fast is not None:
        res = _fast.scan_step(h, u_t, delta_t, A, B_t, C_t, D, dt_bias, z_t, delta_softplus, out_dtype, out)
        if res is not None:
            return _done(res, "mb_scan_step")
    if not isinstance(h, torch.Tensor) or h.dim() != 3:
        raise MBScanError("h must be a (batch, dim, N) tensor")
    nb, dim, N = h.shape
    dev, act = h.device, u_t.dtype
    _need(h, "h", (nb, dim, N), torch.float32, dev)
    _need(u_t, "u_t", (nb, dim), act, dev)
    _need(delta_t, "delta_t", (nb, dim), act, dev)
    _need(A, "A", (dim, N), torch.float32, dev)
    _need(B_t, "B_t", (nb, N), act, dev)
    _need(C_t, "C_t", (nb, N), act, dev)
    if z_t is not None:
        _need(z_t, "z_t", (nb, dim), act, dev)
    if D is not None:
        _need(D, "D", (dim,), torch.float32, dev)
    if dt_bias is not None:
        _need(dt_bias, "dt_bias", (dim,), torch.float32, dev)
    if out is None:
        out = torch.empty((nb, dim), dtype=out_dtype, device=dev)
    else:
        _need(out, "out", (nb, dim), None, dev)
    stream = _stream(dev)
    with _on_device(dev):
        st = lib.mb_scan_step(nb, dim, N, _dt(act), _dt(out.dtype), 1 if delta_softplus else 0,
                              _ptr(u_t), _ptr(delta_t), _ptr(A), _ptr(B_t), _ptr(C_t), _ptr(D),
                              _ptr(dt_bias), _ptr(z_t), _ptr(h), _ptr(out), stream)
    _check(st, "mb_scan_step")
    return out


def conv1d(x, w, bias=None, state=None, *, apply_silu=True, out_dtype=None, return_state=False,
           out=None, state_out=None):
    """Causal depthwise convolution (+ Swish) of x (batch, dim, L) with taps w (dim, k).

    bias: (dim,) fp32; state: (batch, dim, k-1) fp32, the k-1 inputs before x (zeros when
    None).  Returns y, or (y, state_out) where state_out holds the last k-1 inputs.
    """
    lib = load_library()
    if _fast is not None:
        res = _fast.conv1d(x, w, bias, state, apply_silu, out_dtype, return_state, out, state_out)
        if res is not None:
            return _done(res, "mb_conv1d_fwd")
    if not isinstance(x, torch.Tensor) or x.dim() != 3:
        raise MBScanError("x must be a (batch, dim, L) tensor")
    nb, dim, L = x.shape
    if not isinstance(w, torch.Tensor) or w.dim() != 2:
        raise MBScanError("w must be a (dim, k) tensor")
    K = w.shape[1]
    dev = x.device
    _need(x, "x", (nb, dim, L), None, dev)
    _need(w, "w", (dim, K), torch.float32, dev)
    if bias is not None:
        _need(bias, "bias", (dim,), torch.float32, dev)
    if state is not None:
        _need(state, "state", (nb, dim, K - 1), torch.float32, dev)
    if out is None:
        out = torch.empty((nb, dim, L), dtype=out_dtype or x.dtype, device=dev)
    else:
        _need(out, "out", (nb, dim, L), None, dev)
    if return_state and state_out is None:
        state_out = torch.empty((nb, dim, max(K - 1, 0)), dtype=torch.float32, device=dev)
    elif state_out is not None:
        _need(state_out, "state_out", (nb, dim, K - 1), torch.float32, dev)
    desc = ConvDesc(nb, dim, L, K, _dt(x.dtype), _dt(out.dtype), 1 if apply_silu else 0, 0, 0)
    stream = _stream(dev)
    with _on_device(dev):
        st = lib.mb_conv1d_fwd(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(bias), _ptr(state), _ptr(out),
                               _ptr(state_out) if K > 1 else None, stream)
    _check(st, "mb_conv1d_fwd")
    return (out, state_out) if (return_state or state_out is not None) else out


def conv1d_step(state, x_t, w, bias=None, *, apply_silu=True, out_dtype=None, out=None):
    """One byte of the convolution; state (batch, dim, k-1) fp32 is updated in place.
    Returns y_t (batch, dim)."""
    lib = load_library()
    if _fast is not None:
        res = _fast.conv1d_step(state, x_t, w, bias, apply_silu, out_dtype, out)
        if res is not None:
            return _done(res, "mb_conv1d_step")
    if not isinstance(x_t, torch.Tensor) or x_t.dim() != 2:
        raise MBScanError("x_t must be a (batch, dim) tensor")
    nb, dim = x_t.shape
    if not isinstance(w, torch.Tensor) or w.dim() != 2:
        raise MBScanError("w must be a (dim, k) tensor")
    K = w.shape[1]
    dev = x_t.device
    _need(x_t, "x_t", (nb, dim), None, dev)
    _need(w, "w", (dim, K), torch.float32, dev)
    if bias is not None:
        _need(bias, "bias", (dim,), torch.float32, dev)
    if K > 1:
        _need(state, "state", (nb, dim, K - 1), torch.float32, dev)
    if out is None:
        out = torch.empty((nb, dim), dtype=out_dtype or x_t.dtype, device=dev)
    else:
        _need(out, "out", (nb, dim), None, dev)
    stream = _stream(dev)
    with _on_device(dev):
        st = lib.mb_conv1d_step(nb, dim, K, _dt(x_t.dtype), _dt(out.dtype), 1 if apply_silu else 0,
                                _ptr(x_t), _ptr(w), _ptr(bias), _ptr(state) if K > 1 else None,
                                _ptr(out), stream)
    _check(st, "mb_conv1d_step")
    return out


def verify_rank(logits, draft, beta, *, return_ranks=False):
    """Top-beta check of drafted bytes.  logits: (batch, ndraft, vocab) fp32 or bf16;
    draft: int32 (batch, ndraft).  Returns (accepted, last_pos), each int32 (batch,),
    and the int32 (batch, ndraft) ranks when ``return_ranks``."""
    lib = load_library()
    if _fast is not None:
        res = _fast.verify_rank(logits, draft, beta, return_ranks)
        if res is not None:
            return _done(res, "mb_verify_rank")
    if not isinstance(logits, torch.Tensor) or logits.dim() != 3:
        raise MBScanError("logits must be a (batch, ndraft, vocab) tensor")
    nb, n, V = logits.shape
    dev = logits.device
    _need(logits, "logits", (nb, n, V), None, dev)
    _need(draft, "draft", (nb, n), torch.int32, dev)
    accepted = torch.empty(nb, dtype=torch.int32, device=dev)
    last_pos = torch.empty(nb, dtype=torch.int32, device=dev)
    ranks = torch.empty((nb, n), dtype=torch.int32, device=dev) if return_ranks else None
    stream = _stream(dev)
    with _on_device(dev):
        st = lib.mb_verify_rank(nb, n, V, _dt(logits.dtype), int(beta), _ptr(logits), _ptr(draft),
                                _ptr(ranks), _ptr(accepted), _ptr(last_pos), stream)
    _check(st, "mb_verify_rank")
    return (accepted, last_pos, ranks) if return_ranks else (accepted, last_pos)


def scan_bwd(u, delta, A, B, C, dy, D=None, dt_bias=None, z=None, h0=None, dh_last=None, *,
             delta_softplus=True, ck=None):
    """Gradients of sum(dy * y) + sum(dh_last * h_last) for the scan of scan_fwd.

    ``ck``: the checkpoints of ``scan_fwd(..., return_ckpt=True)`` on the same inputs;
    without them the call recomputes them with one more forward pass.

    dy has y's dtype (fp32 or bf16), shape (batch, dim, L).  Returns a dict: du, ddelta,
    dz (dy's dtype, (batch, dim, L); dz None without a gate), dA (dim, N), dB, dC
    (batch, N, L), dD and dt_bias gradients ``dD``, ``ddt_bias`` (dim,) or None, and
    dh0 (batch, dim, N), all fp32 but the first three.
    """
    lib = load_library()
    if not isinstance(u, torch.Tensor) or u.dim() != 3:
        raise MBScanError("u must be a (batch, dim, L) tensor")
    nb, dim, L = u.shape
    if not isinstance(A, torch.Tensor) or A.dim() != 2:
        raise MBScanError("A must be a (dim, N) tensor")
    N = A.shape[1]
    dev, act = u.device, u.dtype
    for t, name, shape, dt in ((u, "u", (nb, dim, L), act), (delta, "delta", (nb, dim, L), act),
                               (A, "A", (dim, N), torch.float32), (B, "B", (nb, N, L), act),
                               (C, "C", (nb, N, L), act), (dy, "dy", (nb, dim, L), None)):
        _need(t, name, shape, dt, dev)
    for t, name, shape, dt in ((z, "z", (nb, dim, L), act), (D, "D", (dim,), torch.float32),
                               (dt_bias, "dt_bias", (dim,), torch.float32),
                               (h0, "h0", (nb, dim, N), torch.float32),
                               (dh_last, "dh_last", (nb, dim, N), torch.float32),
                               (ck, "ck", (L // 16, nb, dim, N), torch.float32)):
        if t is not None:
            _need(t, name, shape, dt, dev)
    f32 = dict(dtype=torch.float32, device=dev)
    g = {"du": torch.empty((nb, dim, L), dtype=dy.dtype, device=dev),
         "ddelta": torch.empty((nb, dim, L), dtype=dy.dtype, device=dev),
         "dz": torch.empty((nb, dim, L), dtype=dy.dtype, device=dev) if z is not None else None,
         "dA": torch.empty((dim, N), **f32), "dB": torch.empty((nb, N, L), **f32),
         "dC": torch.empty((nb, N, L), **f32),
         "dD": torch.empty(dim, **f32) if D is not None else None,
         "ddt_bias": torch.empty(dim, **f32) if dt_bias is not None else None,
         "dh0": torch.empty((nb, dim, N), **f32)}
    desc = ScanDesc(nb, dim, L, N, _dt(act), _dt(dy.dtype), 1 if delta_softplus else 0, 0)
    stream = _stream(dev)
    with _on_device(dev):
        st = lib.mb_scan_bwd(ctypes.byref(desc), _ptr(u), _ptr(delta), _ptr(A), _ptr(B), _ptr(C), _ptr(D),
                             _ptr(dt_bias), _ptr(z), _ptr(h0), _ptr(dy), _ptr(dh_last), _ptr(ck),
                             _ptr(g["du"]),
                             _ptr(g["ddelta"]), _ptr(g["dz"]), _ptr(g["dA"]), _ptr(g["dB"]), _ptr(g["dC"]),
                             _ptr(g["dD"]), _ptr(g["ddt_bias"]), _ptr(g["dh0"]), stream)
    _check(st, "mb_scan_bwd")
    return g


def _workspace(size, what, dev):
    """torch's memory for a call's workspace of ``size`` bytes: reused as soon as the stream has passed the call."""
    _check(min(size, 0), what)
    return torch.empty(size, dtype=torch.uint8, device=dev)


def _was_written(tensors):
    """A caller's tensors were written through their addresses: counted, so that autograd refuses a gradient for which it
    had saved one."""
    torch.autograd.graph.increment_version([t for t in tensors if not t.is_inference()])


_TOKEN_TYPES = {torch.uint8: 0, torch.int32: 1, torch.int64: 2}


def _tokens(tokens, dev=None):
    """The tokens' type code; they may have any shape."""
    if not isinstance(tokens, torch.Tensor) or tokens.dtype not in _TOKEN_TYPES:
        raise MBScanError("tokens must be a uint8, int32 or int64 tensor")
    _need(tokens, "tokens", tokens.shape, None, dev)
    return _TOKEN_TYPES[tokens.dtype]


def embedding_fwd(tokens, weight, *, scale=1.0, out_dtype=None, out=None):
    """scale * weight[tokens]: tokens uint8, int32 or int64 of any shape, weight (vocab, dim) fp32 or bf16.
    Returns tokens.shape + (dim,) in ``out_dtype`` (weight's by default).  A negative token (padding) gives
    zeros, a token >= vocab NaN."""
    lib = load_library()
    if _fast is not None:
        res = _fast.embedding_fwd(tokens, weight, scale, out_dtype, out)
        if res is not None:
            return _done(res, "mb_embedding_fwd")
    if not isinstance(weight, torch.Tensor) or weight.dim() != 2:
        raise MBScanError("weight must be a (vocab, dim) tensor")
    V, d = weight.shape
    dev = weight.device
    _need(weight, "weight", (V, d))
    code = _tokens(tokens, dev)
    shape, given = tuple(tokens.shape) + (d,), out is not None
    if out is None:
        out = torch.empty(shape, dtype=out_dtype or weight.dtype, device=dev)
    else:
        _need(out, "out", shape, None, dev)
    with _on_device(dev):
        st = lib.mb_embedding_fwd(tokens.numel(), V, d, code, _dt(weight.dtype), _dt(out.dtype), float(scale),
                                  _ptr(tokens), _ptr(weight), _ptr(out), _stream(dev))
    _check(st, "mb_embedding_fwd")
    if given:
        _was_written([out])
    return out


def embedding_bwd(tokens, dy, vocab, *, scale=1.0, out_dtype=torch.float32, out=None):
    """The gradient of embedding_fwd's table: (vocab, dim) in ``out_dtype``, row v the sum of scale * dy over
    the tokens equal to v (the same bits on every call).  dy: tokens.shape + (dim,), fp32 or bf16."""
    lib = load_library()
    if _fast is not None:
        res = _fast.embedding_bwd(tokens, dy, vocab, scale, out_dtype, out)
        if res is not None:
            return _done(res, "mb_embedding_bwd")
    if not isinstance(dy, torch.Tensor) or dy.dim() < 1:
        raise MBScanError("dy must be a tensor of the tokens' shape and a last dimension dim")
    dev, d = dy.device, dy.shape[-1]
    code = _tokens(tokens, dev)
    _need(dy, "dy", tuple(tokens.shape) + (d,))
    vocab = int(vocab)
    if vocab < 0:
        raise MBScanError("vocab must not be negative")
    given = out is not None
    if out is None:
        out = torch.empty((vocab, d), dtype=out_dtype, device=dev)
    else:
        _need(out, "out", (vocab, d), None, dev)
    ws = _workspace(lib.mb_embedding_bwd_workspace(tokens.numel(), vocab, d), "mb_embedding_bwd", dev)
    with _on_device(dev):
        st = lib.mb_embedding_bwd(tokens.numel(), vocab, d, code, _dt(dy.dtype), _dt(out.dtype), float(scale),
                                  _ptr(tokens), _ptr(dy), _ptr(out), _ptr(ws), _stream(dev))
    _check(st, "mb_embedding_bwd")
    if given:
        _was_written([out])
    return out


def conv1d_bwd(x, w, dy, bias=None, state=None, dstate_out=None, *, apply_silu=True):
    """Gradients of sum(dy * y) + sum(dstate_out * state_out) for the convolution of conv1d.

    x, w, bias, state as for ``conv1d``; dy has y's dtype, shape (batch, dim, L); dstate_out:
    (batch, dim, k-1) fp32 or None.  Returns a dict: dx (dy's dtype), dw (dim, k), dbias (dim,) or None,
    and dstate (batch, dim, k-1), fp32 but the first."""
    lib = load_library()
    if _fast is not None:
        res = _fast.conv1d_bwd(x, w, dy, bias, state, dstate_out, apply_silu)
        if res is not None:
            return dict(zip(("dx", "dw", "dbias", "dstate"), _done(res, "mb_conv1d_bwd")))
    if not isinstance(x, torch.Tensor) or x.dim() != 3:
        raise MBScanError("x must be a (batch, dim, L) tensor")
    nb, dim, L = x.shape
    if not isinstance(w, torch.Tensor) or w.dim() != 2:
        raise MBScanError("w must be a (dim, k) tensor")
    K, dev = w.shape[1], x.device
    H = max(K - 1, 0)
    for t, name, shape, dt in ((x, "x", (nb, dim, L), None), (w, "w", (dim, K), torch.float32),
                               (dy, "dy", (nb, dim, L), None)):
        _need(t, name, shape, dt, dev)
    for t, name, shape in ((bias, "bias", (dim,)), (state, "state", (nb, dim, H)),
                           (dstate_out, "dstate_out", (nb, dim, H))):
        if t is not None:
            _need(t, name, shape, torch.float32, dev)
    f32 = dict(dtype=torch.float32, device=dev)
    g = {"dx": torch.empty((nb, dim, L), dtype=dy.dtype, device=dev), "dw": torch.empty((dim, K), **f32),
         "dbias": torch.empty(dim, **f32) if bias is not None else None,
         "dstate": torch.empty((nb, dim, H), **f32)}
    desc = ConvDesc(nb, dim, L, K, _dt(x.dtype), _dt(dy.dtype), 1 if apply_silu else 0, 0, 0)
    ws = _workspace(lib.mb_conv1d_bwd_workspace(ctypes.byref(desc)), "mb_conv1d_bwd", dev)
    with _on_device(dev):
        st = lib.mb_conv1d_bwd(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(bias), _ptr(state) if H else None, _ptr(dy),
                               _ptr(dstate_out) if H else None, _ptr(g["dx"]), _ptr(g["dw"]), _ptr(g["dbias"]),
                               _ptr(g["dstate"]) if H else None, _ptr(ws), _stream(dev))
    _check(st, "mb_conv1d_bwd")
    return g


def _grad_list(grads):
    """The tensors of a list, one GPU's and dense: their device, and host arrays of addresses, sizes and types."""
    grads = [grads] if isinstance(grads, torch.Tensor) else list(grads)
    if not grads:
        raise MBScanError("the list of tensors is empty")
    dev = grads[0].device if isinstance(grads[0], torch.Tensor) else None
    for i, t in enumerate(grads):
        if not isinstance(t, torch.Tensor):
            raise MBScanError(f"tensor {i} must be a torch.Tensor")
        _need(t, f"tensor {i}", t.shape, None, dev)
    n = len(grads)
    return (grads, dev, (_VP * n)(*(t.data_ptr() for t in grads)), (ctypes.c_int64 * n)(*(t.numel() for t in grads)),
            (ctypes.c_int32 * n)(*(_dt(t.dtype) for t in grads)))


def grad_norm(grads):
    """The 2-norm of all elements of a list of fp32 and bf16 tensors: a 0-dimensional fp32 tensor on their GPU."""
    lib = load_library()
    if _fast is not None:
        res = _fast.grad_norm(grads)
        if res is not None:
            return _done(res, "mb_grad_norm")
    grads, dev, ptrs, sizes, types = _grad_list(grads)
    norm = torch.empty((), dtype=torch.float32, device=dev)
    ws = _workspace(lib.mb_grad_norm_workspace(len(grads)), "mb_grad_norm", dev)
    with _on_device(dev):
        st = lib.mb_grad_norm(len(grads), ptrs, sizes, types, _ptr(norm), _ptr(ws), _stream(dev))
    _check(st, "mb_grad_norm")
    return norm


def clip_grad_norm(grads, max_norm, *, eps=1e-6, out=None):
    """Scales a list of fp32 and bf16 tensors (the gradients, not the parameters) by max_norm / (norm + eps)
    where that is below 1, in place or into ``out`` (tensors of the same shapes and types).  Returns the norm before
    clipping, a 0-dimensional fp32 tensor on the GPU.  The written tensors count as changed for autograd."""
    lib = load_library()
    if _fast is not None:
        res = _fast.clip_grad_norm(grads, max_norm, eps, out)
        if res is not None:
            return _done(res, "mb_clip_grad_norm")
    grads, dev, ptrs, sizes, types = _grad_list(grads)
    optrs = None
    if out is not None:
        out = [out] if isinstance(out, torch.Tensor) else list(out)
        if len(out) != len(grads):
            raise MBScanError(f"out has {len(out)} tensors, expected {len(grads)}")
        for i, (o, t) in enumerate(zip(out, grads)):
            _need(o, f"out {i}", t.shape, t.dtype, dev)
        optrs = (_VP * len(out))(*(o.data_ptr() for o in out))
    if any(t.requires_grad for t in (grads if out is None else out)):
        raise MBScanError("gradients are clipped, not the parameters: a tensor that would be written requires grad")
    norm = torch.empty((), dtype=torch.float32, device=dev)
    ws = _workspace(lib.mb_grad_norm_workspace(len(grads)), "mb_clip_grad_norm", dev)
    with _on_device(dev):
        st = lib.mb_clip_grad_norm(len(grads), ptrs, optrs, sizes, types, float(max_norm), float(eps), _ptr(norm),
                                   _ptr(ws), _stream(dev))
    _check(st, "mb_clip_grad_norm")
    _was_written(grads if out is None else out)
    return norm


def verify_sample(logits, draft, uniform, noise, draft_logits=None, *, lengths=None, temperature=1.0,
                  return_probs=False):
    """Drafted tokens against the target's probabilities, from given random numbers.

    logits: (batch, ndraft + 1, vocab) fp32 or bf16, row i scoring drafted token i and the row after the last
    one the token that follows; draft: int32 (batch, ndraft); uniform: fp32 (batch, ndraft) in [0, 1);
    noise: fp32 (batch, vocab), exponential of mean 1; draft_logits: (batch, ndraft, vocab) of logits' type, or
    None for drafts without probabilities; lengths: int32 (batch,), the tokens drafted for each sequence.
    Returns (accepted, last_pos, next_token), each int32 (batch,), and with ``return_probs`` the target's
    probabilities of the drafted tokens, fp32 (batch, ndraft).  With ndraft = 0 it samples the next token."""
    lib = load_library()
    if _fast is not None:
        res = _fast.verify_sample(logits, draft, uniform, noise, draft_logits, lengths, temperature, return_probs)
        if res is not None:
            return _done(res, "mb_verify_sample")
    if not isinstance(logits, torch.Tensor) or logits.dim() != 3 or logits.shape[1] < 1:
        raise MBScanError("logits must be a (batch, ndraft + 1, vocab) tensor")
    nb, n, V = logits.shape[0], logits.shape[1] - 1, logits.shape[2]
    dev = logits.device
    _need(logits, "logits", (nb, n + 1, V))
    _need(draft, "draft", (nb, n), torch.int32, dev)
    _need(uniform, "uniform", (nb, n), torch.float32, dev)
    _need(noise, "noise", (nb, V), torch.float32, dev)
    if draft_logits is not None:
        _need(draft_logits, "draft_logits", (nb, n, V), logits.dtype, dev)
    if lengths is not None:
        _need(lengths, "lengths", (nb,), torch.int32, dev)
    accepted, last_pos, next_token = (torch.empty(nb, dtype=torch.int32, device=dev) for _ in range(3))
    probs = torch.empty((nb, n), dtype=torch.float32, device=dev) if return_probs else None
    size = lib.mb_verify_sample_workspace(nb, n, V)
    ws = _workspace(size, "mb_verify_sample", dev) if size else None
    with _on_device(dev):
        st = lib.mb_verify_sample(nb, n, V, _dt(logits.dtype), float(temperature), _ptr(logits), _ptr(draft_logits),
                                  _ptr(draft), _ptr(lengths), _ptr(uniform), _ptr(noise), _ptr(accepted),
                                  _ptr(last_pos), _ptr(next_token), _ptr(probs), _ptr(ws), _stream(dev))
    _check(st, "mb_verify_sample")
    return (accepted, last_pos, next_token, probs) if return_probs else (accepted, last_pos, next_token)


FP8 = torch.float8_e4m3fn
_BLOCK = 128                # values that share a scale


def _blocks(n):
    return -(-n // _BLOCK)


def _norm_inputs(x, weight, residual):
    """The checks that both forms of the norm share: rows and columns."""
    if not isinstance(x, torch.Tensor) or x.dim() < 1:
        raise MBScanError("x must be a (..., dim) tensor")
    dev, d = x.device, x.shape[-1]
    _need(x, "x", x.shape)
    if weight is not None:
        _need(weight, "weight", (d,), torch.float32, dev)
    if residual is not None:
        _need(residual, "residual", x.shape, None, dev)
    return math.prod(x.shape[:-1]), d, dev


def _norm(x, weight, residual, eps, code, y, scales, residual_out, rstd, rows, d, dev):
    lib = load_library()
    with _on_device(dev):
        st = lib.mb_rms_norm_fwd(rows, d, _dt(x.dtype), 0 if residual is None else _dt(residual.dtype), code, float(eps),
                                 _ptr(x), _ptr(weight), _ptr(residual), _ptr(y), _ptr(scales), _ptr(residual_out), _ptr(rstd),
                                 _stream(dev))
    _check(st, "mb_rms_norm_fwd")


def _residual_out(residual, given, dev):
    """The tensor for h, and whether it is the caller's."""
    if residual is None:
        if given is not None:
            raise MBScanError("residual_out given without a residual")
        return None
    if given is None:
        return torch.empty_like(residual)
    _need(given, "residual_out", residual.shape, residual.dtype, dev)
    return given


def rms_norm_fwd(x, weight=None, residual=None, *, eps=1e-5, out_dtype=None, return_rstd=False, out=None, residual_out=None):
    """h = x + residual (in residual's type) and y = h / sqrt(mean(h^2) + eps) * weight over the last dimension.

    x: (..., dim) fp32 or bf16; weight: (dim,) fp32 or None; residual: x's shape, fp32 or bf16, or None.
    ``residual_out`` may be ``residual``: h takes its place.  Returns y in ``out_dtype`` (x's by default), or (y, h)
    with a residual; ``return_rstd`` appends 1 / sqrt(mean(h^2) + eps), fp32 of x's leading shape, for ``rms_norm_bwd``."""
    load_library()
    if _fast is not None:
        res = _fast.rms_norm_fwd(x, weight, residual, eps, out_dtype, return_rstd, out, residual_out)
        if res is not None:
            return _done(res, "mb_rms_norm_fwd")
    rows, d, dev = _norm_inputs(x, weight, residual)
    given = [t for t in (out, residual_out) if t is not None]
    if out is None:
        out = torch.empty(x.shape, dtype=out_dtype or x.dtype, device=dev)
    else:
        _need(out, "out", x.shape, None, dev)
    h = _residual_out(residual, residual_out, dev)
    rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=dev) if return_rstd else None
    _norm(x, weight, residual, eps, _dt(out.dtype), out, None, h, rstd, rows, d, dev)
    if given:
        _was_written(given)
    res = (out,) + ((h,) if residual is not None else ()) + ((rstd,) if return_rstd else ())
    return res[0] if len(res) == 1 else res


def rms_norm_fp8(x, weight=None, residual=None, *, eps=1e-5, residual_out=None):
    """rms_norm_fwd with y in 8 bits, as ``matmul_fp8`` takes it.  Returns (q, scale) or, with a residual, (q, scale, h):
    q (..., dim) float8_e4m3fn, scale (..., ceil(dim / 128)) fp32, y being q times its block's scale."""
    load_library()
    if _fast is not None:
        res = _fast.rms_norm_fp8(x, weight, residual, eps, residual_out)
        if res is not None:
            return _done(res, "mb_rms_norm_fwd")
    rows, d, dev = _norm_inputs(x, weight, residual)
    q = torch.empty(x.shape, dtype=FP8, device=dev)
    scale = torch.empty(x.shape[:-1] + (_blocks(d),), dtype=torch.float32, device=dev)
    h = _residual_out(residual, residual_out, dev)
    _norm(x, weight, residual, eps, MB_FP8, q, scale, h, None, rows, d, dev)
    if residual_out is not None:
        _was_written([residual_out])
    return (q, scale) if residual is None else (q, scale, h)


def rms_norm_bwd(dy, h, rstd, weight=None, dh=None, *, dx_dtype=None):
    """Gradients of sum(dy * y) + sum(dh * h) for rms_norm_fwd.

    dy: (..., dim) in y's type; h: the forward's h (x without a residual); rstd: the forward's; dh: h's shape and
    type, the gradient that reaches h from behind, or None.  Returns a dict: dx in ``dx_dtype`` (dy's by default),
    dweight (dim,) fp32 (None without a weight) and, with dh, dresidual in h's type (the tensor dx itself where that is
    dx's type)."""
    lib = load_library()
    if _fast is not None:
        res = _fast.rms_norm_bwd(dy, h, rstd, weight, dh, dx_dtype)
        if res is not None:
            res = dict(zip(("dx", "dweight", "dresidual"), _done(res, "mb_rms_norm_bwd")))
            if dh is None:
                del res["dresidual"]
            return res
    if not isinstance(h, torch.Tensor) or h.dim() < 1:
        raise MBScanError("h must be a (..., dim) tensor")
    dev, d = h.device, h.shape[-1]
    _need(h, "h", h.shape)
    _need(dy, "dy", h.shape, None, dev)
    _need(rstd, "rstd", h.shape[:-1], torch.float32, dev)
    if weight is not None:
        _need(weight, "weight", (d,), torch.float32, dev)
    if dh is not None:
        _need(dh, "dh", h.shape, h.dtype, dev)
    rows = rstd.numel()
    dx = torch.empty(h.shape, dtype=dx_dtype or dy.dtype, device=dev)
    g = {"dx": dx, "dweight": None if weight is None else torch.empty(d, dtype=torch.float32, device=dev)}
    apart = dh is not None and h.dtype != dx.dtype
    if dh is not None:
        g["dresidual"] = torch.empty_like(h) if apart else dx
    ws = _workspace(lib.mb_rms_norm_bwd_workspace(rows, d), "mb_rms_norm_bwd", dev) if weight is not None else None
    with _on_device(dev):
        st = lib.mb_rms_norm_bwd(rows, d, _dt(dy.dtype), _dt(h.dtype), _dt(dx.dtype), _ptr(dy), _ptr(h), _ptr(rstd), _ptr(weight),
                                 _ptr(dh), _ptr(dx), _ptr(g["dresidual"]) if apart else None, _ptr(g["dweight"]), _ptr(ws),
                                 _stream(dev))
    _check(st, "mb_rms_norm_bwd")
    return g


def quantize_fp8(x, *, tile=False, transpose=False):
    """Matrices (..., rows, cols), fp32 or bf16, in 8 bits: (q, scale), q float8_e4m3fn of x's shape and scale fp32
    (..., rows, ceil(cols / 128)), or with ``tile`` (..., ceil(rows / 128), ceil(cols / 128)).  ``transpose``: the same of
    x's transposed matrices, q (..., cols, rows)."""
    lib = load_library()
    if _fast is not None:
        res = _fast.quantize_fp8(x, tile, transpose)
        if res is not None:
            return _done(res, "mb_quantize_fp8")
    if not isinstance(x, torch.Tensor) or x.dim() < 2:
        raise MBScanError("x must be a (..., rows, cols) tensor")
    _need(x, "x", x.shape)
    dev, lead = x.device, tuple(x.shape[:-2])
    rows, cols = x.shape[-2:]
    R, C = (cols, rows) if transpose else (rows, cols)
    q = torch.empty(lead + (R, C), dtype=FP8, device=dev)
    scale = torch.empty(lead + (_blocks(R) if tile else R, _blocks(C)), dtype=torch.float32, device=dev)
    batch = 1
    for n in lead:
        batch *= n
    with _on_device(dev):
        st = lib.mb_quantize_fp8(batch, rows, cols, _dt(x.dtype), 1 if tile else 0, 1 if transpose else 0, _ptr(x), _ptr(q),
                                 _ptr(scale), _stream(dev))
    _check(st, "mb_quantize_fp8")
    return q, scale


def _matrix(t, s, name, dev):
    """An 8-bit matrix or a batch of them with its scales: batch (None without), rows, and whether scales are of tiles."""
    if not isinstance(t, torch.Tensor) or t.dim() not in (2, 3):
        raise MBScanError(f"{name} must be a (rows, k) or (batch, rows, k) tensor")
    _need(t, name, t.shape, FP8, dev)
    lead, (rows, k) = tuple(t.shape[:-2]), t.shape[-2:]
    by_row, by_tile = lead + (rows, _blocks(k)), lead + (_blocks(rows), _blocks(k))
    tile = isinstance(s, torch.Tensor) and tuple(s.shape) == by_tile and by_tile != by_row
    _need(s, f"{name}_scale", by_tile if tile else by_row, torch.float32, dev)
    return (lead[0] if lead else None), rows, tile


def matmul_fp8(a, a_scale, b, b_scale, *, out_dtype=torch.bfloat16, out=None):
    """c[m][n] = sum over k of a[m][k] b[n][k], values being 8 bits times their scales.

    a: (m, k) or (batch, m, k), b: (n, k) or (batch, n, k), float8_e4m3fn, with the scales of ``quantize_fp8`` (per row
    or per tile, told by their shape) or ``rms_norm_fp8``.  Returns (m, n), or (batch, m, n) if either has a batch, in
    ``out_dtype``: fp32 or bf16."""
    lib = load_library()
    if _fast is not None:
        res = _fast.matmul_fp8(a, a_scale, b, b_scale, out_dtype, out)
        if res is not None:
            return _done(res, "mb_matmul_fp8")
    dev = a.device if isinstance(a, torch.Tensor) else None
    a_batch, m, a_tile = _matrix(a, a_scale, "a", dev)
    b_batch, n, b_tile = _matrix(b, b_scale, "b", dev)
    k = a.shape[-1]
    if b.shape[-1] != k:
        raise MBScanError(f"b has {b.shape[-1]} columns, expected {k}")
    if a_batch is not None and b_batch is not None and a_batch != b_batch:
        raise MBScanError(f"b is a batch of {b_batch}, expected {a_batch}")
    batch = a_batch if a_batch is not None else b_batch
    shape = ((batch,) if batch is not None else ()) + (m, n)
    given = out is not None
    if out is None:
        out = torch.empty(shape, dtype=out_dtype, device=dev)
    else:
        _need(out, "out", shape, None, dev)
    desc = MatmulDesc(1 if batch is None else batch, m, n, k, a_batch is not None, b_batch is not None, a_tile, b_tile,
                      _dt(out.dtype), 0)
    with _on_device(dev):
        st = lib.mb_matmul_fp8(ctypes.byref(desc), _ptr(a), _ptr(a_scale), _ptr(b), _ptr(b_scale), _ptr(out), _stream(dev))
    _check(st, "mb_matmul_fp8")
    if given:
        _was_written([out])
    return out


def sample(logits, noise, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, return_prob=False):
    """The next token of each sequence from its filtered probabilities and given random numbers.

    logits: (batch, vocab) fp32 or bf16; noise: fp32 (batch, vocab), exponential of mean 1.  ``temperature`` (0: the
    largest logit), ``top_k`` (<= 0: all), ``top_p`` (>= 1: all) and ``min_p`` (<= 0: all) are numbers, or tensors (batch,)
    on the GPU, fp32 (top_k: int32), of one for each sequence.  Filters apply in this order; equal logits rank by
    their index.  Returns the tokens, int32 (batch,), -1 for a row that is no distribution; ``return_prob`` adds the
    probabilities that they were drawn with, fp32 (batch,)."""
    lib = load_library()
    if _fast is not None:
        res = _fast.sample(logits, noise, temperature, top_k, top_p, min_p, return_prob)
        if res is not None:
            return _done(res, "mb_sample")
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2:
        raise MBScanError("logits must be a (batch, vocab) tensor")
    nb, V = logits.shape
    dev = logits.device
    _need(logits, "logits", (nb, V))
    _need(noise, "noise", (nb, V), torch.float32, dev)
    each = {}
    for name, v, dt in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32),
                        ("top_p", top_p, torch.float32), ("min_p", min_p, torch.float32)):
        if isinstance(v, torch.Tensor):
            _need(v, name, (nb,), dt, dev)
            each[name] = v
    one = {n: d if n in each else v for n, v, d in (("temperature", temperature, 1.0), ("top_k", top_k, 0),
                                                    ("top_p", top_p, 1.0), ("min_p", min_p, 0.0))}
    token = torch.empty(nb, dtype=torch.int32, device=dev)
    prob = torch.empty(nb, dtype=torch.float32, device=dev) if return_prob else None
    with _on_device(dev):
        st = lib.mb_sample(nb, V, _dt(logits.dtype), float(one["temperature"]), min(max(int(one["top_k"]), 0), 2 ** 31 - 1),
                           float(one["top_p"]), float(one["min_p"]), *(_ptr(each.get(n)) for n in
                                                                       ("temperature", "top_k", "top_p", "min_p")),
                           _ptr(logits), _ptr(noise), _ptr(token), _ptr(prob), _stream(dev))
    _check(st, "mb_sample")
    return (token, prob) if return_prob else token
