"""Thin Python binding of libchela's C ABI (argument marshalling only).

Each function mirrors the C entry point of the same name: it reads shapes and device pointers
from torch tensors, allocates the output and the workspace with torch, and passes torch's
current CUDA stream.  Every step of the computation runs in the library's kernels.  There is no
CPU fallback: if ``libchela.so`` has not been built (``python -m paper_2406_08128_b200.build``)
loading fails with an error.
"""
from __future__ import annotations

import collections
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libchela.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = range(6)
F32, BF16, BF16_PAIR = 0, 1, 2
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
ZERO_REST = 256   # CHELA_ZERO_REST

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}
_lib = None

_c_int, _c_float, _c_size_t, _vp = ctypes.c_int, ctypes.c_float, ctypes.c_size_t, ctypes.c_void_p
_c_ll = ctypes.c_longlong


class SelscanArgs(ctypes.Structure):
    """chela_selscan_args_t"""
    _fields_ = [(n, _vp) for n in ("x", "dt", "b", "c", "z")] \
        + [(n, _c_ll) for n in ("x_stride", "dt_stride", "b_stride", "c_stride", "z_stride")] \
        + [(n, _vp) for n in ("a", "d_skip", "dt_bias", "state_in", "seq_offsets")] \
        + [(n, _c_int) for n in ("S", "T", "D", "N", "G", "softplus", "in_dtype")]


class BlocknormArgs(ctypes.Structure):
    """chela_blocknorm_args_t"""
    _fields_ = [(n, _vp) for n in ("res", "y", "gate")] + [(n, _c_ll) for n in ("res_stride", "y_stride", "gate_stride")] \
        + [(n, _vp) for n in ("w_post", "b_post", "scale", "w_pre", "b_pre")] \
        + [(n, _c_int) for n in ("T", "D", "gate_act", "gate_after", "norm_post", "norm_pre")] + [("eps", _c_float)] \
        + [(n, _c_int) for n in ("in_dtype", "res_dtype")]


_SIGNATURES = {
    "chela_status_string": (ctypes.c_char_p, [_c_int]),
    "chela_version": (_c_int, []),
    "chela_linattn_kernel_kind": (_c_int, [_c_int] * 6 + [_c_int, _c_int]),
    "chela_shortconv_fwd": (_c_int, [_vp, _vp, _vp, _vp, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _vp]),
    "chela_second_short_width": (_c_int, [_c_int]),
    "chela_shortconv_reparam": (_c_int, [_vp, _c_int, _vp, _c_int, _vp, _c_int, _vp]),
    "chela_longconv_workspace_bytes": (_c_size_t, [_c_int, _c_int, _c_int, _c_int, _c_int]),
    "chela_longconv_fwd": (_c_int, [_vp, _vp, _vp, _c_int, _vp, _c_int, _c_int, _c_int, _c_int, _c_int,
                                    _vp, _c_size_t, _vp]),
    "chela_linattn_workspace_bytes": (_c_size_t, [_c_int] * 6),
    "chela_linattn_fwd": (_c_int, [_vp, _vp, _vp, _vp] + [_c_int] * 6 + [_c_int, _c_int, _c_int, _c_float,
                                   _c_float, _vp, _c_size_t, _vp]),
    "chela_linattn_carry_fwd": (_c_int, [_vp, _vp, _vp, _vp, _vp, _vp] + [_c_int] * 6 + [_c_int, _c_int, _c_int, _c_float,
                                         _c_float, _vp, _c_size_t, _vp]),
    "chela_linattn_split_plan": (_c_int, [_c_int] * 6 + [_vp, _vp, _vp]),
    "chela_linattn_step": (_c_int, [_vp] * 5 + [_c_int] * 4 + [_c_int, _c_int, _c_int, _c_float, _c_float, _vp]),
    "chela_linattn_bwd_workspace_bytes": (_c_size_t, [_c_int] * 5),
    "chela_linattn_bwd": (_c_int, [_vp] * 7 + [_c_int] * 5 + [_c_int, _c_int, _c_float, _c_float, _vp, _c_size_t, _vp]),
    "chela_dense_workspace_bytes": (_c_size_t, []),
    "chela_dense_fwd": (_c_int, [_vp, _vp, _vp, _vp, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _vp,
                                 _c_size_t, _vp]),
    "chela_async_status": (_c_int, [_vp, _vp]),
    "chela_debug_wait_control": (None, [ctypes.c_longlong, _c_int]),
    "chela_debug_sm_clock": (_c_int, [_vp, ctypes.c_longlong, _vp]),
    "chela_linattn_static_ws_status": (_c_int, [_vp]),
    "chela_linattn_fwd_static_ws": (_c_int, [_vp, _vp, _vp, _vp] + [_c_int] * 6 + [_c_int, _c_int, _c_int, _c_float,
                                             _c_float, _vp]),
    "chela_mixer_workspace_bytes": (_c_size_t, [_c_int] * 5 + [_c_int]),
    "chela_mixer_gated_workspace_bytes": (_c_size_t, [_c_int] * 5 + [_c_int]),
    "chela_mixer_gated_fwd": (_c_int, [_vp, _vp, _c_int, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_int, _c_int,
                                       _vp, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_float,
                                       _vp, _c_size_t, _vp]),
    "chela_longconv_spectrum_bytes": (_c_size_t, [_c_int, _c_int]),
    "chela_longconv_prepare": (_c_int, [_vp, _c_int, _c_int, _vp, _c_size_t, _vp]),
    "chela_longconv_prepared_fwd": (_c_int, [_vp, _vp, _vp, _c_int, _vp, _c_int, _c_int, _c_int, _c_int, _c_int, _vp, _c_size_t, _vp]),
    "chela_mixer_prepared_fwd": (_c_int, [_vp, _vp, _c_int, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_int, _c_int,
                                          _vp, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_float,
                                          _vp, _c_size_t, _vp]),
    "chela_mixer_fwd": (_c_int, [_vp, _vp, _c_int, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _c_int, _c_int, _vp,
                                 _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_float,
                                 _vp, _c_size_t, _vp]),
    "chela_shortconv_carry_fwd": (_c_int, [_vp, _c_ll] + [_vp] * 6 + [_c_int] * 5 + [_c_int, _vp]),
    "chela_shortconv_step": (_c_int, [_vp, _c_ll] + [_vp] * 5 + [_c_int] * 4 + [_c_int, _vp]),
    "chela_shortconv_bwd_workspace_bytes": (_c_size_t, [_c_int] * 3),
    "chela_shortconv_bwd": (_c_int, [_vp, _c_ll, _vp, _vp, _vp, _c_ll] + [_vp] * 7 + [_c_int] * 7 + [_vp, _c_size_t, _vp]),
    "chela_selscan_checkpoint_bytes": (_c_size_t, [_c_int] * 4),
    "chela_selscan_workspace_bytes": (_c_size_t, [_c_int] * 4),
    "chela_selscan_fwd": (_c_int, [_vp] * 4 + [_c_int, _vp, _c_size_t, _vp]),
    "chela_selscan_step": (_c_int, [_vp] * 3 + [_c_int, _vp]),
    "chela_selscan_bwd_workspace_bytes": (_c_size_t, [_c_int] * 5),
    "chela_selscan_bwd": (_c_int, [_vp, _vp, _c_ll] + [_vp] * 11 + [_c_int, _vp, _c_size_t, _vp]),
    "chela_blocknorm_fwd": (_c_int, [_vp] * 3 + [_c_int, _vp]),
    "chela_blocknorm_bwd_workspace_bytes": (_c_size_t, [_c_int] * 2),
    "chela_blocknorm_bwd": (_c_int, [_vp] * 11 + [_c_int, _vp, _c_size_t, _vp]),
}


class ChelaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (status %d)" % (where, status_string(status), status))


def exported_symbols():
    """Names the C header declares (the loader resolves every one of them)."""
    return sorted(_SIGNATURES)


def lib():
    """Load libchela.so (once).  Raises if the library has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libchela.so is missing: build it with `python -m paper_2406_08128_b200.build` "
                               "(there is no CPU fallback)")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype, fn.argtypes = res, args
        _lib = handle
    return _lib


def status_string(status: int) -> str:
    return lib().chela_status_string(int(status)).decode()


def version() -> int:
    return int(lib().chela_version())


def _check(status: int, where: str):
    if status != OK:
        raise ChelaError(int(status), where)


def _ptr(t):
    return None if t is None else _vp(t.data_ptr())


def _stream():
    return _vp(torch.cuda.current_stream().cuda_stream)


def _dt(t) -> int:
    return _DTYPES[t.dtype]


def _tdtype(code: int):
    return torch.float32 if code == F32 else torch.bfloat16


def _workspace(nbytes: int, device):
    return torch.empty(max(int(nbytes), 16), dtype=torch.uint8, device=device)


def linattn_kernel_kind(B, H, L, d_k, d_v, chunk, in_dtype=BF16, out_dtype=F32) -> int:
    return int(lib().chela_linattn_kernel_kind(B, H, L, d_k, d_v, chunk, in_dtype, out_dtype))


def shortconv_fwd(x, w, bias=None, act=True, out=None):
    """x [B,L,D] (bf16/f32), w [D,width] f32 -> y like x."""
    B, L, D = x.shape
    y = torch.empty_like(x) if out is None else out
    _check(lib().chela_shortconv_fwd(_ptr(x), _ptr(w), _ptr(bias), _ptr(y), B, L, D, w.shape[1], int(bool(act)),
                                     _dt(x), _stream()), "chela_shortconv_fwd")
    return y


def second_short_width(L: int) -> int:
    """Width of the length-dependent short kernel, 2 log10(L) + 1 rounded to the nearest odd integer."""
    return int(lib().chela_second_short_width(int(L)))


def shortconv_reparam(w1, w2):
    """Merge two parallel short kernels [D,width1], [D,width2] (fp32) into one [D,max(width)] kernel."""
    D = w1.shape[0]
    merged = torch.empty((D, max(w1.shape[1], w2.shape[1])), dtype=torch.float32, device=w1.device)
    _check(lib().chela_shortconv_reparam(_ptr(w1), w1.shape[1], _ptr(w2), w2.shape[1], _ptr(merged), D, _stream()),
           "chela_shortconv_reparam")
    return merged


def longconv_workspace_bytes(B, L, D, in_dtype=BF16, out_dtype=F32) -> int:
    return int(lib().chela_longconv_workspace_bytes(B, L, D, in_dtype, out_dtype))


def longconv_fwd(x, k_long, w_short=None, out_dtype=F32, out=None, workspace=None):
    """x [B,L,D], k_long [D,L] f32, optional short taps [D,width] f32 -> z [B,L,D] of out_dtype."""
    B, L, D = x.shape
    z = torch.empty((B, L, D), dtype=_tdtype(out_dtype), device=x.device) if out is None else out
    if workspace is None:
        workspace = _workspace(longconv_workspace_bytes(B, L, D, _dt(x), out_dtype), x.device)
    width = 0 if w_short is None else w_short.shape[1]
    _check(lib().chela_longconv_fwd(_ptr(x), _ptr(k_long), _ptr(w_short), width, _ptr(z), B, L, D, _dt(x),
                                    _dt(z), _ptr(workspace), workspace.numel(), _stream()), "chela_longconv_fwd")
    return z


def linattn_workspace_bytes(B, H, L, d_k, d_v, chunk) -> int:
    return int(lib().chela_linattn_workspace_bytes(B, H, L, d_k, d_v, chunk))


def linattn_fwd(q, k, v, chunk=64, out_dtype=F32, norm=NORM_RMS, eps=1e-6, scale=1.0, out=None, workspace=None,
                in_dtype=None):
    """q,k [B,L,H,d_k], v [B,L,H,d_v] -> o [B,L,H,d_v] of out_dtype.

    With in_dtype=BF16_PAIR q, k, v are [2,B,L,H,d] bf16 tensors (high plane, low plane)."""
    in_dtype = _dt(q) if in_dtype is None else in_dtype
    B, L, H, d_k = q.shape[-4:]
    d_v = v.shape[-1]
    o = torch.empty((B, L, H, d_v), dtype=_tdtype(out_dtype), device=q.device) if out is None else out
    if workspace is None:
        workspace = _workspace(linattn_workspace_bytes(B, H, L, d_k, d_v, chunk), q.device)
    _check(lib().chela_linattn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), B, H, L, d_k, d_v, chunk, in_dtype, _dt(o),
                                   int(norm), float(eps), float(scale), _ptr(workspace), workspace.numel(),
                                   _stream()), "chela_linattn_fwd")
    return o


def linattn_carry_fwd(q, k, v, state_in=None, chunk=64, out_dtype=F32, norm=NORM_RMS, eps=1e-6, scale=1.0, out=None,
                      state_out=None, workspace=None, in_dtype=None):
    """chela_linattn_carry_fwd: returns (o, state_out); state tensors are [B,H,d_k,d_v] fp32."""
    in_dtype = _dt(q) if in_dtype is None else in_dtype
    B, L, H, d_k = q.shape[-4:]
    d_v = v.shape[-1]
    o = torch.empty((B, L, H, d_v), dtype=_tdtype(out_dtype), device=q.device) if out is None else out
    if state_out is None:
        state_out = torch.empty((B, H, d_k, d_v), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = _workspace(linattn_workspace_bytes(B, H, L, d_k, d_v, chunk), q.device)
    _check(lib().chela_linattn_carry_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(state_in), _ptr(state_out), B, H, L,
                                         d_k, d_v, chunk, in_dtype, _dt(o), int(norm), float(eps), float(scale),
                                         _ptr(workspace), workspace.numel(), _stream()), "chela_linattn_carry_fwd")
    return o, state_out


def linattn_split_plan(B, H, L, d=64, in_dtype=BF16, sms=0):
    """chela_linattn_split_plan: (groups, first_chunks, other_chunks), or None if no tensor-core kernel takes d."""
    g, c0, c = ctypes.c_int(0), ctypes.c_int(0), ctypes.c_int(0)
    ok = lib().chela_linattn_split_plan(B, H, L, d, int(in_dtype), int(sms), ctypes.byref(g), ctypes.byref(c0), ctypes.byref(c))
    return (g.value, c0.value, c.value) if ok else None


def linattn_step(q, k, v, state, out_dtype=F32, norm=NORM_RMS, eps=1e-6, scale=1.0, out=None):
    """chela_linattn_step: one token per sequence; q, k, v [B,H,d]; state [B,H,d,d] fp32 is updated in place."""
    B, H, d_k = q.shape
    d_v = v.shape[2]
    o = torch.empty((B, H, d_v), dtype=_tdtype(out_dtype), device=q.device) if out is None else out
    _check(lib().chela_linattn_step(_ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(state), B, H, d_k, d_v, _dt(q), _dt(o),
                                    int(norm), float(eps), float(scale), _stream()), "chela_linattn_step")
    return o


def linattn_bwd(q, k, v, d_o, norm=NORM_RMS, eps=1e-6, scale=1.0, workspace=None):
    """Gradients (dq, dk, dv), fp32, of linattn_fwd for the output gradient d_o (same dtype as q)."""
    B, L, H, d_k = q.shape
    d_v = v.shape[3]
    dq, dk, dv = (torch.empty(t.shape, dtype=torch.float32, device=q.device) for t in (q, k, v))
    if workspace is None:
        workspace = _workspace(int(lib().chela_linattn_bwd_workspace_bytes(B, H, L, d_k, d_v)), q.device)
    _check(lib().chela_linattn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(d_o), _ptr(dq), _ptr(dk), _ptr(dv), B, H, L, d_k, d_v,
                                   _dt(q), int(norm), float(eps), float(scale), _ptr(workspace), workspace.numel(),
                                   _stream()), "chela_linattn_bwd")
    return dq, dk, dv


def linattn_fwd_static_ws(q, k, v, chunk=64, out_dtype=F32, norm=NORM_RMS, eps=1e-6, scale=1.0, out=None):
    """chela_linattn_fwd_static_ws: same result as linattn_fwd, scratch from the library's built-in array.

    For hosts that cannot allocate device memory; here torch still allocates the output unless ``out`` is
    given, the library call itself allocates nothing.
    """
    B, L, H, d_k = q.shape
    d_v = v.shape[3]
    o = torch.empty((B, L, H, d_v), dtype=_tdtype(out_dtype), device=q.device) if out is None else out
    _check(lib().chela_linattn_fwd_static_ws(_ptr(q), _ptr(k), _ptr(v), _ptr(o), B, H, L, d_k, d_v, chunk, _dt(q),
                                             _dt(o), int(norm), float(eps), float(scale), _stream()),
           "chela_linattn_fwd_static_ws")
    return o


def dense_fwd(a, w, bias=None, act=False, a_dtype=None, y_dtype=BF16, out=None, workspace=None):
    """y = act(a w + bias).  a [M,K] (a bf16 pair is passed as a [2,M,K] bf16 tensor with a_dtype=BF16_PAIR),
    w [K,N]; returns y [M,N] (or [2,M,N] bf16 for y_dtype=BF16_PAIR)."""
    a_dtype = _dt(a) if a_dtype is None else a_dtype
    M, K = a.shape[-2], a.shape[-1]
    N = w.shape[1]
    if out is None:
        shape = (2, M, N) if y_dtype == BF16_PAIR else (M, N)
        out = torch.empty(shape, dtype=torch.float32 if y_dtype == F32 else torch.bfloat16, device=a.device)
    if workspace is None:
        workspace = _workspace(int(lib().chela_dense_workspace_bytes()), a.device)
    _check(lib().chela_dense_fwd(_ptr(a), _ptr(w), _ptr(bias), _ptr(out), M, K, N, int(act), a_dtype, _dt(w),
                                 y_dtype, _ptr(workspace), workspace.numel(), _stream()), "chela_dense_fwd")
    return out


def async_status(workspace) -> int:
    """Synchronise the current stream and return the asynchronous status recorded in ``workspace``."""
    return int(lib().chela_async_status(_ptr(workspace), _stream()))


def longconv_prepare(k_long, out=None):
    """chela_longconv_prepare: the spectra of the long kernels k_long [D, L] (and the twiddle table) in a device buffer."""
    D, L = k_long.shape
    n = int(lib().chela_longconv_spectrum_bytes(L, D))
    if n == 0:
        raise ChelaError(ERR_UNSUPPORTED, "chela_longconv_spectrum_bytes")
    spec = torch.empty(n, dtype=torch.uint8, device=k_long.device) if out is None else out
    _check(lib().chela_longconv_prepare(_ptr(k_long), L, D, _ptr(spec), spec.numel(), _stream()), "chela_longconv_prepare")
    return spec


def longconv_prepared_fwd(x, spectrum, w_short=None, out_dtype=F32, out=None, workspace=None):
    """chela_longconv_prepared_fwd: chela_longconv_fwd with prepared spectra in place of the kernels."""
    B, L, D = x.shape
    z = torch.empty((B, L, D), dtype=_tdtype(out_dtype), device=x.device) if out is None else out
    if workspace is None:
        workspace = _workspace(longconv_workspace_bytes(B, L, D, _dt(x), out_dtype), x.device)
    _check(lib().chela_longconv_prepared_fwd(_ptr(x), _ptr(spectrum), _ptr(w_short), 0 if w_short is None else w_short.shape[1],
                                             _ptr(z), B, L, D, _dt(x), _dt(z), _ptr(workspace), workspace.numel(), _stream()),
           "chela_longconv_prepared_fwd")
    return z


def mixer_prepared_fwd(x, w_short, spectrum, w_q, w_k, w_v, H, w_a=None, w_o=None, chunk=64, b_q=None, b_k=None, b_v=None,
                       b_a=None, b_o=None, qk_diag=False, v_silu=True, out_dtype=F32, norm=NORM_RMS, eps=1e-6, out=None,
                       workspace=None):
    """chela_mixer_prepared_fwd: the mixer (gated when w_a and w_o are given) with prepared long-kernel spectra."""
    B, L, D = x.shape
    o = torch.empty((B, L, D), dtype=_tdtype(out_dtype), device=x.device) if out is None else out
    if workspace is None:
        need = mixer_gated_workspace_bytes(B, L, D, H, chunk, _dt(x)) if w_a is not None else mixer_workspace_bytes(B, L, D, H, chunk, _dt(x))
        workspace = _workspace(need, x.device)
    _check(lib().chela_mixer_prepared_fwd(_ptr(x), _ptr(w_short), w_short.shape[1], _ptr(spectrum), _ptr(w_q), _ptr(w_k), _ptr(w_v),
                                          _ptr(b_q), _ptr(b_k), _ptr(b_v), _ptr(w_a), _ptr(b_a), _ptr(w_o), _ptr(b_o), int(qk_diag),
                                          int(v_silu), _ptr(o), B, L, D, H, chunk, _dt(x), _dt(o), int(norm), float(eps),
                                          _ptr(workspace), workspace.numel(), _stream()), "chela_mixer_prepared_fwd")
    return o


def debug_wait_control(limit_cycles=0, skip_arrival=0) -> None:
    """chela_debug_wait_control: the wait limit (SM cycles, 0 = default) and the skipped-arrival test hook."""
    lib().chela_debug_wait_control(int(limit_cycles), int(skip_arrival))


def debug_sm_clock_mhz(spin_cycles=400000, device=None) -> float:
    """chela_debug_sm_clock on the current stream: the SM clock in MHz as SM cycles over global-timer nanoseconds."""
    out = torch.zeros(2, dtype=torch.int64, device=device if device is not None else torch.device("cuda", torch.cuda.current_device()))
    _check(lib().chela_debug_sm_clock(_ptr(out), int(spin_cycles), _stream()), "chela_debug_sm_clock")
    cycles, ns = (int(x) for x in out.cpu())
    return cycles * 1000.0 / max(ns, 1)


def linattn_static_ws_status() -> int:
    """Synchronise the current stream and return the status word of the built-in scratch (current device)."""
    return int(lib().chela_linattn_static_ws_status(_stream()))


def mixer_workspace_bytes(B, L, D, H, chunk, in_dtype=BF16) -> int:
    return int(lib().chela_mixer_workspace_bytes(B, L, D, H, chunk, in_dtype))


def mixer_fwd(x, w_short, k_long, w_q, w_k, w_v, H, chunk=64, b_q=None, b_k=None, b_v=None, qk_diag=False,
              v_silu=True, out_dtype=F32, norm=NORM_RMS, eps=1e-6, out=None, workspace=None):
    """x [B,L,D] -> o [B,L,D]; weights as in the C header."""
    B, L, D = x.shape
    o = torch.empty((B, L, D), dtype=_tdtype(out_dtype), device=x.device) if out is None else out
    if workspace is None:
        workspace = _workspace(mixer_workspace_bytes(B, L, D, H, chunk, _dt(x)), x.device)
    _check(lib().chela_mixer_fwd(_ptr(x), _ptr(w_short), w_short.shape[1], _ptr(k_long), _ptr(w_q), _ptr(w_k),
                                 _ptr(w_v), _ptr(b_q), _ptr(b_k), _ptr(b_v), int(bool(qk_diag)),
                                 int(bool(v_silu)), _ptr(o), B, L, D, H, chunk, _dt(x), _dt(o), int(norm),
                                 float(eps), _ptr(workspace), workspace.numel(), _stream()), "chela_mixer_fwd")
    return o


def mixer_gated_workspace_bytes(B, L, D, H, chunk, in_dtype=BF16) -> int:
    return int(lib().chela_mixer_gated_workspace_bytes(B, L, D, H, chunk, in_dtype))


def mixer_gated_fwd(x, w_short, k_long, w_q, w_k, w_v, w_a, w_o, H, chunk=64, b_q=None, b_k=None, b_v=None, b_a=None,
                    b_o=None, qk_diag=False, v_silu=True, out_dtype=F32, norm=NORM_RMS, eps=1e-6, out=None, workspace=None):
    """x [B,L,D] -> u [B,L,D]: the mixer with its gates G_a, G_o and the residual mix."""
    B, L, D = x.shape
    u = torch.empty((B, L, D), dtype=_tdtype(out_dtype), device=x.device) if out is None else out
    if workspace is None:
        workspace = _workspace(mixer_gated_workspace_bytes(B, L, D, H, chunk, _dt(x)), x.device)
    _check(lib().chela_mixer_gated_fwd(_ptr(x), _ptr(w_short), w_short.shape[1], _ptr(k_long), _ptr(w_q), _ptr(w_k), _ptr(w_v),
                                       _ptr(b_q), _ptr(b_k), _ptr(b_v), _ptr(w_a), _ptr(b_a), _ptr(w_o), _ptr(b_o),
                                       int(bool(qk_diag)), int(bool(v_silu)), _ptr(u), B, L, D, H, chunk, _dt(x), _dt(u),
                                       int(norm), float(eps), _ptr(workspace), workspace.numel(), _stream()),
           "chela_mixer_gated_fwd")
    return u


# ---------------------------------------------------------------------------------------------------------------------
# Operators over packed sequences.  Token tensors are [T, D] (sequences one behind the other, with seq_offsets) or
# [B, L, D] (B sequences of L tokens); the channel axis must be contiguous and consecutive tokens a fixed distance
# apart, so column slices of a wider projection are taken as they are.  All tensors of a call live on one CUDA device;
# the call runs on that device's current stream.  Rows of tokens behind the last sequence (from seq_offsets[-1] on) are not
# read; they are zero in the outputs and gradients that a call allocates and left as they were in an ``out`` that it is given.

ShortconvGrads = collections.namedtuple("ShortconvGrads", "d_x d_w d_bias d_state_in")
SelscanGrads = collections.namedtuple("SelscanGrads", "d_x d_dt d_a d_b d_c d_skip d_z d_dt_bias d_state_in")
_MAX_TOKENS = 2 ** 31 - 4096
_MAX_INT = 2 ** 31 - 1   # of the sizes that the C entry points take as int
BlocknormGrads = collections.namedtuple("BlocknormGrads", "d_res d_y d_gate d_w_post d_b_post d_scale d_w_pre d_b_pre")


def _need(ok, where, what):
    if not ok:
        err = ChelaError(ERR_INVALID_ARG, where)
        err.args = ("%s: %s" % (err.args[0], what),)
        raise err


def _raw_stream(index):
    return torch._C._cuda_getCurrentRawStream(index)


def _rows(t, where, name, lead, dtype, index, inner, shape=None):
    """Address and token stride of a token tensor [*lead, *inner] (= shape, where the caller has it); the inner axes
    contiguous, one step between tokens."""
    if t.dtype is not dtype or t.get_device() != index or t.shape != (shape or lead + inner):
        _need(False, where, "%s must be a %s tensor %s on device %d" % (name, dtype, lead + inner, index))
    if t.is_contiguous():
        return t.data_ptr(), inner[0] if len(inner) == 1 else inner[0] * inner[1]
    n = len(lead)
    strides, step = t.stride(), 1
    for i in range(len(inner) - 1, -1, -1):
        if strides[n + i] != step and inner[i] != 1:
            _need(False, where, "%s: a token's values must be contiguous" % name)
        step *= inner[i]
    if n == 1:
        stride = strides[0] if lead[0] > 1 else -(-step // 8) * 8
    else:
        stride = strides[1] if lead[1] > 1 else (strides[0] if lead[0] > 1 else -(-step // 8) * 8)
        if strides[0] != lead[1] * stride and lead[0] != 1:
            _need(False, where, "%s: tokens must be a fixed distance apart" % name)
    return t.data_ptr(), stride


def _width(w, where):
    """The number of taps of short kernels [D, width]."""
    if w.dim() != 2 or not 1 <= w.shape[1] <= _MAX_INT:
        _need(False, where, "w is [D, width] with a width of at least 1")
    return w.shape[1]


def _flat(t, where, name, shape, dtype, index):
    """Address of an optional contiguous tensor of the given shape."""
    if t is None:
        return None
    if t.dtype is not dtype or t.get_device() != index or t.shape != shape or not t.is_contiguous():
        _need(False, where, "%s must be a contiguous %s tensor %s on device %d" % (name, dtype, tuple(shape), index))
    return t.data_ptr()


def _seqs(x, seq_offsets, where):
    """(leading shape, S, T, address of the offsets, device) of a token tensor."""
    lead = x.shape[:-1]
    if x.dtype not in _DTYPES or len(lead) not in (1, 2):
        _need(False, where, "tokens must be [T, D] or [B, L, D] of float32 or bfloat16")
    T = lead[0] if len(lead) == 1 else lead[0] * lead[1]
    if T > _MAX_TOKENS or x.shape[-1] > _MAX_INT:   # before ctypes cuts them to 32 bits
        _need(False, where, "%d tokens, at most %d, of %d channels, at most %d" % (T, _MAX_TOKENS, x.shape[-1], _MAX_INT))
    if not x.is_cuda:
        _need(False, where, "tensors must be on a CUDA device (there is no CPU fallback)")
    index = x.get_device()
    if seq_offsets is None:
        return lead, 1 if len(lead) == 1 else lead[0], T, None, index
    _need(len(lead) == 1 and seq_offsets.dim() == 1 and 2 <= seq_offsets.shape[0] <= _MAX_INT, where,
          "seq_offsets [S + 1] goes with packed tokens [T, D]")
    return lead, seq_offsets.shape[0] - 1, T, _flat(seq_offsets, where, "seq_offsets", seq_offsets.shape, torch.int32, index), index


def _run(fn, where, index, *args):
    """fn(*args, stream) on the current stream of the call's device."""
    if index == torch._C._cuda_getDevice():
        status = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, _raw_stream(index))
    if status != OK:
        raise ChelaError(int(status), where)


def _new(out, where, name, shape, dtype, device, index):
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _flat(out, where, name, shape, dtype, index)
    return out


def _like(t, dtype):
    """An uninitialised contiguous tensor of t's shape; None for None."""
    return None if t is None else torch.empty_like(t, dtype=dtype, memory_format=torch.contiguous_format)


def _at(t):
    return None if t is None else t.data_ptr()


def _new_like(out, where, name, like, dtype, index):
    """A contiguous output of like's shape."""
    if out is None:
        return _like(like, dtype)
    _flat(out, where, name, like.shape, dtype, index)
    return out


def _scratch(need, workspace, device, where, index):
    """A call's workspace (allocated here unless the caller brings one), its address and its bytes.  The caller keeps the
    tensor until the library's function has returned: that runs without the interpreter's lock, and a block given back
    before could go to another thread whose work is queued before the call's kernels, or between them."""
    if workspace is None:
        if need == 0:
            return None, None, 0
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    elif workspace.get_device() != index or not workspace.is_contiguous():
        _need(False, where, "workspace must be contiguous and on device %d" % index)
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def shortconv_carry_fwd(x, w, bias=None, act=True, state_in=None, state_out=None, seq_offsets=None, out=None):
    """chela_shortconv_carry_fwd: (y, state_out).  x [T,D] or [B,L,D]; w [D,width] f32; states [S,width-1,D] like x."""
    where, f32 = "chela_shortconv_carry_fwd", torch.float32
    lead, S, T, off, dev = _seqs(x, seq_offsets, where)
    D, width, dt = x.shape[-1], _width(w, where), x.dtype
    px, xs = _rows(x, where, "x", lead, dt, dev, (D,), x.shape)
    y = _new_like(out, where, "out", x, dt, dev)
    held = (S, width - 1, D)
    state_out = _new(state_out, where, "state_out", held, dt, x.device, dev)
    _run(lib().chela_shortconv_carry_fwd, where, dev, px, xs, _flat(w, where, "w", (D, width), f32, dev),
         _flat(bias, where, "bias", (D,), f32, dev), y.data_ptr(), _flat(state_in, where, "state_in", held, dt, dev),
         state_out.data_ptr() or None, off, S, T, D, width, int(bool(act)) | (ZERO_REST if out is None else 0), _DTYPES[dt])
    return y, state_out


def shortconv_step(x, w, state, bias=None, act=True, state_out=None, out=None):
    """chela_shortconv_step: y [S,D] for one new token per sequence; state [S,width-1,D] is updated in place unless
    state_out is given."""
    where, f32 = "chela_shortconv_step", torch.float32
    lead, _, S, _, dev = _seqs(x, None, where)
    _need(len(lead) == 1, where, "x must be [S, D]")
    D, width, dt = x.shape[-1], _width(w, where), x.dtype
    px, xs = _rows(x, where, "x", lead, dt, dev, (D,), x.shape)
    y = _new_like(out, where, "out", x, dt, dev)
    held = (S, width - 1, D)
    before = _flat(state, where, "state", held, dt, dev)
    after = before if state_out is None else _flat(state_out, where, "state_out", held, dt, dev)
    _run(lib().chela_shortconv_step, where, dev, px, xs, _flat(w, where, "w", (D, width), f32, dev),
         _flat(bias, where, "bias", (D,), f32, dev), y.data_ptr(), before or None, after or None, S, D, width, int(bool(act)), _DTYPES[dt])
    return y


def shortconv_bwd(x, w, d_y, bias=None, act=True, state_in=None, d_state_out=None, seq_offsets=None, grad_dtype=F32,
                  want_d_state=False, workspace=None):
    """chela_shortconv_bwd: ShortconvGrads; d_x (and d_state_in, if wanted) of grad_dtype, d_w and d_bias f32."""
    where, f32 = "chela_shortconv_bwd", torch.float32
    lead, S, T, off, dev = _seqs(x, seq_offsets, where)
    D, width, dt, gt, device = x.shape[-1], _width(w, where), x.dtype, _tdtype(grad_dtype), x.device
    px, xs = _rows(x, where, "x", lead, dt, dev, (D,), x.shape)
    pdy, dys = _rows(d_y, where, "d_y", lead, dt, dev, (D,))
    held = (S, width - 1, D)
    g = ShortconvGrads(_like(x, gt), _like(w, f32), torch.empty((D,), dtype=f32, device=device),
                       torch.empty(held, dtype=gt, device=device) if want_d_state else None)
    workspace, ws, nbytes = _scratch(lib().chela_shortconv_bwd_workspace_bytes(T, D, width), workspace, device, where, dev)
    _run(lib().chela_shortconv_bwd, where, dev, px, xs, _flat(w, where, "w", (D, width), f32, dev),
         _flat(bias, where, "bias", (D,), f32, dev), pdy, dys, _flat(state_in, where, "state_in", held, dt, dev),
         _flat(d_state_out, where, "d_state_out", held, dt, dev), g.d_x.data_ptr(), g.d_w.data_ptr(), g.d_bias.data_ptr(),
         _at(g.d_state_in), off, S, T, D, width, int(bool(act)), _DTYPES[dt], int(grad_dtype), ws, nbytes)
    return g


def _selscan_args(where, x, dt, a, b, c, d_skip, z, dt_bias, softplus, state_in, seq_offsets, step=False):
    """(SelscanArgs, device): step = one token per sequence, the state required."""
    lead, S, T, off, dev = _seqs(x, seq_offsets, where)
    kind, f32, D = x.dtype, torch.float32, x.shape[-1]
    if a.dim() != 2 or b.dim() != len(lead) + 2:
        _need(False, where, "a is [D, N], b and c are [..., G, N]")
    if step:
        _need(len(lead) == 1, where, "x must be [S, D]")
        S = T
    G, N = gn = b.shape[-2:]
    if G * N > _MAX_INT:
        _need(False, where, "b and c have %d x %d values a token" % (G, N))
    row, shape, g_shape = (D,), x.shape, lead + gn
    px, xs = _rows(x, where, "x", lead, kind, dev, row, shape)
    pdt, dts = _rows(dt, where, "dt", lead, kind, dev, row, shape)
    pb, bs = _rows(b, where, "b", lead, kind, dev, gn, g_shape)
    pc, cs = _rows(c, where, "c", lead, kind, dev, gn, g_shape)
    pz, zs = (None, 0) if z is None else _rows(z, where, "z", lead, kind, dev, row, shape)
    return SelscanArgs(px, pdt, pb, pc, pz, xs, dts, bs, cs, zs, _flat(a, where, "a", (D, N), f32, dev),
                       _flat(d_skip, where, "d_skip", row, f32, dev), _flat(dt_bias, where, "dt_bias", row, f32, dev),
                       _flat(state_in, where, "state", (S, D, N), f32, dev), off, S, T, D, N, G, int(bool(softplus)), _DTYPES[kind]), dev


def selscan_checkpoints(T, S, D, N, device):
    """A buffer for the states that selscan_fwd saves for selscan_bwd."""
    return torch.empty(int(lib().chela_selscan_checkpoint_bytes(T, S, D, N)) // 4, dtype=torch.float32, device=device)


def _checkpoints(t, where, r, dev):
    if t is None:
        return None
    need = int(lib().chela_selscan_checkpoint_bytes(r.T, r.S, r.D, r.N)) // 4
    _need(t.dim() == 1 and t.shape[0] >= need, where, "checkpoints must come from selscan_checkpoints for these sizes")
    return _flat(t, where, "checkpoints", t.shape, torch.float32, dev)


def selscan_fwd(x, dt, a, b, c, d_skip=None, z=None, dt_bias=None, softplus=True, state_in=None, state_out=None,
                seq_offsets=None, checkpoints=None, out_dtype=None, out=None, workspace=None):
    """chela_selscan_fwd: (y, state_out).  x, dt, z [T,D] or [B,L,D]; a [D,N] f32; b, c [...,G,N]; states [S,D,N] f32."""
    where = "chela_selscan_fwd"
    r, dev = _selscan_args(where, x, dt, a, b, c, d_skip, z, dt_bias, softplus, state_in, seq_offsets)
    y = _new_like(out, where, "out", x, x.dtype if out_dtype is None else _tdtype(out_dtype), dev)
    state_out = _new(state_out, where, "state_out", (r.S, r.D, r.N), torch.float32, x.device, dev)
    if out is None:
        r.softplus |= ZERO_REST
    ckpt = _checkpoints(checkpoints, where, r, dev)
    workspace, ws, nbytes = _scratch(lib().chela_selscan_workspace_bytes(r.T, r.S, r.D, r.N), workspace, x.device, where, dev)
    _run(lib().chela_selscan_fwd, where, dev, ctypes.byref(r), y.data_ptr(), state_out.data_ptr(), ckpt, _DTYPES[y.dtype], ws, nbytes)
    return y, state_out


def selscan_step(x, dt, a, b, c, state, d_skip=None, z=None, dt_bias=None, softplus=True, state_out=None, out_dtype=None,
                 out=None):
    """chela_selscan_step: y [S,D] for one new token per sequence; state [S,D,N] f32 is updated in place unless state_out
    is given."""
    where = "chela_selscan_step"
    r, dev = _selscan_args(where, x, dt, a, b, c, d_skip, z, dt_bias, softplus, state, None, True)
    y = _new_like(out, where, "out", x, x.dtype if out_dtype is None else _tdtype(out_dtype), dev)
    after = _at(state) if state_out is None else _flat(state_out, where, "state_out", (r.S, r.D, r.N), torch.float32, dev)
    _run(lib().chela_selscan_step, where, dev, ctypes.byref(r), y.data_ptr(), after, _DTYPES[y.dtype])
    return y


def selscan_bwd(x, dt, a, b, c, d_y, d_skip=None, z=None, dt_bias=None, softplus=True, state_in=None, seq_offsets=None,
                checkpoints=None, d_state_out=None, grad_dtype=F32, want_d_state=False, workspace=None):
    """chela_selscan_bwd: SelscanGrads; d_x, d_dt, d_b, d_c, d_z of grad_dtype, the others f32 (None where not given)."""
    where = "chela_selscan_bwd"
    r, dev = _selscan_args(where, x, dt, a, b, c, d_skip, z, dt_bias, softplus, state_in, seq_offsets)
    device, gt, f32, held = x.device, _tdtype(grad_dtype), torch.float32, (r.S, r.D, r.N)
    pdy, dys = _rows(d_y, where, "d_y", x.shape[:-1], x.dtype, dev, (r.D,))
    ckpt = _checkpoints(checkpoints, where, r, dev)
    g = SelscanGrads(d_x=_like(x, gt), d_dt=_like(dt, gt), d_a=_like(a, f32), d_b=_like(b, gt), d_c=_like(c, gt), d_skip=_like(d_skip, f32),
                     d_z=_like(z, gt), d_dt_bias=_like(dt_bias, f32),
                     d_state_in=torch.empty(held, dtype=f32, device=device) if want_d_state else None)
    workspace, ws, nbytes = _scratch(lib().chela_selscan_bwd_workspace_bytes(r.T, r.S, r.D, r.N, int(ckpt is not None)), workspace, device, where, dev)
    _run(lib().chela_selscan_bwd, where, dev, ctypes.byref(r), pdy, dys, _flat(d_state_out, where, "d_state_out", held, f32, dev), ckpt,
         *map(_at, g), int(grad_dtype), ws, nbytes)
    return g


def _blocknorm_args(where, res, y, gate, w_post, b_post, norm_post, scale, w_pre, b_pre, norm_pre, gate_act, gate_after, eps):
    """(BlocknormArgs, the tensor that gives shape and residual dtype, device)"""
    first = res if res is not None else y
    _need(first is not None, where, "res or y must be given")
    lead, _, T, _, dev = _seqs(first, None, where)
    shape, f32 = first.shape, torch.float32
    D = shape[-1]
    row = (D,)
    pr, rs = (None, 0) if res is None else _rows(res, where, "res", lead, res.dtype, dev, row, shape)
    py = pg = None
    ys = gs = 0
    kind = first.dtype
    if y is not None:
        kind = y.dtype
        _need(kind in _DTYPES, where, "y must be float32 or bfloat16")
        py, ys = _rows(y, where, "y", lead, kind, dev, row, shape)
    if gate is not None:
        _need(y is not None, where, "gate goes with y")
        pg, gs = _rows(gate, where, "gate", lead, kind, dev, row, shape)
    return BlocknormArgs(pr, py, pg, rs, ys, gs, _flat(w_post, where, "w_post", row, f32, dev), _flat(b_post, where, "b_post", row, f32, dev),
                         _flat(scale, where, "scale", row, f32, dev), _flat(w_pre, where, "w_pre", row, f32, dev),
                         _flat(b_pre, where, "b_pre", row, f32, dev), T, D, int(gate_act), int(bool(gate_after)), int(norm_post),
                         int(norm_pre), float(eps), _DTYPES[kind], _DTYPES[first.dtype]), first, dev


def blocknorm_fwd(res, y=None, gate=None, w_post=None, b_post=None, norm_post=NORM_RMS, scale=None, w_pre=None, b_pre=None,
                  norm_pre=NORM_RMS, gate_act=1, gate_after=False, eps=1e-6, pre=True, out_dtype=None, res_out=None, out=None):
    """chela_blocknorm_fwd: (r', o).  y=None: only the norm before a block (r' is res itself); pre=False: only gate, norm,
    scale and residual behind one (o is None).  o is of out_dtype, or y's (without y: res's) dtype."""
    where = "chela_blocknorm_fwd"
    r, first, dev = _blocknorm_args(where, res, y, gate, w_post, b_post, norm_post, scale, w_pre, b_pre, norm_pre, gate_act, gate_after, eps)
    _need(pre or y is not None, where, "nothing to compute")
    if y is not None:
        res_out = _new_like(res_out, where, "res_out", first, first.dtype, dev)
    else:
        _need(res_out is None, where, "res_out goes with y")
    o, code = None, F32
    if pre:
        dt = (y if y is not None else res).dtype if out_dtype is None else _tdtype(out_dtype)
        o, code = _new_like(out, where, "out", first, dt, dev), _DTYPES[dt]
    _run(lib().chela_blocknorm_fwd, where, dev, ctypes.byref(r), None if res_out is None else res_out.data_ptr(),
         None if o is None else o.data_ptr(), code)
    return res_out if y is not None else res, o


def blocknorm_bwd(res_out, y=None, gate=None, d_o=None, d_res_out=None, w_post=None, b_post=None, norm_post=NORM_RMS, scale=None,
                  w_pre=None, b_pre=None, norm_pre=NORM_RMS, gate_act=1, gate_after=False, eps=1e-6, grad_dtype=F32, workspace=None):
    """chela_blocknorm_bwd: BlocknormGrads from r' (as blocknorm_fwd returned it), y and gate; d_o of y's dtype (without y:
    res_out's), d_res_out of res_out's dtype, either may be None.  d_res is of res_out's dtype, d_y and d_gate of grad_dtype."""
    where = "chela_blocknorm_bwd"
    r, first, dev = _blocknorm_args(where, res_out, y, gate, w_post, b_post, norm_post, scale, w_pre, b_pre, norm_pre, gate_act, gate_after, eps)
    device, shape, gt, D = first.device, first.shape, _tdtype(grad_dtype), r.D
    kind = first.dtype if y is None else y.dtype
    g = BlocknormGrads(_like(first, first.dtype), _like(y, gt), _like(gate, gt), *(_like(w, torch.float32) for w in (w_post, b_post, scale, w_pre, b_pre)))
    workspace, ws, nbytes = _scratch(lib().chela_blocknorm_bwd_workspace_bytes(r.T, D), workspace, device, where, dev)
    _run(lib().chela_blocknorm_bwd, where, dev, ctypes.byref(r), _flat(d_o, where, "d_o", shape, kind, dev),
         _flat(d_res_out, where, "d_res_out", shape, first.dtype, dev), *map(_at, g), int(grad_dtype), ws, nbytes)
    return g
