"""Blurry Window Attention forward operator (and its backward pass) on MI355X (gfx950), and the sequence operators beside it:
window attention with sinks, also with a learned bias, behind a shared prefix and over a cache of bounded size, the short causal convolution, the selective
state space scan.

A thin ctypes binding over ``libbla.so`` (the C ABI in ``include/bla.h``).  It
only marshals arguments: every step of the operator runs in the library's HIP
kernels.  torch is used for device buffers and the current stream.  If the
library has not been built, importing works but every call raises.
"""
from __future__ import annotations

import ctypes
import functools
import operator
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbla.so")

BLA_F32, BLA_BF16 = 0, 1
STATUS = {0: "BLA_OK", 1: "BLA_ERR_INVALID_ARG", 2: "BLA_ERR_UNSUPPORTED", 3: "BLA_ERR_WORKSPACE",
          4: "BLA_ERR_HIP"}


class BlaError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what} failed: {STATUS.get(status, status)}")
        self.status = status


class Params(ctypes.Structure):
    """Mirror of ``bla_params``."""
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("L", ctypes.c_int32),
                ("d_k", ctypes.c_int32), ("d_v", ctypes.c_int32), ("M", ctypes.c_int32),
                ("S", ctypes.c_int32), ("chunk", ctypes.c_int32), ("t0", ctypes.c_int64),
                ("scale", ctypes.c_float), ("io_dtype", ctypes.c_int32),
                ("phase_anchor", ctypes.c_int32), ("reuse_tables", ctypes.c_int32)]


class WindowParams(ctypes.Structure):
    """Mirror of ``bla_window_params``."""
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("H_kv", ctypes.c_int32), ("L", ctypes.c_int32),
                ("d", ctypes.c_int32), ("window", ctypes.c_int32), ("sinks", ctypes.c_int32),
                ("io_dtype", ctypes.c_int32), ("t0", ctypes.c_int64), ("scale", ctypes.c_float)]


class PrefixParams(ctypes.Structure):
    """Mirror of ``bla_prefix_params``."""
    _fields_ = [("w", WindowParams), ("P", ctypes.c_int32), ("G", ctypes.c_int32)]


class EvictParams(ctypes.Structure):
    """Mirror of ``bla_evict_params``."""
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("H_kv", ctypes.c_int32), ("L", ctypes.c_int32),
                ("d", ctypes.c_int32), ("slots", ctypes.c_int32), ("recent", ctypes.c_int32),
                ("io_dtype", ctypes.c_int32), ("t0", ctypes.c_int64), ("scale", ctypes.c_float)]


class ConvParams(ctypes.Structure):
    """Mirror of ``bla_conv_params``."""
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("L", ctypes.c_int32), ("d", ctypes.c_int32),
                ("taps", ctypes.c_int32), ("silu", ctypes.c_int32), ("io_dtype", ctypes.c_int32)]


class SsmParams(ctypes.Structure):
    """Mirror of ``bla_ssm_params``."""
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("G", ctypes.c_int32), ("L", ctypes.c_int32),
                ("d", ctypes.c_int32), ("N", ctypes.c_int32), ("io_dtype", ctypes.c_int32)]


_lib = None
_dp = ctypes.POINTER(ctypes.c_double)
_vp = ctypes.c_void_p


def lib():
    """The loaded library; raises if it is missing (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2606_09862_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        P = ctypes.POINTER(Params)
        L.bla_status_string.argtypes = [ctypes.c_int]
        L.bla_status_string.restype = ctypes.c_char_p
        L.bla_supported.argtypes = [P]
        L.bla_supported.restype = ctypes.c_int
        L.bla_workspace_size.argtypes = [P]
        L.bla_workspace_size.restype = ctypes.c_size_t
        L.bla_step_workspace_size.argtypes = [P]
        L.bla_step_workspace_size.restype = ctypes.c_size_t
        L.bla_forward.argtypes = [P, _dp] + [_vp] * 9 + [ctypes.c_size_t, _vp]
        L.bla_forward.restype = ctypes.c_int
        L.bla_step.argtypes = [P, _dp] + [_vp] * 8 + [ctypes.c_size_t, _vp]
        L.bla_forward_noalloc.argtypes = [P, _dp] + [_vp] * 8 + [_vp]
        L.bla_forward_noalloc.restype = ctypes.c_int
        L.bla_interp_tables.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_double, _dp, _dp,
                                        ctypes.POINTER(ctypes.c_int32)]
        L.bla_interp_tables.restype = ctypes.c_int
        L.bla_step.restype = ctypes.c_int
        L.bla_decay_workspace_size.argtypes = [P]
        L.bla_decay_workspace_size.restype = ctypes.c_size_t
        L.bla_decay_forward.argtypes = [P, _dp] + [_vp] * 9 + [ctypes.c_size_t, _vp]
        L.bla_decay_forward.restype = ctypes.c_int
        L.bla_decay_step.argtypes = [P, _dp] + [_vp] * 8 + [ctypes.c_size_t, _vp]
        L.bla_decay_step.restype = ctypes.c_int
        L.bla_backward_workspace_size.argtypes = [P]
        L.bla_backward_workspace_size.restype = ctypes.c_size_t
        L.bla_backward.argtypes = [P, _dp] + [_vp] * 14 + [ctypes.c_size_t, _vp]
        L.bla_backward.restype = ctypes.c_int
        L.bla_backward_timed.argtypes = [P, _dp] + [_vp] * 14 + [ctypes.c_size_t, _vp,
                                                                  ctypes.POINTER(ctypes.c_void_p)]
        L.bla_backward_timed.restype = ctypes.c_int
        L.bla_layer_workspace_size.argtypes = [P]
        L.bla_layer_workspace_size.restype = ctypes.c_size_t
        L.bla_layer_forward.argtypes = [P, _dp] + [_vp] * 9 + [ctypes.c_size_t, _vp]
        L.bla_layer_forward.restype = ctypes.c_int
        L.bla_layer_forward_timed.argtypes = [P, _dp] + [_vp] * 9 + [ctypes.c_size_t, _vp,
                                                                       ctypes.POINTER(ctypes.c_void_p)]
        L.bla_layer_forward_timed.restype = ctypes.c_int
        W = ctypes.POINTER(WindowParams)
        for name in ("bla_window_workspace_size", "bla_window_step_workspace_size", "bla_window_backward_workspace_size"):
            getattr(L, name).argtypes = [W]
            getattr(L, name).restype = ctypes.c_size_t
        L.bla_window_supported.argtypes = [W]
        L.bla_window_forward.argtypes = [W] + [_vp] * 12 + [ctypes.c_size_t, _vp]
        L.bla_window_step.argtypes = [W] + [_vp] * 8 + [ctypes.c_size_t, _vp]
        L.bla_window_backward.argtypes = [W] + [_vp] * 11 + [ctypes.c_size_t, _vp]
        for name in ("bla_window_supported", "bla_window_forward", "bla_window_step", "bla_window_backward"):
            getattr(L, name).restype = ctypes.c_int
        i32, ip = ctypes.c_int32, ctypes.POINTER(ctypes.c_int32)
        L.bla_bias_forward.argtypes = [W, i32, ip] + [_vp] * 13 + [ctypes.c_size_t, _vp]
        L.bla_bias_step.argtypes = [W, i32, ip] + [_vp] * 9 + [ctypes.c_size_t, _vp]
        L.bla_bias_backward.argtypes = [W, i32, ip] + [_vp] * 13 + [ctypes.c_size_t, _vp]
        L.bla_bias_step_workspace_size.argtypes = [W]
        L.bla_bias_step_workspace_size.restype = ctypes.c_size_t
        L.bla_bias_backward_workspace_size.argtypes = [W, i32]
        L.bla_bias_backward_workspace_size.restype = ctypes.c_size_t
        for name in ("bla_bias_forward", "bla_bias_step", "bla_bias_backward"):
            getattr(L, name).restype = ctypes.c_int
        X = ctypes.POINTER(PrefixParams)
        for name in ("bla_prefix_workspace_size", "bla_prefix_step_workspace_size"):
            getattr(L, name).argtypes = [X]
            getattr(L, name).restype = ctypes.c_size_t
        L.bla_prefix_supported.argtypes = [X]
        L.bla_prefix_forward.argtypes = [X] + [_vp] * 15 + [ctypes.c_size_t, _vp]
        L.bla_prefix_step.argtypes = [X] + [_vp] * 11 + [ctypes.c_size_t, _vp]
        for name in ("bla_prefix_supported", "bla_prefix_forward", "bla_prefix_step"):
            getattr(L, name).restype = ctypes.c_int
        E = ctypes.POINTER(EvictParams)
        for name in ("bla_evict_workspace_size", "bla_evict_step_workspace_size"):
            getattr(L, name).argtypes = [E]
            getattr(L, name).restype = ctypes.c_size_t
        L.bla_evict_supported.argtypes = [E]
        L.bla_evict_forward.argtypes = [E] + [_vp] * 12 + [ctypes.c_size_t, _vp]
        L.bla_evict_select.argtypes = [E] + [_vp] * 13
        L.bla_evict_step.argtypes = [E] + [_vp] * 12 + [ctypes.c_size_t, _vp]
        for name in ("bla_evict_supported", "bla_evict_forward", "bla_evict_select", "bla_evict_step"):
            getattr(L, name).restype = ctypes.c_int
        C = ctypes.POINTER(ConvParams)
        L.bla_conv_backward_workspace_size.argtypes = [C]
        L.bla_conv_backward_workspace_size.restype = ctypes.c_size_t
        L.bla_conv_supported.argtypes = [C]
        L.bla_conv_forward.argtypes = [C] + [_vp] * 8
        L.bla_conv_step.argtypes = [C] + [_vp] * 7
        L.bla_conv_backward.argtypes = [C] + [_vp] * 12 + [ctypes.c_size_t, _vp]
        for name in ("bla_conv_supported", "bla_conv_forward", "bla_conv_step", "bla_conv_backward"):
            getattr(L, name).restype = ctypes.c_int
        S = ctypes.POINTER(SsmParams)
        for name in ("bla_ssm_workspace_size", "bla_ssm_backward_workspace_size"):
            getattr(L, name).argtypes = [S]
            getattr(L, name).restype = ctypes.c_size_t
        L.bla_ssm_supported.argtypes = [S]
        L.bla_ssm_forward.argtypes = [S] + [_vp] * 11 + [ctypes.c_size_t, _vp]
        L.bla_ssm_step.argtypes = [S] + [_vp] * 10
        L.bla_ssm_backward.argtypes = [S] + [_vp] * 18 + [ctypes.c_size_t, _vp]
        for name in ("bla_ssm_supported", "bla_ssm_forward", "bla_ssm_step", "bla_ssm_backward"):
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def make_params(B, H, L, d, M, S, dtype, t0=0, scale=0.0, chunk=0, phase_anchor=False,
                reuse_tables=False) -> Params:
    io = BLA_BF16 if dtype == torch.bfloat16 else BLA_F32
    return Params(B, H, L, d, d, M, S, chunk, int(t0), float(scale), io, int(phase_anchor),
                  int(reuse_tables))


@functools.lru_cache(maxsize=64)
def _period_array(H):
    return ctypes.c_double * max(H, 1)


def _periods(T, H):
    vals = T if hasattr(T, "__len__") else [T] * H
    if len(vals) != H:
        raise ValueError("T must have one period per head")
    try:
        return _period_array(H)(*vals)
    except TypeError:  # values that only float() converts
        return _period_array(H)(*map(float, vals))


# A decode step of a small model runs for 7 us on the device, so its call must not take longer on
# the host.  Pointers and the stream therefore go to the library as plain integers (the declared
# argument types convert them), and the stream is asked for by device index: a call of one
# layer takes 10 us instead of 12.7.
def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(device):
    return torch._C._cuda_getCurrentRawStream(device.index)


def interp_tables(M: int, S: int, T: float):
    """Float64 slot tables of one head from the library: A, B [S, M] and thresholds [S]."""
    import numpy as np
    A = np.zeros((S, M), np.float64)
    B = np.zeros((S, M), np.float64)
    th = np.zeros((S,), np.int32)
    st = lib().bla_interp_tables(M, S, float(T), A.ctypes.data_as(_dp), B.ctypes.data_as(_dp),
                                 th.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)))
    if st != 0:
        raise BlaError(st, "bla_interp_tables")
    return A, B, th


def supported(p: Params) -> int:
    return lib().bla_supported(ctypes.byref(p))


def workspace_size(p: Params) -> int:
    return lib().bla_workspace_size(ctypes.byref(p))


def step_workspace_size(p: Params) -> int:
    return lib().bla_step_workspace_size(ctypes.byref(p))


def _check(t, shape, dtype, name):
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name}: expected contiguous {dtype} cuda tensor of shape {tuple(shape)}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")


def _out(out, like, shape):
    """A fresh output like `like`, or the caller's `out` after the same checks as the inputs
    (shape, dtype, contiguity, device), so that a wrong buffer fails before any launch."""
    if out is None:
        return torch.empty_like(like)
    _check(out, shape, like.dtype, "out")
    if out.device != like.device:
        raise ValueError(f"out: expected a tensor on {like.device}, got {out.device}")
    return out


def forward(q, k, v, T, M: int, S: int, t0: int = 0, scale: float | None = None,
            state_k=None, state_v=None, want_state: bool = True, workspace=None, out=None,
            phase_anchor: bool = False, reuse_tables: bool = False, chunk: int = 0):
    """bla_forward on q, k, v [B,H,L,d] (float32 or bfloat16 cuda tensors).

    Returns (o, state_k_out, state_v_out); the states are float32 [B,H,2,M,d]
    (None when want_state is False).  phase_anchor selects the anchored slots of
    Sec. 3.3 (Alg. 1 / Alg. 3); the state is the same mode state in both forms.
    reuse_tables: keep the tables an earlier call built in the same `workspace`
    (bla_params.reuse_tables; only meaningful with a caller-kept workspace).  chunk: tokens
    per chunk of the parallel form (16, 32, 64 or 128; 0 = 64).
    """
    B, H, L, d = q.shape
    dt = q.dtype
    for name, t in (("k", k), ("v", v)):
        _check(t, (B, H, L, d), dt, name)
    _check(q, (B, H, L, d), dt, "q")
    p = make_params(B, H, L, d, M, S, dt, t0, 0.0 if scale is None else scale, chunk=chunk,
                    phase_anchor=phase_anchor, reuse_tables=reuse_tables)
    for name, t in (("state_k", state_k), ("state_v", state_v)):
        if t is not None:
            _check(t, (B, H, 2, M, d), torch.float32, name)
    dev = q.device
    o = _out(out, q, (B, H, L, d))
    sk = torch.empty((B, H, 2, M, d), dtype=torch.float32, device=dev) if want_state else None
    sv = torch.empty((B, H, 2, M, d), dtype=torch.float32, device=dev) if want_state else None
    need = workspace_size(p)
    if need == 0 and supported(p) != 0:
        raise BlaError(supported(p), "bla_forward (shape check)")
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    st = lib().bla_forward(ctypes.byref(p), _periods(T, H), _ptr(q), _ptr(k), _ptr(v), _ptr(state_k),
                           _ptr(state_v), _ptr(o), _ptr(sk), _ptr(sv), _ptr(workspace),
                           workspace.numel(), _stream(dev))
    if st != 0:
        raise BlaError(st, "bla_forward")
    return o, sk, sv


def forward_noalloc(q, k, v, T, M: int, S: int, t0: int = 0, scale: float | None = None,
                    state_k=None, state_v=None, out=None, state_k_out=None, state_v_out=None,
                    phase_anchor: bool = False, reuse_tables: bool = False):
    """bla_forward_noalloc: bla_forward with the library's own fixed device workspace.  The
    library allocates nothing; the caller passes every output (`out`, and `state_k_out` /
    `state_v_out` float32 [B,H,2,M,d], None = not wanted).  Returns (o, state_k_out, state_v_out)."""
    B, H, L, d = q.shape
    dt = q.dtype
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check(t, (B, H, L, d), dt, name)
    if out is None:
        raise ValueError("out: bla_forward_noalloc needs the caller's output buffer")
    o = _out(out, q, (B, H, L, d))
    for name, t in (("state_k", state_k), ("state_v", state_v), ("state_k_out", state_k_out),
                    ("state_v_out", state_v_out)):
        if t is not None:
            _check(t, (B, H, 2, M, d), torch.float32, name)
    p = make_params(B, H, L, d, M, S, dt, t0, 0.0 if scale is None else scale,
                    phase_anchor=phase_anchor, reuse_tables=reuse_tables)
    st = lib().bla_forward_noalloc(ctypes.byref(p), _periods(T, H), _ptr(q), _ptr(k), _ptr(v), _ptr(state_k),
                                   _ptr(state_v), _ptr(o), _ptr(state_k_out), _ptr(state_v_out),
                                   _stream(q.device))
    if st != 0:
        raise BlaError(st, "bla_forward_noalloc")
    return o, state_k_out, state_v_out


def step(q, k, v, T, M: int, S: int, state_k, state_v, pos=None, t0: int = 0,
         scale: float | None = None, workspace=None, out=None, phase_anchor: bool = False,
         reuse_tables: bool = False):
    """bla_step: one decode token per row; q,k,v [B,H,d]; updates state_k/state_v in place."""
    B, H, d = q.shape
    dt = q.dtype
    _check(q, (B, H, d), dt, "q")
    _check(k, (B, H, d), dt, "k")
    _check(v, (B, H, d), dt, "v")
    _check(state_k, (B, H, 2, M, d), torch.float32, "state_k")
    _check(state_v, (B, H, 2, M, d), torch.float32, "state_v")
    if pos is not None:
        _check(pos, (B,), torch.int64, "pos")
    p = make_params(B, H, 1, d, M, S, dt, t0, 0.0 if scale is None else scale,
                    phase_anchor=phase_anchor, reuse_tables=reuse_tables)
    dev = q.device
    o = _out(out, q, (B, H, d))
    need = step_workspace_size(p)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    st = lib().bla_step(ctypes.byref(p), _periods(T, H), _ptr(q), _ptr(k), _ptr(v), _ptr(pos),
                        _ptr(state_k), _ptr(state_v), _ptr(o), _ptr(workspace), workspace.numel(),
                        _stream(dev))
    if st != 0:
        raise BlaError(st, "bla_step")
    return o


def decay_workspace_size(p: Params) -> int:
    return lib().bla_decay_workspace_size(ctypes.byref(p))


def decay_forward(q, k, v, T, M: int, S: int, t0: int = 0, scale: float | None = None,
                  slot_k=None, slot_v=None, want_state: bool = True, workspace=None, out=None):
    """bla_decay_forward (state-decay form, Sec. 3.4) on q, k, v [B,H,L,d].

    Returns (o, slot_k_out, slot_v_out); slot states are float32 [B,H,S,d].
    """
    B, H, L, d = q.shape
    dt = q.dtype
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check(t, (B, H, L, d), dt, name)
    for name, t in (("slot_k", slot_k), ("slot_v", slot_v)):
        if t is not None:
            _check(t, (B, H, S, d), torch.float32, name)
    p = make_params(B, H, L, d, M, S, dt, t0, 0.0 if scale is None else scale)
    dev = q.device
    o = _out(out, q, (B, H, L, d))
    sk = torch.empty((B, H, S, d), dtype=torch.float32, device=dev) if want_state else None
    sv = torch.empty((B, H, S, d), dtype=torch.float32, device=dev) if want_state else None
    need = decay_workspace_size(p)
    if need == 0 and supported(p) != 0:
        raise BlaError(supported(p), "bla_decay_forward (shape check)")
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    st = lib().bla_decay_forward(ctypes.byref(p), _periods(T, H), _ptr(q), _ptr(k), _ptr(v), _ptr(slot_k),
                                 _ptr(slot_v), _ptr(o), _ptr(sk), _ptr(sv), _ptr(workspace),
                                 workspace.numel(), _stream(dev))
    if st != 0:
        raise BlaError(st, "bla_decay_forward")
    return o, sk, sv


def decay_step(q, k, v, T, M: int, S: int, slot_k, slot_v, pos=None, t0: int = 0,
               scale: float | None = None, workspace=None, out=None):
    """bla_decay_step: one decode token per row; q,k,v [B,H,d]; updates slot_k/slot_v in place."""
    B, H, d = q.shape
    dt = q.dtype
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check(t, (B, H, d), dt, name)
    _check(slot_k, (B, H, S, d), torch.float32, "slot_k")
    _check(slot_v, (B, H, S, d), torch.float32, "slot_v")
    if pos is not None:
        _check(pos, (B,), torch.int64, "pos")
    p = make_params(B, H, 1, d, M, S, dt, t0, 0.0 if scale is None else scale)
    dev = q.device
    o = _out(out, q, (B, H, d))
    need = decay_workspace_size(p)
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    st = lib().bla_decay_step(ctypes.byref(p), _periods(T, H), _ptr(q), _ptr(k), _ptr(v), _ptr(pos),
                              _ptr(slot_k), _ptr(slot_v), _ptr(o), _ptr(workspace), workspace.numel(),
                              _stream(dev))
    if st != 0:
        raise BlaError(st, "bla_decay_step")
    return o


def backward_workspace_size(p: Params) -> int:
    return lib().bla_backward_workspace_size(ctypes.byref(p))


def backward(q, k, v, dO, T, M: int, S: int, t0: int = 0, scale: float | None = None,
             state_k=None, state_v=None, dstate_k=None, dstate_v=None, want_state_grad: bool = True,
             workspace=None):
    """bla_backward: gradients of ``forward`` (rotating slots) for dO = dLoss/dO [B,H,L,d] and
    dstate_k / dstate_v = dLoss/d(final states) [B,H,2,M,d] (None = zero).  state_k / state_v
    are the forward's input states.  Returns (dq, dk, dv, dLoss/d(state_k in),
    dLoss/d(state_v in)); the last two are None when want_state_grad is False.
    """
    B, H, L, d = q.shape
    dt = q.dtype
    for name, t in (("q", q), ("k", k), ("v", v), ("dO", dO)):
        _check(t, (B, H, L, d), dt, name)
    for name, t in (("state_k", state_k), ("state_v", state_v), ("dstate_k", dstate_k),
                    ("dstate_v", dstate_v)):
        if t is not None:
            _check(t, (B, H, 2, M, d), torch.float32, name)
    p = make_params(B, H, L, d, M, S, dt, t0, 0.0 if scale is None else scale)
    dev = q.device
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    gsk = torch.empty((B, H, 2, M, d), dtype=torch.float32, device=dev) if want_state_grad else None
    gsv = torch.empty((B, H, 2, M, d), dtype=torch.float32, device=dev) if want_state_grad else None
    need = backward_workspace_size(p)
    if need == 0:
        raise BlaError(2, "bla_backward (shape check)")
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    st = lib().bla_backward(ctypes.byref(p), _periods(T, H), _ptr(q), _ptr(k), _ptr(v), _ptr(dO),
                            _ptr(state_k), _ptr(state_v), _ptr(dstate_k), _ptr(dstate_v), _ptr(dq),
                            _ptr(dk), _ptr(dv), _ptr(gsk), _ptr(gsv), _ptr(workspace), workspace.numel(),
                            _stream(dev))
    if st != 0:
        raise BlaError(st, "bla_backward")
    return dq, dk, dv, gsk, gsv


def layer_workspace_size(p: Params) -> int:
    return lib().bla_layer_workspace_size(ctypes.byref(p))


def layer_forward(x, w_qkv, w_o, T, H: int, M: int, S: int, t0: int = 0, scale: float | None = None,
                  state_k=None, state_v=None, want_state: bool = True, workspace=None, out=None,
                  phase_anchor: bool = False):
    """bla_layer_forward: y = BLA(x W_qkv) W_o on hidden states x [B, L, D] (bf16, D = H d);
    w_qkv [D, 3D] and w_o [D, D] bf16.  Returns (y [B, L, D], state_k_out, state_v_out)."""
    B, L, D = x.shape
    d = D // H
    dt = x.dtype
    if dt != torch.bfloat16 or d * H != D:
        raise ValueError("layer_forward: bf16 hidden states with D = H * d")
    _check(x, (B, L, D), dt, "x")
    _check(w_qkv, (D, 3 * D), dt, "w_qkv")
    _check(w_o, (D, D), dt, "w_o")
    for name, t in (("state_k", state_k), ("state_v", state_v)):
        if t is not None:
            _check(t, (B, H, 2, M, d), torch.float32, name)
    p = make_params(B, H, L, d, M, S, dt, t0, 0.0 if scale is None else scale, phase_anchor=phase_anchor)
    dev = x.device
    y = _out(out, x, (B, L, D))
    sk = torch.empty((B, H, 2, M, d), dtype=torch.float32, device=dev) if want_state else None
    sv = torch.empty((B, H, 2, M, d), dtype=torch.float32, device=dev) if want_state else None
    need = layer_workspace_size(p)
    if need == 0:
        raise BlaError(supported(p) or 2, "bla_layer_forward (shape check)")
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    st = lib().bla_layer_forward(ctypes.byref(p), _periods(T, H), _ptr(x), _ptr(w_qkv), _ptr(w_o), _ptr(state_k),
                                 _ptr(state_v), _ptr(y), _ptr(sk), _ptr(sv), _ptr(workspace), workspace.numel(),
                                 _stream(dev))
    if st != 0:
        raise BlaError(st, "bla_layer_forward")
    return y, sk, sv


# ---- window attention, the short convolution and the selective scan ----
#
# A decode step of these runs for a few microseconds on the device as well, so what depends on shapes alone (the
# parameter block, whether the shape is supported, the workspace's size) is kept per shape.  A position is no part of a shape: it goes into
# a copy of the block.

def _check_on(t, shape, dtype, name, dev):
    """A contiguous tensor of this shape and type on GPU number dev."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev or dev < 0 or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous {dtype} tensor of shape {tuple(shape)} on cuda:{max(dev, 0)}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")


def _io(dtype, name):
    if dtype is torch.bfloat16:
        return BLA_BF16
    if dtype is torch.float32:
        return BLA_F32
    raise ValueError(f"{name}: expected torch.float32 or torch.bfloat16, got {dtype}")


def _call(fn, what, dev, *args):
    """The library's call on the tensors' device (which need not be the current one) and its current stream."""
    stream = torch._C._cuda_getCurrentRawStream(dev)
    if dev != torch._C._cuda_getDevice():
        with torch.cuda.device(dev):
            st = fn(*args, stream)
    else:
        st = fn(*args, stream)
    if st != 0:
        raise BlaError(st, what)


def _result(out, like, shape, name="out"):
    """A fresh tensor like `like`, or the caller's after the checks of an input."""
    if out is None:
        return torch.empty_like(like)
    _check_on(out, shape, like.dtype, name, like.get_device())
    return out


def _room(workspace, need, like):
    """The caller's workspace where it is large enough (a uint8 tensor on the call's device), a fresh one otherwise, or
    None where none is needed: (tensor, address, bytes)."""
    if need == 0:
        return None, None, 0
    if workspace is not None and workspace.numel() >= need:
        _check_on(workspace, workspace.shape, torch.uint8, "workspace", like.get_device())
    else:
        workspace = torch.empty(need, dtype=torch.uint8, device=like.device)
    return workspace, workspace.data_ptr(), workspace.numel()


def _shape_status(st, what):
    if st != 0:
        raise BlaError(st, f"{what} (shape check)")


def _int32(what, *values):
    """Refuses sizes past the parameter block's fields, which would take their lower bits."""
    if not all(-(1 << 31) <= v < 1 << 31 for v in values):
        raise BlaError(2, f"{what} (shape check)")


@functools.lru_cache(maxsize=256)
def _window_plan(what, B, H, Hkv, L, d, window, sinks, scale, dtype):
    """(parameters at t0 = 0, the same by reference, workspace bytes) of the library's call `what`."""
    _int32(what, B, H, Hkv, L, d, window, sinks)
    block = WindowParams(B, H, Hkv, L, d, window, sinks, _io(dtype, "q"), 0, scale)
    p = ctypes.byref(block)
    st = lib().bla_window_supported(p)
    if what == "bla_window_forward" or st != 2:  # the launches of the other calls have limits of their own, which they check
        _shape_status(st, what)
    return block, p, getattr(lib(), what.replace("_forward", "") + "_workspace_size")(p)


def _window_params(what, B, H, Hkv, L, d, window, sinks, t0, scale, dtype):
    """(parameters by reference, workspace bytes)."""
    block, p, need = _window_plan(what, B, H, Hkv, L, d, int(window), int(sinks), 0.0 if scale is None else float(scale), dtype)
    if t0 != 0:
        if not -(1 << 63) <= t0 < 1 << 63:
            raise BlaError(1, what)
        block = WindowParams.from_buffer_copy(block)
        block.t0 = int(t0)
        p = ctypes.byref(block)
    return p, need


def window_forward(q, k, v, window: int, sinks: int = 0, t0: int = 0, scale: float | None = None, lengths=None, pos=None,
                   cache_k=None, cache_v=None, want_lse: bool = False, want_cache: bool = False, workspace=None,
                   out=None):
    """bla_window_forward: softmax attention over the last `window` tokens and the first `sinks` tokens.

    q [B,H,L,d], k and v [B,H_kv,L,d] (float32 or bfloat16), H a multiple of H_kv.  lengths (int32 [B]): tokens of each
    row, the rest is padding (zeros in the output).  pos (int64 [B]) or t0: the position of each row's first token.
    cache_k / cache_v [B,H_kv,sinks+window,d]: the rings before the call.  Returns (o, lse, cache_k_out, cache_v_out);
    lse is float32 [B,H,L] (None unless want_lse), the rings are those after the call (None unless want_cache).
    """
    B, H, L, d = q.shape
    Hkv, dt, dev = k.shape[1], q.dtype, q.get_device()
    p, need = _window_params("bla_window_forward", B, H, Hkv, L, d, window, sinks, t0, scale, dt)
    _check_on(q, (B, H, L, d), dt, "q", dev)
    _check_on(k, (B, Hkv, L, d), dt, "k", dev)
    _check_on(v, (B, Hkv, L, d), dt, "v", dev)
    ring = (B, Hkv, sinks + window, d)
    if (cache_k is None) != (cache_v is None):
        raise ValueError("cache_k and cache_v: both or neither")
    if cache_k is not None:
        _check_on(cache_k, ring, dt, "cache_k", dev)
        _check_on(cache_v, ring, dt, "cache_v", dev)
    if lengths is not None:
        _check_on(lengths, (B,), torch.int32, "lengths", dev)
    if pos is not None:
        _check_on(pos, (B,), torch.int64, "pos", dev)
    o = _result(out, q, (B, H, L, d))
    lse = torch.empty((B, H, L), dtype=torch.float32, device=q.device) if want_lse else None
    ck = torch.empty(ring, dtype=dt, device=q.device) if want_cache else None
    cv = torch.empty(ring, dtype=dt, device=q.device) if want_cache else None
    keep, ws, n = _room(workspace, need, q)
    _call(lib().bla_window_forward, "bla_window_forward", dev, p, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(lengths),
          _ptr(pos), _ptr(cache_k), _ptr(cache_v), o.data_ptr(), _ptr(lse), _ptr(ck), _ptr(cv), ws, n)
    return o, lse, ck, cv


def window_step(q, k, v, window: int, sinks: int, cache_k, cache_v, pos=None, t0: int = 0, scale: float | None = None,
                workspace=None, out=None):
    """bla_window_step: one decode token per row, q [B,H,d], k and v [B,H_kv,d]; the rings cache_k / cache_v
    [B,H_kv,sinks+window,d] take its key and value in place.  A row with a negative pos is idle (zeros)."""
    B, H, d = q.shape
    Hkv, dt, dev = k.shape[1], q.dtype, q.get_device()
    p, need = _window_params("bla_window_step", B, H, Hkv, 1, d, window, sinks, t0, scale, dt)
    _check_on(q, (B, H, d), dt, "q", dev)
    _check_on(k, (B, Hkv, d), dt, "k", dev)
    _check_on(v, (B, Hkv, d), dt, "v", dev)
    ring = (B, Hkv, sinks + window, d)
    _check_on(cache_k, ring, dt, "cache_k", dev)
    _check_on(cache_v, ring, dt, "cache_v", dev)
    if pos is not None:
        _check_on(pos, (B,), torch.int64, "pos", dev)
    o = _result(out, q, (B, H, d))
    keep, ws, n = _room(workspace, need, q)
    _call(lib().bla_window_step, "bla_window_step", dev, p, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(pos),
          cache_k.data_ptr(), cache_v.data_ptr(), o.data_ptr(), ws, n)
    return o


def window_backward(q, k, v, o, lse, dO, window: int, sinks: int = 0, scale: float | None = None, lengths=None,
                    workspace=None):
    """bla_window_backward: (dq, dk, dv) of window_forward without rings from its outputs o and lse and dO = dLoss/dO."""
    B, H, L, d = q.shape
    Hkv, dt, dev = k.shape[1], q.dtype, q.get_device()
    p, need = _window_params("bla_window_backward", B, H, Hkv, L, d, window, sinks, 0, scale, dt)
    for name, t, h in (("q", q, H), ("k", k, Hkv), ("v", v, Hkv), ("o", o, H), ("dO", dO, H)):
        _check_on(t, (B, h, L, d), dt, name, dev)
    _check_on(lse, (B, H, L), torch.float32, "lse", dev)
    if lengths is not None:
        _check_on(lengths, (B,), torch.int32, "lengths", dev)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    keep, ws, n = _room(workspace, need, q)
    _call(lib().bla_window_backward, "bla_window_backward", dev, p, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(),
          lse.data_ptr(), dO.data_ptr(), _ptr(lengths), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ws, n)
    return dq, dk, dv


# ---- window attention with a learned bias ----

def bias_edges(buckets: int, max_distance: int) -> tuple:
    """The edges of the usual buckets of a causal relative position bias: half of the buckets hold one distance each, the bounds of the
    others are in geometric progression up to max_distance, the last holds what is beyond.  Bucket half + e begins at the smallest whole n with
    (n / half)^m >= (max_distance / half)^e, m = buckets - half, found in whole numbers."""
    half = int(buckets) // 2
    m, far = int(buckets) - half, int(max_distance)
    if half < 1 or far < half:
        raise ValueError(f"bias_edges: expected buckets >= 2 and max_distance >= buckets // 2, got {buckets} and {max_distance}")
    edges = list(range(1, half + 1))
    for e in range(1, m):
        lo, hi, want = half, far, half ** m * far ** e
        while lo < hi:
            n = (lo + hi) // 2
            if n ** m * half ** e >= want:
                hi = n
            else:
                lo = n + 1
        edges.append(lo)
    return tuple(edges)


@functools.lru_cache(maxsize=256)
def _edge_array(edges):
    _int32("bla_bias", *edges)
    return (ctypes.c_int32 * max(len(edges), 1))(*edges)


def _bias_check(bias, edges, H, dev):
    """(buckets, the edges' host array)."""
    edges = tuple(map(operator.index, edges))
    _check_on(bias, (H, len(edges) + 1), torch.float32, "bias", dev)
    return len(edges) + 1, _edge_array(edges)


def bias_forward(q, k, v, bias, edges, window: int, sinks: int = 0, t0: int = 0, scale: float | None = None, lengths=None, pos=None,
                 cache_k=None, cache_v=None, want_lse: bool = False, want_cache: bool = False, workspace=None, out=None):
    """bla_bias_forward: window_forward whose scores carry bias[h][bucket(p - j)].

    bias [H, len(edges) + 1] float32; edges: whole numbers on the host, ascending; a distance's bucket is the number of edges at or below it
    (bias_edges gives the usual ones).  The rest, and what returns, as for window_forward.
    """
    B, H, L, d = q.shape
    Hkv, dt, dev = k.shape[1], q.dtype, q.get_device()
    p, need = _window_params("bla_window_forward", B, H, Hkv, L, d, window, sinks, t0, scale, dt)
    _check_on(q, (B, H, L, d), dt, "q", dev)
    _check_on(k, (B, Hkv, L, d), dt, "k", dev)
    _check_on(v, (B, Hkv, L, d), dt, "v", dev)
    n, e = _bias_check(bias, edges, H, dev)
    ring = _past_check(B, Hkv, d, window, sinks, dt, dev, cache_k, cache_v, lengths, pos)
    o = _result(out, q, (B, H, L, d))
    lse = q.new_empty((B, H, L), dtype=torch.float32) if want_lse else None
    ck, cv = (q.new_empty(ring), q.new_empty(ring)) if want_cache else (None, None)
    keep, ws, m = _room(workspace, need, q)
    _call(lib().bla_bias_forward, "bla_bias_forward", dev, p, n, e, q.data_ptr(), k.data_ptr(), v.data_ptr(), bias.data_ptr(), _ptr(lengths),
          _ptr(pos), _ptr(cache_k), _ptr(cache_v), o.data_ptr(), _ptr(lse), _ptr(ck), _ptr(cv), ws, m)
    return o, lse, ck, cv


def _past_check(B, Hkv, d, window, sinks, dt, dev, cache_k, cache_v, lengths, pos):
    """The checks of a prompt's rings, lengths and positions: the rings' shape."""
    ring = (B, Hkv, sinks + window, d)
    if (cache_k is None) != (cache_v is None):
        raise ValueError("cache_k and cache_v: both or neither")
    if cache_k is not None:
        _check_on(cache_k, ring, dt, "cache_k", dev)
        _check_on(cache_v, ring, dt, "cache_v", dev)
    if lengths is not None:
        _check_on(lengths, (B,), torch.int32, "lengths", dev)
    if pos is not None:
        _check_on(pos, (B,), torch.int64, "pos", dev)
    return ring


def _step_check(q, k, v, window, sinks, cache_k, cache_v, pos):
    """The checks of a single token's tensors and rings."""
    B, H, d = q.shape
    Hkv, dt, dev = k.shape[1], q.dtype, q.get_device()
    _check_on(q, (B, H, d), dt, "q", dev)
    _check_on(k, (B, Hkv, d), dt, "k", dev)
    _check_on(v, (B, Hkv, d), dt, "v", dev)
    _check_on(cache_k, (B, Hkv, sinks + window, d), dt, "cache_k", dev)
    _check_on(cache_v, (B, Hkv, sinks + window, d), dt, "cache_v", dev)
    if pos is not None:
        _check_on(pos, (B,), torch.int64, "pos", dev)


def bias_step(q, k, v, bias, edges, window: int, sinks: int, cache_k, cache_v, pos=None, t0: int = 0, scale: float | None = None,
              workspace=None, out=None):
    """bla_bias_step: window_step whose scores carry the bias of bias_forward."""
    B, H, d = q.shape
    Hkv, dev = k.shape[1], q.get_device()
    p, need = _window_params("bla_bias_step", B, H, Hkv, 1, d, window, sinks, t0, scale, q.dtype)
    _step_check(q, k, v, window, sinks, cache_k, cache_v, pos)
    n, e = _bias_check(bias, edges, H, dev)
    o = _result(out, q, (B, H, d))
    keep, ws, m = _room(workspace, need, q)
    _call(lib().bla_bias_step, "bla_bias_step", dev, p, n, e, q.data_ptr(), k.data_ptr(), v.data_ptr(), bias.data_ptr(), _ptr(pos),
          cache_k.data_ptr(), cache_v.data_ptr(), o.data_ptr(), ws, m)
    return o


def bias_backward(q, k, v, o, lse, dO, bias, edges, window: int, sinks: int = 0, scale: float | None = None, lengths=None, workspace=None):
    """bla_bias_backward: (dq, dk, dv, dbias) of bias_forward without rings from its outputs o and lse and dO = dLoss/dO; dbias is float32."""
    B, H, L, d = q.shape
    Hkv, dt, dev = k.shape[1], q.dtype, q.get_device()
    p, _ = _window_params("bla_window_backward", B, H, Hkv, L, d, window, sinks, 0, scale, dt)
    for name, t, h in (("q", q, H), ("k", k, Hkv), ("v", v, Hkv), ("o", o, H), ("dO", dO, H)):
        _check_on(t, (B, h, L, d), dt, name, dev)
    _check_on(lse, (B, H, L), torch.float32, "lse", dev)
    n, e = _bias_check(bias, edges, H, dev)
    if lengths is not None:
        _check_on(lengths, (B,), torch.int32, "lengths", dev)
    dq, dk, dv, db = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), torch.empty_like(bias)
    keep, ws, m = _room(workspace, lib().bla_bias_backward_workspace_size(p, n), q)
    _call(lib().bla_bias_backward, "bla_bias_backward", dev, p, n, e, q.data_ptr(), k.data_ptr(), v.data_ptr(), bias.data_ptr(), o.data_ptr(),
          lse.data_ptr(), dO.data_ptr(), _ptr(lengths), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), db.data_ptr(), ws, m)
    return dq, dk, dv, db


# ---- window attention behind a shared prefix ----

@functools.lru_cache(maxsize=256)
def _prefix_plan(what, B, H, Hkv, L, d, window, sinks, scale, dtype, P, G):
    _int32(what, B, H, Hkv, L, d, window, sinks, P, G)
    block = PrefixParams(WindowParams(B, H, Hkv, L, d, window, sinks, _io(dtype, "q"), 0, scale), P, G)
    p = ctypes.byref(block)
    st = lib().bla_prefix_supported(p)
    if what == "bla_prefix_forward" or st != 2:  # the step's launch has a limit of its own, which it checks
        _shape_status(st, what)
    return block, p, getattr(lib(), what.replace("_forward", "") + "_workspace_size")(p)


def _prefix_check(what, q, k, prefix_k, prefix_v, prefix_lengths, L, window, sinks, t0, scale):
    """(parameters by reference, workspace bytes)."""
    B, H, d = q.shape[0], q.shape[1], q.shape[-1]
    Hkv, dt, dev = k.shape[1], q.dtype, q.get_device()
    if prefix_k.dim() != 4:
        raise ValueError(f"prefix_k: expected [G, H_kv, P, d], got {tuple(prefix_k.shape)}")
    G, P = prefix_k.shape[0], prefix_k.shape[2]
    _check_on(prefix_k, (G, Hkv, P, d), dt, "prefix_k", dev)
    _check_on(prefix_v, (G, Hkv, P, d), dt, "prefix_v", dev)
    if prefix_lengths is not None:
        _check_on(prefix_lengths, (G,), torch.int32, "prefix_lengths", dev)
    block, p, need = _prefix_plan(what, B, H, Hkv, L, d, int(window), int(sinks), 0.0 if scale is None else float(scale), dt, P, G)
    if t0 != 0:
        if not -(1 << 63) <= t0 < 1 << 63:
            raise BlaError(1, what)
        block = PrefixParams.from_buffer_copy(block)
        block.w.t0 = int(t0)
        p = ctypes.byref(block)
    return p, need


def prefix_forward(q, k, v, prefix_k, prefix_v, window: int, sinks: int = 0, t0: int = 0, scale: float | None = None, lengths=None, pos=None,
                   prefix_lengths=None, cache_k=None, cache_v=None, want_lse: bool = False, want_cache: bool = False, workspace=None, out=None):
    """bla_prefix_forward: window_forward whose queries also see every token of a prefix that rows share.

    prefix_k, prefix_v [G,H_kv,P,d]: rows b with the same b // (B // G) share one; prefix_lengths (int32 [G]): its tokens (None: all P).
    The rest, and what returns, as for window_forward: the window, the rings and positions are those of the row's own tokens.
    """
    B, H, L, d = q.shape
    Hkv, dt, dev = k.shape[1], q.dtype, q.get_device()
    p, need = _prefix_check("bla_prefix_forward", q, k, prefix_k, prefix_v, prefix_lengths, L, window, sinks, t0, scale)
    _check_on(q, (B, H, L, d), dt, "q", dev)
    _check_on(k, (B, Hkv, L, d), dt, "k", dev)
    _check_on(v, (B, Hkv, L, d), dt, "v", dev)
    ring = _past_check(B, Hkv, d, window, sinks, dt, dev, cache_k, cache_v, lengths, pos)
    o = _result(out, q, (B, H, L, d))
    lse = q.new_empty((B, H, L), dtype=torch.float32) if want_lse else None
    ck, cv = (q.new_empty(ring), q.new_empty(ring)) if want_cache else (None, None)
    keep, ws, n = _room(workspace, need, q)
    _call(lib().bla_prefix_forward, "bla_prefix_forward", dev, p, q.data_ptr(), k.data_ptr(), v.data_ptr(), prefix_k.data_ptr(),
          prefix_v.data_ptr(), _ptr(prefix_lengths), _ptr(lengths), _ptr(pos), _ptr(cache_k), _ptr(cache_v), o.data_ptr(), _ptr(lse), _ptr(ck),
          _ptr(cv), ws, n)
    return o, lse, ck, cv


def prefix_step(q, k, v, prefix_k, prefix_v, window: int, sinks: int, cache_k, cache_v, pos=None, t0: int = 0, scale: float | None = None,
                prefix_lengths=None, workspace=None, out=None):
    """bla_prefix_step: window_step behind the prefix of prefix_forward, which is read once for all the rows that share it."""
    B, H, d = q.shape
    dev = q.get_device()
    p, need = _prefix_check("bla_prefix_step", q, k, prefix_k, prefix_v, prefix_lengths, 1, window, sinks, t0, scale)
    _step_check(q, k, v, window, sinks, cache_k, cache_v, pos)
    o = _result(out, q, (B, H, d))
    keep, ws, n = _room(workspace, need, q)
    _call(lib().bla_prefix_step, "bla_prefix_step", dev, p, q.data_ptr(), k.data_ptr(), v.data_ptr(), prefix_k.data_ptr(), prefix_v.data_ptr(),
          _ptr(prefix_lengths), _ptr(pos), cache_k.data_ptr(), cache_v.data_ptr(), o.data_ptr(), ws, n)
    return o


# ---- attention over a cache of bounded size ----

@functools.lru_cache(maxsize=256)
def _evict_plan(what, B, H, Hkv, L, d, slots, recent, scale, dtype):
    _int32(what, B, H, Hkv, L, d, slots, recent)
    block = EvictParams(B, H, Hkv, L, d, slots, recent, _io(dtype, "k"), 0, scale)
    p = ctypes.byref(block)
    st = lib().bla_evict_supported(p)
    if what == "bla_evict_forward" or st != 2:  # the launches of the other calls have limits of their own, which they check
        _shape_status(st, what)
    return block, p, 0 if what == "bla_evict_select" else getattr(lib(), what.replace("_forward", "") + "_workspace_size")(p)


def _evict_params(what, B, H, Hkv, L, d, slots, recent, t0, scale, dtype):
    """(parameters by reference, workspace bytes)."""
    block, p, need = _evict_plan(what, B, H, Hkv, L, d, int(slots), int(recent), 0.0 if scale is None else float(scale), dtype)
    if t0 != 0:
        if not -(1 << 63) <= t0 < 1 << 63:
            raise BlaError(1, what)
        block = EvictParams.from_buffer_copy(block)
        block.t0 = int(t0)
        p = ctypes.byref(block)
    return p, need


def _evict_cache(cache_k, cache_v, other, name, dtype, B, Hkv, slots, d, dt, dev):
    """The checks of a cache, which comes with its scores or positions or not at all."""
    given = [x is not None for x in (cache_k, cache_v, other)]
    if any(given) and not all(given):
        raise ValueError(f"cache_k, cache_v and {name}: all or none")
    if cache_k is not None:
        _check_on(cache_k, (B, Hkv, slots, d), dt, "cache_k", dev)
        _check_on(cache_v, (B, Hkv, slots, d), dt, "cache_v", dev)
        _check_on(other, (B, Hkv, slots), dtype, name, dev)


def evict_forward(q, k, v, slots: int, cache_k=None, cache_v=None, score=None, t0: int = 0, scale: float | None = None, lengths=None, pos=None,
                  want_lse: bool = False, workspace=None, out=None):
    """bla_evict_forward: attention of L tokens over a cache of up to `slots` tokens and themselves, and the weight that each token gets.

    q [B,H,L,d], k and v [B,H_kv,L,d]; cache_k / cache_v [B,H_kv,slots,d] with score [B,H_kv,slots] float32 (all or none): a row at position
    pos (int64 [B], or t0) has min(pos, slots) tokens there.  lengths (int32 [B]): tokens of each row.  Returns (o, lse or None, scores after the call
    [B,H_kv,slots+L]: the cache's entries, then the call's); evict_select makes the cache after the call of them.
    """
    B, H, L, d = q.shape
    Hkv, dt, dev = k.shape[1], q.dtype, q.get_device()
    p, need = _evict_params("bla_evict_forward", B, H, Hkv, L, d, slots, 0, t0, scale, dt)
    _check_on(q, (B, H, L, d), dt, "q", dev)
    _check_on(k, (B, Hkv, L, d), dt, "k", dev)
    _check_on(v, (B, Hkv, L, d), dt, "v", dev)
    _evict_cache(cache_k, cache_v, score, "score", torch.float32, B, Hkv, slots, d, dt, dev)
    if lengths is not None:
        _check_on(lengths, (B,), torch.int32, "lengths", dev)
    if pos is not None:
        _check_on(pos, (B,), torch.int64, "pos", dev)
    o = _result(out, q, (B, H, L, d))
    lse = q.new_empty((B, H, L), dtype=torch.float32) if want_lse else None
    after = q.new_empty((B, Hkv, slots + L), dtype=torch.float32)
    keep, ws, n = _room(workspace, need, q)
    _call(lib().bla_evict_forward, "bla_evict_forward", dev, p, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(lengths), _ptr(pos), _ptr(cache_k),
          _ptr(cache_v), _ptr(score), o.data_ptr(), _ptr(lse), after.data_ptr(), ws, n)
    return o, lse, after


def evict_select(k, v, score, slots: int, recent: int = 0, cache_k=None, cache_v=None, at=None, t0: int = 0, lengths=None, pos=None):
    """bla_evict_select: the cache after L tokens: of the cache's tokens and the call's k, v [B,H_kv,L,d] the newest `recent` stay, and of the others those
    with the largest score [B,H_kv,slots+L] (of equal ones the lowest entries), `slots` in all, in the order of their entries.

    cache_k / cache_v [B,H_kv,slots,d] and at [B,H_kv,slots] int64 (the tokens' positions): all or none.  Returns (cache_k, cache_v, score, at)
    after the call, new tensors; slots without a token hold zeros and a position of -1.  Without a cache a row should be at position 0 or have `slots` tokens
    or more: a later call takes min(position, slots) of the slots as tokens.
    """
    B, Hkv, L, d = k.shape
    dt, dev = k.dtype, k.get_device()
    p, _ = _evict_params("bla_evict_select", B, Hkv, Hkv, L, d, slots, recent, t0, None, dt)
    _check_on(k, (B, Hkv, L, d), dt, "k", dev)
    _check_on(v, (B, Hkv, L, d), dt, "v", dev)
    _check_on(score, (B, Hkv, slots + L), torch.float32, "score", dev)
    _evict_cache(cache_k, cache_v, at, "at", torch.int64, B, Hkv, slots, d, dt, dev)
    if lengths is not None:
        _check_on(lengths, (B,), torch.int32, "lengths", dev)
    if pos is not None:
        _check_on(pos, (B,), torch.int64, "pos", dev)
    ck, cv = k.new_empty((B, Hkv, slots, d)), k.new_empty((B, Hkv, slots, d))
    kept = score.new_empty((B, Hkv, slots))
    where = k.new_empty((B, Hkv, slots), dtype=torch.int64)
    _call(lib().bla_evict_select, "bla_evict_select", dev, p, k.data_ptr(), v.data_ptr(), score.data_ptr(), _ptr(lengths), _ptr(pos), _ptr(cache_k),
          _ptr(cache_v), _ptr(at), ck.data_ptr(), cv.data_ptr(), kept.data_ptr(), where.data_ptr())
    return ck, cv, kept, where


def evict_step(q, k, v, cache_k, cache_v, score, at, recent: int = 0, pos=None, t0: int = 0, scale: float | None = None, workspace=None,
               out=None, score_out=None, at_out=None):
    """bla_evict_step: one decode token per row, q [B,H,d], k and v [B,H_kv,d], over a cache [B,H_kv,slots,d] that takes it in place: in slot pos while it is not
    full, then in that of the least score among the tokens older than the newest `recent` before it (evict_select counts the call's own among
    them).  score [B,H_kv,slots] float32 and at [B,H_kv,slots] int64 are updated in place, or written to score_out and at_out.  A row with a negative pos is idle (zeros).  Returns (o, score after the call, at after the call)."""
    B, H, d = q.shape
    Hkv, dt, dev = k.shape[1], q.dtype, q.get_device()
    if cache_k.dim() != 4:
        raise ValueError(f"cache_k: expected [B, H_kv, slots, d], got {tuple(cache_k.shape)}")
    slots = cache_k.shape[2]
    p, need = _evict_params("bla_evict_step", B, H, Hkv, 1, d, slots, recent, t0, scale, dt)
    _step_check(q, k, v, slots, 0, cache_k, cache_v, pos)
    _check_on(score, (B, Hkv, slots), torch.float32, "score", dev)
    _check_on(at, (B, Hkv, slots), torch.int64, "at", dev)
    for x, like, name in ((score_out, score, "score_out"), (at_out, at, "at_out")):
        if x is not None:
            _check_on(x, like.shape, like.dtype, name, dev)
    score_out, at_out = score if score_out is None else score_out, at if at_out is None else at_out
    o = _result(out, q, (B, H, d))
    keep, ws, n = _room(workspace, need, q)
    _call(lib().bla_evict_step, "bla_evict_step", dev, p, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(pos), cache_k.data_ptr(), cache_v.data_ptr(),
          score.data_ptr(), at.data_ptr(), o.data_ptr(), score_out.data_ptr(), at_out.data_ptr(), ws, n)
    return o, score_out, at_out


@functools.lru_cache(maxsize=256)
def _conv_plan(what, B, H, L, d, K, silu, dtype):
    _int32(what, B, H, L, d, K, silu)
    p = ctypes.byref(ConvParams(B, H, L, d, K, silu, _io(dtype, "x")))
    _shape_status(lib().bla_conv_supported(p), what)
    return p, lib().bla_conv_backward_workspace_size(p)


def _conv_check(x, w, bias, silu, what):
    """The checks that the convolution's calls share: (parameters, bytes of the backward's workspace, taps)."""
    H, d, dev = x.shape[1], x.shape[-1], x.get_device()
    if w.dim() != 3:
        raise ValueError(f"w: expected [H, d, taps], got {tuple(w.shape)}")
    K = w.shape[2]
    p, need = _conv_plan(what, x.shape[0], H, x.shape[2] if x.dim() == 4 else 1, d, K, int(silu), x.dtype)
    _check_on(x, x.shape, x.dtype, "x", dev)
    _check_on(w, (H, d, K), torch.float32, "w", dev)
    if bias is not None:
        _check_on(bias, (H, d), torch.float32, "bias", dev)
    return p, need, K


def conv_forward(x, w, bias=None, silu: bool = True, state=None, lengths=None, want_state: bool = True, out=None):
    """bla_conv_forward: the causal convolution of each channel of x [B,H,L,d] (float32 or bfloat16) with w [H,d,taps] and
    bias [H,d] (float32), then SiLU if silu.  state [B,H,taps-1,d] float32: the tokens before the call (None = zeros).
    lengths (int32 [B]): tokens of each row.  Returns (y, state after the call or None)."""
    B, H, L, d = x.shape
    dev = x.get_device()
    p, _, K = _conv_check(x, w, bias, silu, "bla_conv_forward")
    if state is not None:
        _check_on(state, (B, H, K - 1, d), torch.float32, "state", dev)
    if lengths is not None:
        _check_on(lengths, (B,), torch.int32, "lengths", dev)
    y = _result(out, x, (B, H, L, d))
    so = torch.empty((B, H, K - 1, d), dtype=torch.float32, device=x.device) if want_state else None
    _call(lib().bla_conv_forward, "bla_conv_forward", dev, p, x.data_ptr(), w.data_ptr(), _ptr(bias), _ptr(lengths),
          _ptr(state), y.data_ptr(), _ptr(so))
    return y, so


def conv_step(x, w, state, bias=None, silu: bool = True, state_out=None, out=None):
    """bla_conv_step: one token per row, x [B,H,d].  The state [B,H,taps-1,d] is updated in place, or left alone where
    state_out receives it."""
    B, H, d = x.shape
    dev = x.get_device()
    p, _, K = _conv_check(x, w, bias, silu, "bla_conv_step")
    _check_on(state, (B, H, K - 1, d), torch.float32, "state", dev)
    if state_out is None:
        state_out = state
    else:
        _check_on(state_out, (B, H, K - 1, d), torch.float32, "state_out", dev)
    y = _result(out, x, (B, H, d))
    _call(lib().bla_conv_step, "bla_conv_step", dev, p, x.data_ptr(), w.data_ptr(), _ptr(bias), state.data_ptr(),
          y.data_ptr(), state_out.data_ptr())
    return y


def conv_backward(x, w, dy, bias=None, silu: bool = True, state=None, dstate=None, lengths=None,
                  want_state_grad: bool = True, workspace=None):
    """bla_conv_backward: gradients of conv_forward for dy = dLoss/dy and dstate = dLoss/d(state after the call) (None =
    zero).  Returns (dx, dw, dbias, dLoss/d(state before the call) or None); dbias is that of a zero bias where bias is
    None."""
    B, H, L, d = x.shape
    dev = x.get_device()
    p, need, K = _conv_check(x, w, bias, silu, "bla_conv_backward")
    _check_on(dy, (B, H, L, d), x.dtype, "dy", dev)
    for name, t in (("state", state), ("dstate", dstate)):
        if t is not None:
            _check_on(t, (B, H, K - 1, d), torch.float32, name, dev)
    if lengths is not None:
        _check_on(lengths, (B,), torch.int32, "lengths", dev)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    db = torch.empty((H, d), dtype=torch.float32, device=x.device)
    ds = torch.empty((B, H, K - 1, d), dtype=torch.float32, device=x.device) if want_state_grad else None
    keep, ws, n = _room(workspace, need, x)
    _call(lib().bla_conv_backward, "bla_conv_backward", dev, p, x.data_ptr(), w.data_ptr(), _ptr(bias), dy.data_ptr(),
          _ptr(lengths), _ptr(state), _ptr(dstate), dx.data_ptr(), dw.data_ptr(), db.data_ptr(), _ptr(ds), ws, n)
    return dx, dw, db, ds


@functools.lru_cache(maxsize=256)
def _ssm_plan(size, what, B, H, G, L, d, N, dtype):
    _int32(what, B, H, G, L, d, N)
    p = ctypes.byref(SsmParams(B, H, G, L, d, N, _io(dtype, "x")))
    _shape_status(lib().bla_ssm_supported(p), what)
    return p, getattr(lib(), size)(p) if size else 0


def _ssm_check(x, dt, A, Bm, Cm, D, size, what):
    """The checks that the scan's calls share: (parameters, workspace bytes, shape of a state)."""
    tok = x.shape[2:-1]
    B, H, d, io, dev = x.shape[0], x.shape[1], x.shape[-1], x.dtype, x.get_device()
    if Bm.dim() != x.dim():
        raise ValueError(f"Bm: expected {x.dim()} dimensions, got {tuple(Bm.shape)}")
    G, N = Bm.shape[1], Bm.shape[-1]
    p, need = _ssm_plan(size, what, B, H, G, tok[0] if tok else 1, d, N, io)
    _check_on(x, x.shape, io, "x", dev)
    _check_on(Bm, (B, G, *tok, N), io, "Bm", dev)
    _check_on(Cm, (B, G, *tok, N), io, "Cm", dev)
    _check_on(dt, (B, H, *tok), torch.float32, "dt", dev)
    _check_on(A, (H,), torch.float32, "A", dev)
    if D is not None:
        _check_on(D, (H,), torch.float32, "D", dev)
    return p, need, (B, H, N, d)


def ssm_forward(x, dt, A, Bm, Cm, D=None, state=None, lengths=None, want_state: bool = True, workspace=None, out=None):
    """bla_ssm_forward: the selective state space scan h_t = exp(dt_t A) h_{t-1} + dt_t B_t x_t^T, y_t = C_t h_t + D x_t.

    x [B,H,L,d], Bm and Cm [B,G,L,N] (float32 or bfloat16), dt [B,H,L], A and D [H] (float32; D None = zero), state
    [B,H,N,d] float32 before the call (None = zero), lengths (int32 [B]): tokens of each row.  Returns (y, state after
    the call or None)."""
    B, H, L, d = x.shape
    dev = x.get_device()
    p, need, shape = _ssm_check(x, dt, A, Bm, Cm, D, "bla_ssm_workspace_size", "bla_ssm_forward")
    if state is not None:
        _check_on(state, shape, torch.float32, "state", dev)
    if lengths is not None:
        _check_on(lengths, (B,), torch.int32, "lengths", dev)
    y = _result(out, x, (B, H, L, d))
    so = torch.empty(shape, dtype=torch.float32, device=x.device) if want_state else None
    keep, ws, n = _room(workspace, need, x)
    _call(lib().bla_ssm_forward, "bla_ssm_forward", dev, p, x.data_ptr(), dt.data_ptr(), A.data_ptr(), Bm.data_ptr(),
          Cm.data_ptr(), _ptr(D), _ptr(lengths), _ptr(state), y.data_ptr(), _ptr(so), ws, n)
    return y, so


def ssm_step(x, dt, A, Bm, Cm, state, D=None, state_out=None, out=None):
    """bla_ssm_step: one token per row, x [B,H,d], dt [B,H], Bm and Cm [B,G,N].  The state [B,H,N,d] is updated in place, or
    left alone where state_out receives it."""
    B, H, d = x.shape
    dev = x.get_device()
    p, _, shape = _ssm_check(x, dt, A, Bm, Cm, D, None, "bla_ssm_step")
    _check_on(state, shape, torch.float32, "state", dev)
    if state_out is None:
        state_out = state
    else:
        _check_on(state_out, shape, torch.float32, "state_out", dev)
    y = _result(out, x, (B, H, d))
    _call(lib().bla_ssm_step, "bla_ssm_step", dev, p, x.data_ptr(), dt.data_ptr(), A.data_ptr(), Bm.data_ptr(),
          Cm.data_ptr(), _ptr(D), state.data_ptr(), y.data_ptr(), state_out.data_ptr())
    return y


def ssm_backward(x, dt, A, Bm, Cm, dy, D=None, state=None, dstate=None, lengths=None, want_state_grad: bool = True,
                 workspace=None):
    """bla_ssm_backward: gradients of ssm_forward for dy = dLoss/dy and dstate = dLoss/d(state after the call) (None =
    zero).  Returns (dx, ddt, dA, dBm, dCm, dD, dLoss/d(state before the call) or None); dD is that of a zero D where D is
    None."""
    B, H, L, d = x.shape
    dev = x.get_device()
    p, need, shape = _ssm_check(x, dt, A, Bm, Cm, D, "bla_ssm_backward_workspace_size", "bla_ssm_backward")
    _check_on(dy, (B, H, L, d), x.dtype, "dy", dev)
    for name, t in (("state", state), ("dstate", dstate)):
        if t is not None:
            _check_on(t, shape, torch.float32, name, dev)
    if lengths is not None:
        _check_on(lengths, (B,), torch.int32, "lengths", dev)
    dx, ddt, dA = torch.empty_like(x), torch.empty_like(dt), torch.empty_like(A)
    dB, dC, dD = torch.empty_like(Bm), torch.empty_like(Cm), torch.empty_like(A)
    ds = torch.empty(shape, dtype=torch.float32, device=x.device) if want_state_grad else None
    keep, ws, n = _room(workspace, need, x)
    _call(lib().bla_ssm_backward, "bla_ssm_backward", dev, p, x.data_ptr(), dt.data_ptr(), A.data_ptr(), Bm.data_ptr(),
          Cm.data_ptr(), _ptr(D), dy.data_ptr(), _ptr(lengths), _ptr(state), _ptr(dstate), dx.data_ptr(), ddt.data_ptr(),
          dA.data_ptr(), dB.data_ptr(), dC.data_ptr(), dD.data_ptr(), _ptr(ds), ws, n)
    return dx, ddt, dA, dB, dC, dD, ds
