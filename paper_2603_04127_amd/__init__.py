"""Python binding over the C-ABI DARK attention library (libdark.so).

Argument marshalling only: every step of the computation runs in the HIP
kernels behind ``include/dark.h``.  PyTorch supplies device memory (tensors)
and the current HIP stream.  There is no CPU fallback: if the shared library is
missing the import of this binding's functions raises.
"""
from __future__ import annotations

import ctypes
import math
import os
import threading
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdark.so")

DARK_OK, DARK_EINVAL, DARK_EUNSUPPORTED, DARK_EWORKSPACE, DARK_EALIGN, DARK_EHIP, DARK_ESCRATCH = range(7)
DARK_F32, DARK_BF16 = 0, 1
OP_FEATURIZE, OP_ATTN_FWD, OP_ATTN_CAUSAL_FWD, OP_ATTN_BWD, OP_WHITEN = range(5)
PATH_AUTO, PATH_F32, PATH_FUSED = range(3)
BHLD, BLHD = range(2)


class DarkParams(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("L", ctypes.c_int32),
        ("d", ctypes.c_int32), ("r", ctypes.c_int32), ("m", ctypes.c_int32), ("dv", ctypes.c_int32),
        ("chunk", ctypes.c_int32), ("io_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32),
        ("scale", ctypes.c_float), ("w_shared", ctypes.c_int32), ("path", ctypes.c_int32),
        ("sched_kv_wgs", ctypes.c_int32), ("sched_ro_wgs", ctypes.c_int32), ("sched_cs_wgs", ctypes.c_int32),
        ("sched_cs_state", ctypes.c_int32),
    ]


class DecayParams(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("L", ctypes.c_int32), ("dk", ctypes.c_int32), ("dv", ctypes.c_int32),
        ("io_dtype", ctypes.c_int32), ("layout", ctypes.c_int32), ("scale", ctypes.c_float), ("sched_segments", ctypes.c_int32),
    ]


class DeltaParams(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("L", ctypes.c_int32), ("dk", ctypes.c_int32), ("dv", ctypes.c_int32),
        ("io_dtype", ctypes.c_int32), ("layout", ctypes.c_int32), ("scale", ctypes.c_float),
    ]


class BeamParams(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("n", ctypes.c_int32), ("V", ctypes.c_int32), ("io_dtype", ctypes.c_int32), ("eos", ctypes.c_int32),
        ("keep_slots", ctypes.c_int32),
    ]


class SampleParams(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("V", ctypes.c_int32), ("io_dtype", ctypes.c_int32), ("top_k", ctypes.c_int32), ("temperature", ctypes.c_float),
        ("top_p", ctypes.c_float), ("min_p", ctypes.c_float),
    ]


class DarkError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


_lib = None


def lib() -> ctypes.CDLL:
    """Load libdark.so (built in-tree by ``build.py``); raises if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} not found: build it first (python -m paper_2603_04127_amd.build or __graft_entry__.build())")
    L = ctypes.CDLL(LIB_PATH)
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    pp = ctypes.POINTER(DarkParams)
    L.dark_version.restype = i32
    L.dark_status_string.restype = ctypes.c_char_p
    L.dark_status_string.argtypes = [i32]
    L.dark_workspace_bytes.restype = sz
    L.dark_workspace_bytes.argtypes = [pp, i32, i32]
    L.dark_featurize.restype = i32
    L.dark_featurize.argtypes = [pp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
    for f in (L.dark_attn_fwd, L.dark_attn_causal_fwd):
        f.restype = i32
        f.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.dark_attn_fwd_static.restype = i32
    L.dark_attn_fwd_static.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp]
    L.dark_static_scratch_bytes.restype = sz
    L.dark_attn_bwd.restype = i32
    L.dark_attn_bwd.argtypes = [pp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.dark_attn_bwd_dw.restype = i32
    L.dark_attn_bwd_dw.argtypes = [pp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.dark_decode_step.restype = i32
    L.dark_decode_step.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.dark_whiten.restype = i32
    L.dark_whiten.argtypes = [pp, vp, vp, vp, vp, vp, sz, vp]
    L.dark_saved_bytes.restype = sz
    L.dark_saved_bytes.argtypes = [pp]
    L.dark_attn_causal_fwd_save.restype = i32
    L.dark_attn_causal_fwd_save.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, sz, vp, sz, vp]
    L.dark_attn_bwd_saved.restype = i32
    L.dark_attn_bwd_saved.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, sz, vp, vp, vp, vp, vp, vp, sz, vp]
    dp, bp = ctypes.POINTER(DecayParams), ctypes.POINTER(BeamParams)
    L.dark_decay_workspace_bytes.restype = sz
    L.dark_decay_workspace_bytes.argtypes = [dp, i32]
    L.dark_decay_fwd.restype = i32
    L.dark_decay_fwd.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.dark_decay_bwd.restype = i32
    L.dark_decay_bwd.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.dark_decay_step.restype = i32
    L.dark_decay_step.argtypes = [dp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp]
    ep = ctypes.POINTER(DeltaParams)
    L.dark_delta_workspace_bytes.restype = sz
    L.dark_delta_workspace_bytes.argtypes = [ep, i32]
    L.dark_delta_fwd.restype = i32
    L.dark_delta_fwd.argtypes = [ep, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.dark_delta_bwd.restype = i32
    L.dark_delta_bwd.argtypes = [ep, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.dark_delta_step.restype = i32
    L.dark_delta_step.argtypes = [ep, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp]
    L.dark_beam_workspace_bytes.restype = sz
    L.dark_beam_workspace_bytes.argtypes = [bp]
    L.dark_beam_select.restype = i32
    L.dark_beam_select.argtypes = [bp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.dark_sample.restype = i32
    L.dark_sample.argtypes = [ctypes.POINTER(SampleParams), vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.dark_state_reorder.restype = i32
    L.dark_state_reorder.argtypes = [i32, i32, vp, i32, ctypes.POINTER(vp), ctypes.POINTER(sz), vp]
    L.dark_timing_enable.argtypes = [i32]
    L.dark_timing_enable.restype = None
    L.dark_timing_reset.restype = None
    L.dark_timing_slots.restype = i32
    L.dark_timing_read.restype = i32
    L.dark_timing_read.argtypes = [i32, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_int64),
                                   ctypes.POINTER(ctypes.c_double)]
    L.dark_timeline_read.restype = i32
    L.dark_timeline_read.argtypes = [i32, ctypes.POINTER(ctypes.c_int64), sz]
    L.dark_ceiling_copy.restype = i32
    L.dark_ceiling_copy.argtypes = [vp, vp, sz, vp]
    L.dark_ceiling_read.restype = i32
    L.dark_ceiling_read.argtypes = [vp, sz, vp, vp]
    L.dark_ceiling_mfma.restype = i32
    L.dark_ceiling_mfma.argtypes = [i32, vp, ctypes.POINTER(ctypes.c_double), vp]
    _lib = L
    return L


def status_string(status: int) -> str:
    return lib().dark_status_string(int(status)).decode()


def make_params(B, H, L, d, r, m, dv, *, io_dtype=DARK_F32, out_dtype=None, chunk=0, scale=0.0, w_shared=False,
                path=PATH_AUTO, sched=None) -> DarkParams:
    """`sched`: optional dict of the schedule overrides of dark_params (kv_wgs, ro_wgs, cs_wgs, cs_state)."""
    sched = sched or {}
    unknown = set(sched) - {"kv_wgs", "ro_wgs", "cs_wgs", "cs_state"}
    if unknown:
        raise ValueError(f"unknown schedule override(s) {sorted(unknown)}")
    return DarkParams(B, H, L, d, r, m, dv, chunk, io_dtype, io_dtype if out_dtype is None else out_dtype,
                      float(scale), int(bool(w_shared)), path, int(sched.get("kv_wgs", 0)), int(sched.get("ro_wgs", 0)),
                      int(sched.get("cs_wgs", 0)), int(sched.get("cs_state", 0)))


def workspace_bytes(p: DarkParams, op: int, causal: bool = False) -> int:
    return int(lib().dark_workspace_bytes(ctypes.byref(p), op, int(causal)))


# ----------------------------------------------------------------------------
# torch-facing helpers
# ----------------------------------------------------------------------------
def _torch():
    import torch
    return torch


def _dtype_code(t) -> int:
    torch = _torch()
    if t.dtype == torch.float32:
        return DARK_F32
    if t.dtype == torch.bfloat16:
        return DARK_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("tensors must be contiguous device tensors")
    return t.data_ptr()


def _stream() -> int:
    """The current HIP stream (the raw handle: building a torch.cuda.Stream around it takes 2.8 us)."""
    C = _torch()._C
    return C._cuda_getCurrentRawStream(C._cuda_getDevice())


# Scratch per device, stream and thread: calls on different streams, or enqueued by different threads, are not ordered against
# each other.  Each buffer is allocated under its stream, so that the allocator hands its memory on in that stream's order once it
# is replaced or, beyond the bound, dropped (oldest first; a call that is being enqueued holds its own reference).
_ws_cache = {}
_MAX_WORKSPACES = 8


def _workspace(nbytes: int, device):
    """(A device byte buffer of at least nbytes, owned by torch, and the current stream, whose calls it serves.)"""
    torch = _torch()
    index = device.index
    if index is None:   # host tensors: their pointers are refused
        return torch.empty(256, dtype=torch.uint8, device=device), None
    stream = _stream()
    # a graph keeps its own scratch: it may be replayed at any time (the default stream, 0, cannot be captured)
    if stream and torch._C._cuda_isCurrentStreamCapturing():
        return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device), stream
    key = (index, stream, threading.get_ident())
    buf = _ws_cache.get(key)
    if buf is None or buf.numel() < nbytes:
        _ws_cache.pop(key, None)
        buf = None
        _drop_oldest(_ws_cache, _MAX_WORKSPACES)
        buf = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        _ws_cache[key] = buf
    return buf, stream


def _drop_oldest(cache, most):
    while len(cache) >= most:
        try:
            cache.pop(next(iter(cache)), None)
        except (StopIteration, RuntimeError):   # another thread has just emptied or changed it
            pass


# Parameters and workspace size of a call, by everything they are derived from: shapes, dtypes and the values of the options
# (no tensor, no address; an option may come as a 0-d tensor, which hashes as the object and whose value changes in place).
# Deriving them anew takes 4 us of a call whose kernels take 8; bounded, oldest entries first.
_plans = {}
_MAX_PLANS = 256


def _plan(op, causal, Q, V, M, W, out_dtype=None, chunk=0, scale=0.0, path=PATH_AUTO, sched=None):
    """(DarkParams, workspace bytes of `op`) of a call."""
    scale = float(scale)
    # 128.0 finds the entry of 128 in a dictionary, but the parameter block takes whole numbers only: the types are part of
    # the key.  Schedule overrides are for tests and tuning: not kept.
    key = (op, causal, Q.shape, Q.dtype, None if V is None else V.shape, None if M is None else (M.shape, M.dtype), W.shape,
           W.dtype, out_dtype, chunk, chunk.__class__, scale, path, path.__class__)
    plan = None if sched else _plans.get(key)
    if plan is None:
        p = _params_from(Q, V, M, W, out_dtype=out_dtype, chunk=chunk, scale=scale, path=path, sched=sched)
        plan = (p, workspace_bytes(p, op, causal) if op is not None else 0)
        if not sched:
            _keep_plan(key, plan)
    return plan


def _keep_plan(key, plan):
    _drop_oldest(_plans, _MAX_PLANS)
    _plans[key] = plan


def _params_from(Q, V, M, W, *, out_dtype=None, chunk=0, scale=0.0, path=PATH_AUTO, sched=None) -> DarkParams:
    B, H, L, d = Q.shape
    dv = V.shape[-1] if V is not None else 1
    r = M.shape[-2] if M is not None else d      # M = None: the identity (isotropic features), r = d
    w_shared = W.dim() == 2
    m = W.shape[-2]
    torch = _torch()
    if (M is not None and M.dtype != torch.float32) or W.dtype != torch.float32:
        raise TypeError("M and W must be float32")
    if (M is not None and tuple(M.shape) != (H, r, d)) or W.shape[-1] != r or (not w_shared and W.shape[0] != H):
        raise ValueError("M must be [H, r, d] (or None) and W [H, m, r] or [m, r]")
    io = _dtype_code(Q)
    od = io if out_dtype is None else (DARK_BF16 if out_dtype == torch.bfloat16 else DARK_F32)
    return make_params(B, H, L, d, r, m, dv, io_dtype=io, out_dtype=od, chunk=chunk, scale=scale, w_shared=w_shared,
                       path=path, sched=sched)


def _result(V, dtype, Q):
    """An uninitialised contiguous tensor of V's shape on Q's device."""
    torch = _torch()
    if dtype == V.dtype and V.__class__ is torch.Tensor and V.get_device() == Q.get_device():
        return torch.empty_like(V, memory_format=torch.contiguous_format)   # a third of the host time of the other form
    return torch.empty(V.shape, dtype=dtype, device=Q.device)


def _check(status: int, where: str):
    if status != DARK_OK:
        raise DarkError(status, where)


def dark_featurize(X, M, W, is_query: bool, *, scale=0.0, path=PATH_AUTO):
    """phi_Sigma of every row of X [B,H,L,d] -> (phi [B,H,L,m], stab)."""
    torch = _torch()
    p, nb = _plan(OP_FEATURIZE, False, X, None, M, W, scale=scale, path=path)
    B, H, L, _ = X.shape
    phi = torch.empty((B, H, L, p.m), dtype=X.dtype, device=X.device)
    stab = torch.empty((B, H, L) if is_query else (B, H), dtype=torch.float32, device=X.device)
    ws, stream = _workspace(nb, X.device)
    _check(lib().dark_featurize(ctypes.byref(p), _ptr(X), _ptr(M), _ptr(W), int(is_query), _ptr(phi), _ptr(stab),
                                ws.data_ptr(), ws.numel(), stream), "dark_featurize")
    return phi, stab


def _attn(fn_name, op, Q, K, V, M, W, out, chunk, scale, path, out_dtype, sched=None):
    p, nb = _plan(op, False, Q, V, M, W, out_dtype, chunk, scale, path, sched)
    if K.shape != Q.shape or V.shape[:3] != Q.shape[:3] or K.dtype != Q.dtype or V.dtype != Q.dtype:
        raise ValueError("Q, K, V shapes/dtypes disagree")
    if out is None:
        out = _result(V, Q.dtype if out_dtype is None else out_dtype, Q)
    ws, stream = _workspace(nb, Q.device)
    fn = getattr(lib(), fn_name)
    _check(fn(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(M), _ptr(W), _ptr(out), ws.data_ptr(), ws.numel(),
              stream), fn_name)
    return out


def dark_attn_fwd(Q, K, V, M, W, *, out=None, scale=0.0, path=PATH_AUTO, out_dtype=None, sched=None):
    """Bidirectional random-feature attention, out [B,H,L,dv]."""
    return _attn("dark_attn_fwd", OP_ATTN_FWD, Q, K, V, M, W, out, 0, scale, path, out_dtype, sched)


def dark_attn_fwd_static(Q, K, V, M, W, out, *, scale=0.0, path=PATH_AUTO):
    """dark_attn_fwd on the library's static scratch: no workspace, no allocation (``out`` is the caller's)."""
    p, _ = _plan(None, False, Q, V, M, W, out.dtype, 0, scale, path)
    if K.shape != Q.shape or V.shape[:3] != Q.shape[:3] or K.dtype != Q.dtype or V.dtype != Q.dtype:
        raise ValueError("Q, K, V shapes/dtypes disagree")
    if tuple(out.shape) != tuple(V.shape):
        raise ValueError("out must have the shape of V")
    _check(lib().dark_attn_fwd_static(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(M), _ptr(W), _ptr(out),
                                      _stream()), "dark_attn_fwd_static")
    return out


def static_scratch_bytes() -> int:
    return int(lib().dark_static_scratch_bytes())


def dark_attn_causal_fwd(Q, K, V, M, W, *, out=None, chunk=0, scale=0.0, path=PATH_AUTO, out_dtype=None, sched=None):
    """Causal random-feature attention (keys l <= i), out [B,H,L,dv]."""
    return _attn("dark_attn_causal_fwd", OP_ATTN_CAUSAL_FWD, Q, K, V, M, W, out, chunk, scale, path, out_dtype, sched)


def decode_state(B, H, m, dv, device="cuda"):
    """Empty recurrent state (S, z, c) of dark_decode_step."""
    torch = _torch()
    return (torch.zeros((B, H, m, dv), dtype=torch.float32, device=device),
            torch.zeros((B, H, m), dtype=torch.float32, device=device),
            torch.full((B, H), float("-inf"), dtype=torch.float32, device=device))


def _decode_params(q, v, M, W, scale) -> DarkParams:
    scale = float(scale)
    key = ("decode", q.shape, q.dtype, v.shape, None if M is None else (M.shape, M.dtype), W.shape, W.dtype, scale)
    plan = _plans.get(key)
    if plan is None:
        _, _, _ = q.shape   # [B, H, d] and no other rank
        plan = (_params_from(q[:, :, None, :], v[:, :, None, :], M, W, scale=scale), 0)
        _keep_plan(key, plan)
    return plan[0]


def dark_decode_step(q, k, v, M, W, state, *, out=None, scale=0.0):
    """One token: q, k [B,H,d], v [B,H,dv]; state = (S, z, c) is updated in place; returns out [B,H,dv]."""
    S, z, c = state
    p = _decode_params(q, v, M, W, scale)
    if out is None:
        out = _result(v, q.dtype, q)
    _check(lib().dark_decode_step(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(M), _ptr(W), _ptr(S), _ptr(z), _ptr(c),
                                  _ptr(out), _stream()), "dark_decode_step")
    return out


def dark_whiten(Q, K=None, *, r=None, want_cov=False):
    """Whitening geometry M [H, r, d] (float32) from the rows of Q and K [B, H, L, d]; with want_cov also the
    covariance estimate [H, d, d]."""
    torch = _torch()
    B, H, L, d = Q.shape
    r = d if r is None else int(r)
    p = make_params(B, H, L, d, r, 64, 1, io_dtype=_dtype_code(Q))
    M = torch.empty((H, r, d), dtype=torch.float32, device=Q.device)
    cov = torch.empty((H, d, d), dtype=torch.float32, device=Q.device) if want_cov else None
    ws, stream = _workspace(workspace_bytes(p, OP_WHITEN), Q.device)
    _check(lib().dark_whiten(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(M), _ptr(cov), ws.data_ptr(), ws.numel(),
                             stream), "dark_whiten")
    return (M, cov) if want_cov else M


def saved_bytes(p: DarkParams) -> int:
    return int(lib().dark_saved_bytes(ctypes.byref(p)))


def dark_attn_causal_fwd_save(Q, K, V, M, W, *, out=None, saved=None, chunk=0, scale=0.0, path=PATH_AUTO, out_dtype=None):
    """Causal forward that leaves what the backward can take over in `saved` (a uint8 device tensor of at
    least saved_bytes(p) bytes; allocated here when not given).  Returns (out, saved); `saved` is None for
    parameters that have no hand-over."""
    torch = _torch()
    p, nb = _plan(OP_ATTN_CAUSAL_FWD, False, Q, V, M, W, out_dtype, chunk, scale, path)
    if out is None:
        out = torch.empty(V.shape, dtype=Q.dtype if out_dtype is None else out_dtype, device=Q.device)
    ns = saved_bytes(p)
    if ns and saved is None:
        saved = torch.empty(ns, dtype=torch.uint8, device=Q.device)
    ws, stream = _workspace(nb, Q.device)
    _check(lib().dark_attn_causal_fwd_save(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(M), _ptr(W), _ptr(out),
                                           _ptr(saved) if ns else None, saved.numel() if ns else 0,
                                           ws.data_ptr(), ws.numel(), stream), "dark_attn_causal_fwd_save")
    return out, (saved if ns else None)


def dark_attn_bwd(Q, K, V, M, W, dOut, causal: bool, *, chunk=0, scale=0.0, path=PATH_AUTO, need=("dQ", "dK", "dV", "dM"),
                  saved=None, grads=None):
    """Gradients of sum(out*dOut): returns dict with the float32 gradients named in `need`
    ("dQ", "dK", "dV", "dM", and "dW", the gradient with respect to the draws).  `saved`: the hand-over
    buffer of dark_attn_causal_fwd_save for the same inputs (causal only).  `grads`: a dict of preallocated
    output tensors to write into instead of allocating."""
    torch = _torch()
    p, nb = _plan(OP_ATTN_BWD, bool(causal), Q, V, M, W, None, chunk, scale, path)
    f32 = dict(dtype=torch.float32, device=Q.device)
    H, d = Q.shape[1], Q.shape[3]
    if grads is not None:
        g = {k: grads.get(k) for k in ("dQ", "dK", "dV", "dM", "dW")}
    else:
        g = {
            "dQ": torch.empty(Q.shape, **f32) if "dQ" in need else None,
            "dK": torch.empty(K.shape, **f32) if "dK" in need else None,
            "dV": torch.empty(V.shape, **f32) if "dV" in need else None,
            "dM": torch.empty(M.shape if M is not None else (H, d, d), **f32) if "dM" in need else None,
        }
        if "dW" in need:
            g["dW"] = torch.empty(W.shape, **f32)
    ws, stream = _workspace(nb, Q.device)
    if saved is not None:
        if not causal:
            raise ValueError("saved state exists for the causal form only")
        _check(lib().dark_attn_bwd_saved(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(M), _ptr(W), _ptr(dOut),
                                         _ptr(saved), saved.numel(), _ptr(g.get("dQ")), _ptr(g.get("dK")),
                                         _ptr(g.get("dV")), _ptr(g.get("dM")), _ptr(g.get("dW")), ws.data_ptr(),
                                         ws.numel(), stream), "dark_attn_bwd_saved")
        return g
    if g.get("dW") is not None:
        _check(lib().dark_attn_bwd_dw(ctypes.byref(p), int(causal), _ptr(Q), _ptr(K), _ptr(V), _ptr(M), _ptr(W),
                                      _ptr(dOut), _ptr(g["dQ"]), _ptr(g["dK"]), _ptr(g["dV"]), _ptr(g["dM"]),
                                      _ptr(g["dW"]), ws.data_ptr(), ws.numel(), stream), "dark_attn_bwd_dw")
        return g
    _check(lib().dark_attn_bwd(ctypes.byref(p), int(causal), _ptr(Q), _ptr(K), _ptr(V), _ptr(M), _ptr(W), _ptr(dOut),
                               _ptr(g["dQ"]), _ptr(g["dK"]), _ptr(g["dV"]), _ptr(g["dM"]), ws.data_ptr(), ws.numel(),
                               stream), "dark_attn_bwd")
    return g


# ----------------------------------------------------------------------------
# linear attention with a decay for each head
# ----------------------------------------------------------------------------
_LAYOUTS = {"bhld": BHLD, "blhd": BLHD}


def _pointers(*tensors):
    """(The device that all given tensors are on, their addresses; None: not given).  In one pass over them: this is a third of the
    host time of a short call."""
    index, out = None, []
    for t in tensors:
        if t is None:
            out.append(None)
            continue
        i = t.get_device()
        if i != index:
            if i < 0 or index is not None:
                raise ValueError("tensors must be on one GPU")
            index = i
        if not t.is_contiguous():
            raise ValueError("tensors must be contiguous device tensors")
        out.append(t.data_ptr())
    return index, out


def _require(t, dtype, shape, what):
    if t is not None and (t.dtype != dtype or t.shape != shape):
        raise ValueError(f"{what} must be {dtype} of shape {tuple(shape)}")


def _decay_plan(Q, K, V, layout, scale, segments, backward):
    """(DecayParams, workspace bytes) of a call."""
    key = ("decay", Q.shape, Q.dtype, K.shape, K.dtype, V.shape, V.dtype, layout, scale, segments, segments.__class__, backward)
    plan = _plans.get(key)
    if plan is None:
        if layout not in _LAYOUTS:
            raise ValueError(f"layout must be one of {sorted(_LAYOUTS)}")
        if Q.dim() != 4 or K.shape != Q.shape or V.dim() != 4 or V.shape[:3] != Q.shape[:3]:
            raise ValueError("Q, K and V must have the same batch, heads and length, Q and K the same width")
        if K.dtype != Q.dtype or V.dtype != Q.dtype:
            raise TypeError("Q, K and V must have one type")
        B, H, L, dk = Q.shape if layout == "bhld" else (Q.shape[0], Q.shape[2], Q.shape[1], Q.shape[3])
        p = DecayParams(B, H, L, dk, V.shape[3], _dtype_code(Q), _LAYOUTS[layout], scale, segments)
        plan = (p, int(lib().dark_decay_workspace_bytes(ctypes.byref(p), int(backward))))
        _keep_plan(key, plan)
    return plan


def dark_decay_fwd(Q, K, V, log_decay, *, lengths=None, state=None, out=None, state_out=None, want_state=False, scale=0.0,
                   layout="bhld", segments=0):
    """Linear attention with the decay exp(log_decay[h]) of each head, from `state` [B,H,dk,dv] (None: empty):
    S_t = g S_{t-1} + k_t v_t^T, out_t = scale S_t^T q_t.  Q, K [B,H,L,dk], V [B,H,L,dv] (layout "blhd": [B,L,H,..]).
    Returns out, or (out, state after the last token) with want_state or a `state_out` (which may be `state`).
    `lengths` [B] int32: rows of each sequence; out is 0 behind them.  `segments`: a schedule override (0: none)."""
    torch = _torch()
    p, nb = _decay_plan(Q, K, V, layout, float(scale), segments, False)
    f32, shape = torch.float32, (p.B, p.H, p.dk, p.dv)
    _require(log_decay, f32, (p.H,), "log_decay")
    _require(lengths, torch.int32, (p.B,), "lengths")
    _require(state, f32, shape, "state")
    _require(state_out, f32, shape, "state_out")
    _require(out, V.dtype, V.shape, "out")
    index, (q, k, v, a, n, s, o, so) = _pointers(Q, K, V, log_decay, lengths, state, out, state_out)
    if index != torch._C._cuda_getDevice():   # enqueued on the current stream of the tensors' device
        with torch.cuda.device(index):
            return dark_decay_fwd(Q, K, V, log_decay, lengths=lengths, state=state, out=out, state_out=state_out, want_state=want_state,
                                  scale=scale, layout=layout, segments=segments)
    if o is None:
        out = torch.empty_like(V)
        o = out.data_ptr()
    if want_state and so is None:
        state_out = torch.empty(shape, dtype=f32, device=Q.device) if state is None else torch.empty_like(state)
        so = state_out.data_ptr()
    ws, stream = _workspace(nb, Q.device) if nb else (None, torch._C._cuda_getCurrentRawStream(index))
    _check(lib().dark_decay_fwd(ctypes.byref(p), q, k, v, a, n, s, o, so, None if ws is None else ws.data_ptr(), nb, stream), "dark_decay_fwd")
    return out if state_out is None else (out, state_out)


def dark_decay_bwd(Q, K, V, log_decay, dOut, *, lengths=None, state=None, dstate=None, need=("dQ", "dK", "dV", "dstate"), grads=None,
                   scale=0.0, layout="bhld", segments=0):
    """Gradients of sum(out dOut) + sum(state_out dstate) of dark_decay_fwd: a dict of those named in `need` ("dstate", the gradient
    of the incoming state, only where `state` is given), in the types and layouts of what they belong to.
    `grads`: a dict of preallocated tensors to write into instead."""
    torch = _torch()
    p, nb = _decay_plan(Q, K, V, layout, float(scale), segments, True)
    f32, shape = torch.float32, (p.B, p.H, p.dk, p.dv)
    _require(log_decay, f32, (p.H,), "log_decay")
    _require(lengths, torch.int32, (p.B,), "lengths")
    _require(state, f32, shape, "state")
    _require(dstate, f32, shape, "dstate")
    _require(dOut, V.dtype, V.shape, "dOut")
    like = {"dQ": Q, "dK": K, "dV": V}
    unknown = set(need if grads is None else grads) - {"dQ", "dK", "dV", "dstate"}
    if unknown:
        raise ValueError(f"unknown gradient(s) {sorted(unknown)}")
    g = {} if grads is None else {name: t for name, t in grads.items() if t is not None}
    for name, t in g.items():
        _require(t, *((f32, shape) if name == "dstate" else (like[name].dtype, like[name].shape)), name)
    index, (q, k, v, a, do, n, s, ds, gq, gk, gv, gs) = _pointers(Q, K, V, log_decay, dOut, lengths, state, dstate, g.get("dQ"), g.get("dK"),
                                                                  g.get("dV"), g.get("dstate"))
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return dark_decay_bwd(Q, K, V, log_decay, dOut, lengths=lengths, state=state, dstate=dstate, need=need, grads=grads, scale=scale,
                                  layout=layout, segments=segments)
    if grads is None:
        g = {name: torch.empty_like(x) for name, x in like.items() if name in need}
        if "dstate" in need and state is not None:
            g["dstate"] = torch.empty_like(state)
        gq, gk, gv, gs = (g[name].data_ptr() if name in g else None for name in ("dQ", "dK", "dV", "dstate"))
    ws, stream = _workspace(nb, Q.device) if nb else (None, torch._C._cuda_getCurrentRawStream(index))
    _check(lib().dark_decay_bwd(ctypes.byref(p), q, k, v, a, n, s, do, ds, gq, gk, gv, gs, None if ws is None else ws.data_ptr(), nb, stream),
           "dark_decay_bwd")
    return g


def dark_decay_step(q, k, v, log_decay, state, *, parent=None, state_out=None, out=None, scale=0.0):
    """One token of dark_decay_fwd: q, k [B,H,dk], v [B,H,dv]; returns out [B,H,dv].  `state` [B,H,dk,dv] is updated in place,
    or left alone and the new one written to `state_out`.  With `parent` [B] int32 (and a `state_out`) row b continues row
    parent[b] of `state` [any number of rows,H,dk,dv]; a parent that is no row of it stands for an empty state."""
    torch = _torch()
    scale = float(scale)
    key = ("decay_step", q.shape, q.dtype, k.shape, k.dtype, v.shape, v.dtype, scale)
    plan = _plans.get(key)
    if plan is None:
        if q.dim() != 3 or k.shape != q.shape or v.dim() != 3 or v.shape[:2] != q.shape[:2]:
            raise ValueError("q and k must be [B, H, dk], v [B, H, dv]")
        if k.dtype != q.dtype or v.dtype != q.dtype:
            raise TypeError("q, k and v must have one type")
        p = DecayParams(q.shape[0], q.shape[1], 1, q.shape[2], v.shape[2], _dtype_code(q), BHLD, scale, 0)
        plan = (p, (p.B, p.H, p.dk, p.dv))
        _keep_plan(key, plan)
    p, shape = plan
    if state_out is None:
        if parent is not None:
            raise ValueError("a step that reads its states through `parent` needs a state_out")
        state_out = state
    f32, rows = torch.float32, state.shape[0]
    _require(log_decay, f32, shape[1:2], "log_decay")
    _require(parent, torch.int32, shape[:1], "parent")
    _require(state, f32, (rows,) + shape[1:], "state")
    _require(state_out, f32, shape, "state_out")
    _require(out, v.dtype, v.shape, "out")
    index, (pq, pk, pv, a, s, pp, so, o) = _pointers(q, k, v, log_decay, state, parent, state_out, out)
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return dark_decay_step(q, k, v, log_decay, state, parent=parent, state_out=state_out, out=out, scale=scale)
    if o is None:
        out = torch.empty_like(v)
        o = out.data_ptr()
    _check(lib().dark_decay_step(ctypes.byref(p), pq, pk, pv, a, pp, rows, s, so, o, torch._C._cuda_getCurrentRawStream(index)), "dark_decay_step")
    return out


# ----------------------------------------------------------------------------
# the gated delta rule
# ----------------------------------------------------------------------------
def _delta_plan(Q, K, V, layout, scale, backward):
    """(DeltaParams, workspace bytes, shape of the gates) of a call."""
    key = ("delta", Q.shape, Q.dtype, K.shape, K.dtype, V.shape, V.dtype, layout, scale, backward)
    plan = _plans.get(key)
    if plan is None:
        if layout not in _LAYOUTS:
            raise ValueError(f"layout must be one of {sorted(_LAYOUTS)}")
        if Q.dim() != 4 or K.shape != Q.shape or V.dim() != 4 or V.shape[:3] != Q.shape[:3]:
            raise ValueError("Q, K and V must have the same batch, heads and length, Q and K the same width")
        if K.dtype != Q.dtype or V.dtype != Q.dtype:
            raise TypeError("Q, K and V must have one type")
        B, H, L, dk = Q.shape if layout == "bhld" else (Q.shape[0], Q.shape[2], Q.shape[1], Q.shape[3])
        p = DeltaParams(B, H, L, dk, V.shape[3], _dtype_code(Q), _LAYOUTS[layout], scale)
        plan = (p, int(lib().dark_delta_workspace_bytes(ctypes.byref(p), int(backward))), Q.shape[:3])
        _keep_plan(key, plan)
    return plan


def dark_delta_fwd(Q, K, V, log_gate, beta, *, lengths=None, state=None, out=None, state_out=None, want_state=False, scale=0.0, layout="bhld"):
    """Linear attention by the gated delta rule, from `state` [B,H,dk,dv] (None: empty): with a = exp(log_gate_t),
    u_t = beta_t (v_t - a S_{t-1}^T k_t), S_t = a S_{t-1} + k_t u_t^T, out_t = scale S_t^T q_t.
    Q, K [B,H,L,dk], V [B,H,L,dv], log_gate (None: no decay) and beta [B,H,L] float32 (layout "blhd": [B,L,H,..] and [B,L,H]).
    Returns out, or (out, state after the last token) with want_state or a `state_out` (which may be `state`).
    `lengths` [B] int32: rows of each sequence; out is 0 behind them."""
    torch = _torch()
    p, nb, gates = _delta_plan(Q, K, V, layout, float(scale), False)
    f32, shape = torch.float32, (p.B, p.H, p.dk, p.dv)
    _require(log_gate, f32, gates, "log_gate")
    _require(beta, f32, gates, "beta")
    _require(lengths, torch.int32, (p.B,), "lengths")
    _require(state, f32, shape, "state")
    _require(state_out, f32, shape, "state_out")
    _require(out, V.dtype, V.shape, "out")
    index, (q, k, v, a, be, n, s, o, so) = _pointers(Q, K, V, log_gate, beta, lengths, state, out, state_out)
    if index != torch._C._cuda_getDevice():   # enqueued on the current stream of the tensors' device
        with torch.cuda.device(index):
            return dark_delta_fwd(Q, K, V, log_gate, beta, lengths=lengths, state=state, out=out, state_out=state_out, want_state=want_state,
                                  scale=scale, layout=layout)
    if o is None:
        out = torch.empty_like(V)
        o = out.data_ptr()
    if want_state and so is None:
        state_out = torch.empty(shape, dtype=f32, device=Q.device) if state is None else torch.empty_like(state)
        so = state_out.data_ptr()
    ws, stream = _workspace(nb, Q.device) if nb else (None, torch._C._cuda_getCurrentRawStream(index))
    _check(lib().dark_delta_fwd(ctypes.byref(p), q, k, v, a, be, n, s, o, so, None if ws is None else ws.data_ptr(), nb, stream), "dark_delta_fwd")
    return out if state_out is None else (out, state_out)


_DELTA_GRADS = ("dQ", "dK", "dV", "dlog_gate", "dbeta", "dstate")


def dark_delta_bwd(Q, K, V, log_gate, beta, dOut, *, lengths=None, state=None, dstate=None, need=_DELTA_GRADS, grads=None, scale=0.0,
                   layout="bhld"):
    """Gradients of sum(out dOut) + sum(state_out dstate) of dark_delta_fwd: a dict of those named in `need` ("dlog_gate" only where
    `log_gate` is given, "dstate", the gradient of the incoming state, only where `state` is), in the types and layouts of what they belong to.
    `grads`: a dict of preallocated tensors to write into instead.  The scratch, 120 KB and more for 64 rows of a head (dark.h), is kept for
    the stream's next calls."""
    torch = _torch()
    p, nb, gates = _delta_plan(Q, K, V, layout, float(scale), True)
    f32, shape = torch.float32, (p.B, p.H, p.dk, p.dv)
    _require(log_gate, f32, gates, "log_gate")
    _require(beta, f32, gates, "beta")
    _require(lengths, torch.int32, (p.B,), "lengths")
    _require(state, f32, shape, "state")
    _require(dstate, f32, shape, "dstate")
    _require(dOut, V.dtype, V.shape, "dOut")
    like = {"dQ": Q, "dK": K, "dV": V, "dbeta": beta}
    if log_gate is not None:
        like["dlog_gate"] = log_gate
    if state is not None:
        like["dstate"] = state
    unknown = set(need if grads is None else grads) - set(_DELTA_GRADS)
    if unknown:
        raise ValueError(f"unknown gradient(s) {sorted(unknown)}")
    g = {} if grads is None else {name: t for name, t in grads.items() if t is not None}
    for name, t in g.items():
        _require(t, *((f32, shape) if name == "dstate" else (f32, gates) if name in ("dlog_gate", "dbeta") else (like[name].dtype, like[name].shape)), name)
    index, (q, k, v, a, be, do, n, s, ds, *gp) = _pointers(Q, K, V, log_gate, beta, dOut, lengths, state, dstate, *(g.get(x) for x in _DELTA_GRADS))
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return dark_delta_bwd(Q, K, V, log_gate, beta, dOut, lengths=lengths, state=state, dstate=dstate, need=need, grads=grads, scale=scale,
                                  layout=layout)
    if grads is None:
        g = {name: torch.empty_like(x) for name, x in like.items() if name in need}
        gp = [g[name].data_ptr() if name in g else None for name in _DELTA_GRADS]
    ws, stream = _workspace(nb, Q.device) if nb else (None, torch._C._cuda_getCurrentRawStream(index))
    _check(lib().dark_delta_bwd(ctypes.byref(p), q, k, v, a, be, n, s, do, ds, *gp, None if ws is None else ws.data_ptr(), nb, stream),
           "dark_delta_bwd")
    return g


def dark_delta_step(q, k, v, log_gate, beta, state, *, parent=None, state_out=None, out=None, scale=0.0):
    """One token of dark_delta_fwd: q, k [B,H,dk], v [B,H,dv], log_gate (None: no decay) and beta [B,H] float32; returns out [B,H,dv].
    `state`, `state_out` and `parent` as in dark_decay_step."""
    torch = _torch()
    scale = float(scale)
    key = ("delta_step", q.shape, q.dtype, k.shape, k.dtype, v.shape, v.dtype, scale)
    plan = _plans.get(key)
    if plan is None:
        if q.dim() != 3 or k.shape != q.shape or v.dim() != 3 or v.shape[:2] != q.shape[:2]:
            raise ValueError("q and k must be [B, H, dk], v [B, H, dv]")
        if k.dtype != q.dtype or v.dtype != q.dtype:
            raise TypeError("q, k and v must have one type")
        p = DeltaParams(q.shape[0], q.shape[1], 1, q.shape[2], v.shape[2], _dtype_code(q), BHLD, scale)
        plan = (p, (p.B, p.H, p.dk, p.dv))
        _keep_plan(key, plan)
    p, shape = plan
    if state_out is None:
        if parent is not None:
            raise ValueError("a step that reads its states through `parent` needs a state_out")
        state_out = state
    f32, rows = torch.float32, state.shape[0]
    _require(log_gate, f32, shape[:2], "log_gate")
    _require(beta, f32, shape[:2], "beta")
    _require(parent, torch.int32, shape[:1], "parent")
    _require(state, f32, (rows,) + shape[1:], "state")
    _require(state_out, f32, shape, "state_out")
    _require(out, v.dtype, v.shape, "out")
    index, (pq, pk, pv, a, be, s, pp, so, o) = _pointers(q, k, v, log_gate, beta, state, parent, state_out, out)
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return dark_delta_step(q, k, v, log_gate, beta, state, parent=parent, state_out=state_out, out=out, scale=scale)
    if o is None:
        out = torch.empty_like(v)
        o = out.data_ptr()
    _check(lib().dark_delta_step(ctypes.byref(p), pq, pk, pv, a, be, pp, rows, s, so, o, torch._C._cuda_getCurrentRawStream(index)),
           "dark_delta_step")
    return out


# ----------------------------------------------------------------------------
# beam search over recurrent states, tokens drawn from logits
# ----------------------------------------------------------------------------
def dark_beam_select(logits, scores, *, finished=None, eos=0, keep_slots=False, out=None):
    """The next n beams of each batch entry from logits [B,n,V] and scores [B,n] (float32): (scores, parent, token), [B,n] each,
    parent and token int32.  Candidate (j, t) is worth scores[j] + log_softmax(logits[j])[t]; best first, equal ones by the lowest j, then
    the lowest t; with keep_slots a surviving beam's best successor has the beam's own place.  `finished` [B,n] (uint8 or bool): such a
    beam goes on with `eos` at its score.  `out`: the three tensors to write into."""
    torch = _torch()
    key = ("beam", logits.shape, logits.dtype, int(eos), bool(keep_slots))
    plan = _plans.get(key)
    if plan is None:
        B, n, V = logits.shape
        p = BeamParams(B, n, V, _dtype_code(logits), int(eos), int(bool(keep_slots)))
        plan = (p, int(lib().dark_beam_workspace_bytes(ctypes.byref(p))))
        _keep_plan(key, plan)
    p, nb = plan
    f32, i32, shape = torch.float32, torch.int32, (p.B, p.n)
    _require(scores, f32, shape, "scores")
    if finished is not None and (finished.dtype not in (torch.uint8, torch.bool) or finished.shape != shape):
        raise ValueError(f"finished must be uint8 or bool of shape {shape}")
    s, parent, token = (None, None, None) if out is None else out
    _require(s, f32, shape, "the scores of out")
    _require(parent, i32, shape, "the parents of out")
    _require(token, i32, shape, "the tokens of out")
    index, (x, c, f, ps, pp, pt) = _pointers(logits, scores, finished, s, parent, token)
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return dark_beam_select(logits, scores, finished=finished, eos=eos, keep_slots=keep_slots, out=out)
    if out is None:
        s, parent, token = torch.empty_like(scores), torch.empty_like(scores, dtype=i32), torch.empty_like(scores, dtype=i32)
        ps, pp, pt = s.data_ptr(), parent.data_ptr(), token.data_ptr()
    ws, stream = _workspace(nb, logits.device)
    _check(lib().dark_beam_select(ctypes.byref(p), x, c, f, ps, pp, pt, ws.data_ptr(), ws.numel(), stream), "dark_beam_select")
    return s, parent, token


def dark_sample(logits, uniform=None, *, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, want_logprob=False, out=None):
    """The next token of each row of logits [B,V], drawn by uniform [B] (float32, 0 ... 1): int32 [B]; with want_logprob also the logarithm of the
    probability with which it was drawn.  Of softmax(logits / temperature) are kept the top_k likeliest (0: all), of those the likeliest that
    hold top_p of their sum (1: all), of those the ones of min_p times the largest (0: all); the token is where the sum of the kept, in the order
    of their numbers, exceeds the share `uniform` of it.  temperature 0: the largest logit (`uniform` may then be None).  -1: a row without a token.
    The settings are numbers, or tensors [B] with one for each row (float32; top_k int32).  `out`: the token tensor to write into."""
    torch = _torch()
    f32, i32 = torch.float32, torch.int32
    settings = (temperature, top_k, top_p, min_p)
    tensor = [x if isinstance(x, torch.Tensor) and x.dim() > 0 else None for x in settings]
    t, k, p, q = (0 if y is not None else x for x, y in zip(settings, tensor))
    k = min(max(int(k), 0), 2 ** 31 - 1)   # the parameter block has 32 bits
    key = ("sample", logits.shape, logits.dtype, float(t), k, float(p), float(q))
    plan = _plans.get(key)
    if plan is None:
        B, V = logits.shape
        plan = (SampleParams(B, V, _dtype_code(logits), k, float(t), float(p), float(q)), 0)
        _keep_plan(key, plan)
    params, shape = plan[0], logits.shape[:1]
    _require(uniform, f32, shape, "uniform")
    for x, dtype, name in zip(tensor, (f32, i32, f32, f32), ("temperature", "top_k", "top_p", "min_p")):
        _require(x, dtype, shape, name)
    _require(out, i32, shape, "out")
    index, (x, u, *ptrs, o) = _pointers(logits, uniform, *tensor, out)
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return dark_sample(logits, uniform, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, want_logprob=want_logprob, out=out)
    if out is None:
        out = torch.empty(shape, dtype=i32, device=logits.device)
        o = out.data_ptr()
    log = torch.empty(shape, dtype=f32, device=logits.device) if want_logprob else None
    _check(lib().dark_sample(ctypes.byref(params), x, u, *ptrs, o, None if log is None else log.data_ptr(),
                             torch._C._cuda_getCurrentRawStream(index)), "dark_sample")
    return (out, log) if want_logprob else out


def dark_state_reorder(states, parent):
    """States of beams follow their parents, in place: row (b, j) of every tensor [B*n, ...] (or [B, n, ...]) becomes row
    (b, parent[b, j]) of before.  parent [B, n] int32; an entry outside 0 ... n - 1 leaves its row as it is.  The tensors may not overlap."""
    torch = _torch()
    if parent.dim() != 2:
        raise ValueError("parent must be [B, n]")
    B, n = parent.shape
    _require(parent, torch.int32, parent.shape, "parent")
    count = len(states)
    index, ptrs = _pointers(parent, *states)
    sizes = (ctypes.c_size_t * count)()
    for i, t in enumerate(states):
        if t.shape[:1] != (B * n,) and t.shape[:2] != (B, n):
            raise ValueError("a state must have a row for each beam")
        sizes[i] = t.numel() * t.element_size() // (B * n) if B * n else 0
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return dark_state_reorder(states, parent)
    _check(lib().dark_state_reorder(B, n, ptrs[0], count, (ctypes.c_void_p * count)(*ptrs[1:]), sizes,
                                    torch._C._cuda_getCurrentRawStream(index)), "dark_state_reorder")


# ----------------------------------------------------------------------------
# per-kernel timing (benchmarks)
# ----------------------------------------------------------------------------
def timing_enable(on: bool):
    lib().dark_timing_enable(int(on))


def timing_reset():
    lib().dark_timing_reset()


def timing_read() -> dict:
    """{kernel name: (launches, total_ms)} for kernels launched since the last reset."""
    L = lib()
    out = {}
    for k in range(L.dark_timing_slots()):
        name = ctypes.c_char_p()
        n = ctypes.c_int64()
        ms = ctypes.c_double()
        _check(L.dark_timing_read(k, ctypes.byref(name), ctypes.byref(n), ctypes.byref(ms)), "dark_timing_read")
        if n.value:
            out[name.value.decode()] = (n.value, ms.value)
    return out


def timeline_read(which: int, n: int):
    """The wall-clock stamps of the last launch of the key/value pass (which = 0) or the readout (which = 1)
    as a list of n int64 ticks; raises unless the loaded library was built with -DDARK_TIMELINE."""
    buf = (ctypes.c_int64 * n)()
    _check(lib().dark_timeline_read(int(which), buf, n), "dark_timeline_read")
    return list(buf)


# ----------------------------------------------------------------------------
# measured ceilings of the device (benchmarks)
# ----------------------------------------------------------------------------
def ceiling_copy(dst, src):
    """One launch of the plain copy kernel: src -> dst (same byte size, a multiple of 16)."""
    nb = src.numel() * src.element_size()
    _check(lib().dark_ceiling_copy(_ptr(dst), _ptr(src), nb, _stream()), "dark_ceiling_copy")
    return nb


def ceiling_read(src, sink):
    """One launch of the plain read kernel over src."""
    nb = src.numel() * src.element_size()
    _check(lib().dark_ceiling_read(_ptr(src), nb, _ptr(sink), _stream()), "dark_ceiling_read")
    return nb


def ceiling_mfma(iters, sink) -> float:
    """One launch of the MFMA loop kernel; returns the floating-point operations it performs."""
    fl = ctypes.c_double()
    _check(lib().dark_ceiling_mfma(int(iters), _ptr(sink), ctypes.byref(fl), _stream()), "dark_ceiling_mfma")
    return fl.value
