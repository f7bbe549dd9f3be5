"""Python binding of the CCQ C ABI (libccq.so): argument marshalling only.

Every entry point has the same name as its C function.  Tensors are torch
tensors on the GPU; the binding checks dtypes/shapes, allocates outputs and
the workspace with torch when the caller does not pass them, and hands raw
device pointers plus the current HIP stream to the library.  All arithmetic
runs in the library's HIP kernels.  There is no fallback: if libccq.so is
missing the first call raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import threading

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libccq.so")

CCQ_F32, CCQ_BF16 = 0, 1
CCQ_GLA, CCQ_GDN = 0, 1
CCQ_ACT_NONE, CCQ_ACT_SILU, CCQ_ACT_SIGMOID = 0, 1, 2
CCQ_NORM_GROUP, CCQ_NORM_RMS, CCQ_NORM_L2 = 0, 1, 2
_STATUS = {0: "CCQ_OK", 1: "CCQ_ERR_INVALID_ARG", 2: "CCQ_ERR_UNSUPPORTED",
           3: "CCQ_ERR_WORKSPACE", 4: "CCQ_ERR_HIP"}
EXPORTS = ("ccq_workspace_size", "ccq_gla_fwd", "ccq_gdn_fwd", "ccq_gdn_fwd_noalloc", "ccq_fwd_bwd",
           "ccq_varlen_workspace_size", "ccq_gla_fwd_varlen", "ccq_gdn_fwd_varlen",
           "ccq_fwd_bwd_varlen", "ccq_decode_workspace_size", "ccq_decode", "ccq_prep",
           "ccq_fwd_raw_workspace_size", "ccq_fwd_raw",
           "ccq_delta_workspace_size", "ccq_delta_fwd", "ccq_delta_fwd_varlen", "ccq_delta_fwd_bwd",
           "ccq_delta_fwd_bwd_varlen", "ccq_delta_step", "ccq_conv_workspace_size", "ccq_conv_fwd",
           "ccq_conv_fwd_varlen", "ccq_conv_bwd", "ccq_conv_bwd_varlen", "ccq_conv_step",
           "ccq_norm_workspace_size", "ccq_norm_fwd", "ccq_norm_bwd",
           "ccq_trace_events", "ccq_status_string", "ccq_version")


class CcqError(RuntimeError):
    def __init__(self, fn: str, code: int):
        super().__init__("%s returned %s (%d): %s" % (fn, _STATUS.get(code, "?"), code,
                                                      ccq_status_string(code)))
        self.code = code


class Shape(ctypes.Structure):
    """Mirror of ccq_shape (include/ccq.h)."""
    _fields_ = [("B", ctypes.c_int32), ("T", ctypes.c_int32), ("H", ctypes.c_int32),
                ("dk", ctypes.c_int32), ("dv", ctypes.c_int32), ("chunk", ctypes.c_int32),
                ("io_dtype", ctypes.c_int32), ("gate_dtype", ctypes.c_int32),
                ("scale", ctypes.c_float), ("centered", ctypes.c_int32),
                ("decay_aligned", ctypes.c_int32), ("t0", ctypes.c_int64)]


class DeltaShape(ctypes.Structure):
    """Mirror of ccq_delta_shape."""
    _fields_ = [("B", ctypes.c_int32), ("T", ctypes.c_int32), ("HK", ctypes.c_int32),
                ("HV", ctypes.c_int32), ("dk", ctypes.c_int32), ("dv", ctypes.c_int32),
                ("io_dtype", ctypes.c_int32), ("scale", ctypes.c_float)]


class ConvShape(ctypes.Structure):
    """Mirror of ccq_conv_shape."""
    _fields_ = [("B", ctypes.c_int32), ("T", ctypes.c_int32), ("C", ctypes.c_int32),
                ("W", ctypes.c_int32), ("io_dtype", ctypes.c_int32), ("act", ctypes.c_int32),
                ("ldx", ctypes.c_int64)]


class NormShape(ctypes.Structure):
    """Mirror of ccq_norm_shape."""
    _fields_ = [("rows", ctypes.c_int64), ("G", ctypes.c_int32), ("D", ctypes.c_int32),
                ("io_dtype", ctypes.c_int32), ("kind", ctypes.c_int32), ("act", ctypes.c_int32),
                ("shared", ctypes.c_int32), ("eps", ctypes.c_float), ("ldx", ctypes.c_int64),
                ("ldg", ctypes.c_int64)]


_lib = None
_lock = threading.Lock()


def lib() -> ctypes.CDLL:
    """Load libccq.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError("libccq.so is not built (%s); run "
                                   "`python -m paper_2606_01294_amd.build`" % LIB_PATH)
            L = ctypes.CDLL(LIB_PATH)
            P, S = ctypes.c_void_p, ctypes.c_size_t
            SP = ctypes.POINTER(Shape)
            L.ccq_workspace_size.argtypes = [SP, ctypes.c_int, ctypes.c_int]
            L.ccq_workspace_size.restype = S
            L.ccq_gla_fwd.argtypes = [SP] + [P] * 14 + [S, P]
            L.ccq_gla_fwd.restype = ctypes.c_int
            L.ccq_gdn_fwd.argtypes = [SP] + [P] * 15 + [S, P]
            L.ccq_gdn_fwd.restype = ctypes.c_int
            L.ccq_gdn_fwd_noalloc.argtypes = [SP] + [P] * 15
            L.ccq_gdn_fwd_noalloc.restype = ctypes.c_int
            L.ccq_fwd_bwd.argtypes = [SP, ctypes.c_int] + [P] * 15 + [S, P]
            L.ccq_fwd_bwd.restype = ctypes.c_int
            L.ccq_varlen_workspace_size.argtypes = [SP, ctypes.c_int, ctypes.c_int]
            L.ccq_varlen_workspace_size.restype = S
            L.ccq_gla_fwd_varlen.argtypes = [SP] + [P] * 14 + [S, P]
            L.ccq_gla_fwd_varlen.restype = ctypes.c_int
            L.ccq_gdn_fwd_varlen.argtypes = [SP] + [P] * 15 + [S, P]
            L.ccq_gdn_fwd_varlen.restype = ctypes.c_int
            L.ccq_fwd_bwd_varlen.argtypes = [SP, ctypes.c_int] + [P] * 16 + [S, P]
            L.ccq_fwd_bwd_varlen.restype = ctypes.c_int
            L.ccq_decode_workspace_size.argtypes = [SP]
            L.ccq_decode_workspace_size.restype = S
            L.ccq_decode.argtypes = [SP, ctypes.c_int] + [P] * 11 + [S, P]
            L.ccq_decode.restype = ctypes.c_int
            L.ccq_prep.argtypes = [SP] + [P] * 8
            L.ccq_prep.restype = ctypes.c_int
            L.ccq_fwd_raw_workspace_size.argtypes = [SP, ctypes.c_int]
            L.ccq_fwd_raw_workspace_size.restype = S
            L.ccq_fwd_raw.argtypes = [SP, ctypes.c_int] + [P] * 15 + [P, S, P]
            L.ccq_fwd_raw.restype = ctypes.c_int
            for name, cls, n in (("ccq_delta_fwd", DeltaShape, 8), ("ccq_delta_fwd_varlen", DeltaShape, 9),
                                 ("ccq_delta_fwd_bwd", DeltaShape, 14),
                                 ("ccq_delta_fwd_bwd_varlen", DeltaShape, 15),
                                 ("ccq_delta_step", DeltaShape, 7), ("ccq_conv_fwd", ConvShape, 6),
                                 ("ccq_conv_fwd_varlen", ConvShape, 7),
                                 ("ccq_conv_bwd", ConvShape, 10),
                                 ("ccq_conv_bwd_varlen", ConvShape, 11),
                                 ("ccq_conv_step", ConvShape, 5), ("ccq_norm_fwd", NormShape, 5),
                                 ("ccq_norm_bwd", NormShape, 9)):
                f = getattr(L, name)  # shape, tensors, [workspace, its size,] stream
                work = "delta_fwd" in name or name.endswith("bwd") or "bwd_" in name
                f.argtypes = [ctypes.POINTER(cls)] + [P] * n + ([P, S] if work else []) + [P]
                f.restype = ctypes.c_int
            L.ccq_delta_workspace_size.argtypes = [ctypes.POINTER(DeltaShape), ctypes.c_int]
            L.ccq_delta_workspace_size.restype = S
            L.ccq_conv_workspace_size.argtypes = [ctypes.POINTER(ConvShape)]
            L.ccq_conv_workspace_size.restype = S
            L.ccq_norm_workspace_size.argtypes = [ctypes.POINTER(NormShape)]
            L.ccq_norm_workspace_size.restype = S
            L.ccq_trace_events.argtypes = [P, ctypes.c_int]
            L.ccq_trace_events.restype = ctypes.c_int
            L.ccq_status_string.argtypes = [ctypes.c_int]
            L.ccq_status_string.restype = ctypes.c_char_p
            L.ccq_version.argtypes = []
            L.ccq_version.restype = ctypes.c_char_p
            _lib = L
    return _lib


def ccq_status_string(code: int) -> str:
    return lib().ccq_status_string(int(code)).decode()


def ccq_version() -> str:
    return lib().ccq_version().decode()


def ccq_trace_events(events) -> None:
    """Per-kernel timing hook: `events` is a list of torch.cuda.Event(enable_timing=True)
    (2 per kernel: before, after) or None to switch tracing off.  The caller keeps the
    list alive while tracing is on."""
    if not events:
        rc = lib().ccq_trace_events(None, 0)
    else:
        for e in events:
            e.record() if e.cuda_event == 0 else None  # make sure the event exists
        arr = (ctypes.c_void_p * len(events))(*[e.cuda_event for e in events])
        ccq_trace_events._keep = arr
        rc = lib().ccq_trace_events(ctypes.cast(arr, ctypes.c_void_p), len(events))
    if rc != 0:
        raise CcqError("ccq_trace_events", rc)


def _dt(t: torch.dtype) -> int:
    if t == torch.bfloat16:
        return CCQ_BF16
    if t == torch.float32:
        return CCQ_F32
    raise TypeError("unsupported dtype %s (float32 or bfloat16)" % t)


def make_shape(B, T, H, dk, dv, io_dtype, gate_dtype=None, scale=1.0, centered=True, t0=0,
               chunk=64, decay_aligned=False) -> Shape:
    gd = io_dtype if gate_dtype is None else gate_dtype
    return Shape(int(B), int(T), int(H), int(dk), int(dv), int(chunk), _dt(io_dtype), _dt(gd),
                 float(scale), int(bool(centered)), int(bool(decay_aligned)), int(t0))


def ccq_workspace_size(shape: Shape, backbone: int, with_bwd: bool = False) -> int:
    return int(lib().ccq_workspace_size(ctypes.byref(shape), int(backbone), int(bool(with_bwd))))


# The marshalling of a call is the larger part of a decode step of a small batch (its
# kernel takes 7 us), so it is kept short: pointers and sizes are passed as plain ints
# (the argument types convert them), the checks of _check run inline on the usual path.

def _p(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    return (torch.cuda.current_stream() if stream is None else stream).cuda_stream


# Calls on a stream that is not torch's current one (stream=s).  A call is ordered behind what s
# has been given, and behind nothing else: s must have waited for whoever wrote the inputs, and who
# reads the outputs elsewhere waits for s.  Memory follows that order too: what the binding
# allocates comes from s's own pool (_pool), since a block that the current stream has freed may
# still be written by its pending kernels, and every tensor of a call is marked as used where it is
# (_record), so that no memory is handed on while a kernel may still use it.
_SAME = contextlib.nullcontext()


def _pool(stream):
    """The context in which a call on `stream` allocates."""
    return _SAME if stream is None else torch.cuda.stream(stream)


def _record(stream, outs, *others):
    """Marks a call's tensors (tensors, dicts or lists of them, or None) as used on `stream`, and the
    outputs on the current stream as well, where the caller may drop them."""
    if stream is None:
        return
    here = None
    for i, o in enumerate((outs,) + others):
        for t in o.values() if isinstance(o, dict) else o if isinstance(o, (list, tuple)) else (o,):
            if isinstance(t, torch.Tensor) and t.is_cuda:
                if here is None:
                    here = torch.cuda.current_stream(t.device)
                    if stream == here:
                        return
                t.record_stream(stream)
                if i == 0:
                    t.record_stream(here)


def _check(t, name, shape, dtype, device):
    if t is None or (t.shape == shape and t.dtype == dtype and t.device == device and
                     t.is_contiguous()):
        return
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s: shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    if t.dtype != dtype:
        raise TypeError("%s: dtype %s, expected %s" % (name, t.dtype, dtype))
    if t.device != device:
        raise ValueError("%s: on %s, expected %s" % (name, t.device, device))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)


def _workspace(shape, backbone, with_bwd, workspace, device):
    need = ccq_workspace_size(shape, backbone, with_bwd)
    if workspace is None:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=device)
    return workspace, need


def _fwd(backbone, q, k, v, gate, lam, beta, S0, C0, mu0, scale, centered, t0, chunk,
         want_states, want_qclean, out, workspace, stream, decay_aligned=False):
    B, T, H, dk = q.shape
    dv = v.shape[-1]
    dev = q.device
    gate_dtype = gate.dtype if backbone == CCQ_GLA else q.dtype
    shape = make_shape(B, T, H, dk, dv, q.dtype, gate_dtype, scale, centered, t0, chunk,
                       decay_aligned)
    _check(q, "q", q.shape, q.dtype, dev)
    _check(k, "k", (B, T, H, dk), q.dtype, dev)
    _check(v, "v", (B, T, H, dv), q.dtype, dev)
    if backbone == CCQ_GLA:
        _check(gate, "g", (B, T, H, dk), gate.dtype, dev)
    else:
        _check(gate, "logalpha", (B, T, H), torch.float32, dev)
        _check(beta, "beta", (B, T, H), torch.float32, dev)
    _check(lam, "lam", (B, T, H), torch.float32, dev)
    _check(S0, "S0", (B, H, dv, dk), torch.float32, dev)
    _check(C0, "C0", (B, H, dk, dk), torch.float32, dev)
    _check(mu0, "mu0", (B, H, dk), torch.float32, dev)
    out = dict(out or {})
    with _pool(stream):
        if "o" not in out:
            out["o"] = torch.empty((B, T, H, dv), dtype=q.dtype, device=dev)
        if want_states:
            out.setdefault("ST", torch.empty((B, H, dv, dk), dtype=torch.float32, device=dev))
            out.setdefault("CT", torch.empty((B, H, dk, dk), dtype=torch.float32, device=dev))
            out.setdefault("muT", torch.empty((B, H, dk), dtype=torch.float32, device=dev))
        if want_qclean:
            out.setdefault("qclean", torch.empty((B, T, H, dk), dtype=torch.float32, device=dev))
        workspace, need = _workspace(shape, backbone, False, workspace, dev)
    st = _stream(stream)
    if backbone == CCQ_GLA:
        rc = lib().ccq_gla_fwd(ctypes.byref(shape), _p(q), _p(k), _p(v), _p(gate), _p(lam),
                               _p(S0), _p(C0), _p(mu0), _p(out["o"]), _p(out.get("ST")),
                               _p(out.get("CT")), _p(out.get("muT")), _p(out.get("qclean")),
                               _p(workspace), workspace.numel(), st)
        fn = "ccq_gla_fwd"
    else:
        rc = lib().ccq_gdn_fwd(ctypes.byref(shape), _p(q), _p(k), _p(v), _p(gate), _p(beta),
                               _p(lam), _p(S0), _p(C0), _p(mu0), _p(out["o"]),
                               _p(out.get("ST")), _p(out.get("CT")), _p(out.get("muT")),
                               _p(out.get("qclean")), _p(workspace), workspace.numel(), st)
        fn = "ccq_gdn_fwd"
    _record(stream, out, workspace, (q, k, v, gate, lam, beta, S0, C0, mu0))
    if rc != 0:
        raise CcqError(fn, rc)
    return out


def ccq_gla_fwd(q, k, v, g, lam, S0=None, C0=None, mu0=None, scale=1.0, centered=True, t0=0,
                chunk=64, want_states=True, want_qclean=False, out=None, workspace=None,
                stream=None):
    """CCQ-GLA chunkwise forward.  Returns dict o[, ST, CT, muT][, qclean]."""
    return _fwd(CCQ_GLA, q, k, v, g, lam, None, S0, C0, mu0, scale, centered, t0, chunk,
                want_states, want_qclean, out, workspace, stream)


def ccq_gdn_fwd(q, k, v, logalpha, beta, lam, S0=None, C0=None, mu0=None, scale=1.0,
                centered=True, t0=0, chunk=64, want_states=True, want_qclean=False, out=None,
                workspace=None, stream=None, decay_aligned=False):
    """CCQ-Gated-DeltaNet chunkwise forward.  Returns dict o[, ST, CT, muT][, qclean].
    decay_aligned=True: the decay-aligned statistics (ccq_shape.decay_aligned)."""
    return _fwd(CCQ_GDN, q, k, v, logalpha, lam, beta, S0, C0, mu0, scale, centered, t0, chunk,
                want_states, want_qclean, out, workspace, stream, decay_aligned)


# CCQ_NOALLOC_SCRATCH_BYTES of include/ccq.h
NOALLOC_SCRATCH_BYTES = 64 << 20


def ccq_gdn_fwd_noalloc(q, k, v, logalpha, beta, lam, S0=None, C0=None, mu0=None, scale=1.0,
                        centered=True, t0=0, chunk=64, want_states=True, want_qclean=False,
                        out=None, stream=None):
    """CCQ-Gated-DeltaNet forward without a workspace: the library's own per-device
    scratch (CCQ_NOALLOC_SCRATCH_BYTES) serves the kernels.  The binding allocates
    only the outputs it is not given; pass every output in `out` to allocate nothing.
    Returns dict o[, ST, CT, muT][, qclean]."""
    B, T, H, dk = q.shape
    dv = v.shape[-1]
    dev = q.device
    shape = make_shape(B, T, H, dk, dv, q.dtype, q.dtype, scale, centered, t0, chunk)
    _check(q, "q", q.shape, q.dtype, dev)
    _check(k, "k", (B, T, H, dk), q.dtype, dev)
    _check(v, "v", (B, T, H, dv), q.dtype, dev)
    _check(logalpha, "logalpha", (B, T, H), torch.float32, dev)
    _check(beta, "beta", (B, T, H), torch.float32, dev)
    _check(lam, "lam", (B, T, H), torch.float32, dev)
    _check(S0, "S0", (B, H, dv, dk), torch.float32, dev)
    _check(C0, "C0", (B, H, dk, dk), torch.float32, dev)
    _check(mu0, "mu0", (B, H, dk), torch.float32, dev)
    out = dict(out or {})
    with _pool(stream):
        if "o" not in out:
            out["o"] = torch.empty((B, T, H, dv), dtype=q.dtype, device=dev)
        if want_states:
            out.setdefault("ST", torch.empty((B, H, dv, dk), dtype=torch.float32, device=dev))
            out.setdefault("CT", torch.empty((B, H, dk, dk), dtype=torch.float32, device=dev))
            out.setdefault("muT", torch.empty((B, H, dk), dtype=torch.float32, device=dev))
        if want_qclean:
            out.setdefault("qclean", torch.empty((B, T, H, dk), dtype=torch.float32, device=dev))
    rc = lib().ccq_gdn_fwd_noalloc(ctypes.byref(shape), _p(q), _p(k), _p(v), _p(logalpha),
                                   _p(beta), _p(lam), _p(S0), _p(C0), _p(mu0), _p(out["o"]),
                                   _p(out.get("ST")), _p(out.get("CT")), _p(out.get("muT")),
                                   _p(out.get("qclean")), _stream(stream))
    _record(stream, out, (q, k, v, logalpha, beta, lam, S0, C0, mu0))
    if rc != 0:
        raise CcqError("ccq_gdn_fwd_noalloc", rc)
    return out


def ccq_fwd_bwd(q, k, v, g, lam, dO, scale=1.0, centered=True, chunk=64, out=None,
                workspace=None, stream=None, backbone=CCQ_GLA, beta=None):
    """CCQ training step: o and the gradients of sum <dO, o>.

    GLA: g is the log-forget gate [B,T,H,dk]; returns dict o, dq, dk, dv, dg, dlam.
    Gated DeltaNet (backbone=CCQ_GDN): g is log alpha [B,T,H] fp32 and beta
    [B,T,H] fp32 is required; returns o, dq, dk, dv, dg (= d log alpha), dbeta,
    dlam."""
    B, T, H, dk = q.shape
    dv = v.shape[-1]
    dev = q.device
    gate_dtype = g.dtype if backbone == CCQ_GLA else q.dtype
    shape = make_shape(B, T, H, dk, dv, q.dtype, gate_dtype, scale, centered, 0, chunk)
    if backbone == CCQ_GLA:
        _check(g, "g", (B, T, H, dk), g.dtype, dev)
    else:
        if beta is None:
            raise ValueError("beta is required for the Gated DeltaNet training step")
        _check(g, "logalpha", (B, T, H), torch.float32, dev)
        _check(beta, "beta", (B, T, H), torch.float32, dev)
    _check(q, "q", q.shape, q.dtype, dev)
    _check(k, "k", (B, T, H, dk), q.dtype, dev)
    _check(v, "v", (B, T, H, dv), q.dtype, dev)
    _check(dO, "dO", (B, T, H, dv), q.dtype, dev)
    _check(lam, "lam", (B, T, H), torch.float32, dev)
    out = dict(out or {})
    with _pool(stream):
        out.setdefault("o", torch.empty((B, T, H, dv), dtype=q.dtype, device=dev))
        out.setdefault("dq", torch.empty((B, T, H, dk), dtype=q.dtype, device=dev))
        out.setdefault("dk", torch.empty((B, T, H, dk), dtype=q.dtype, device=dev))
        out.setdefault("dv", torch.empty((B, T, H, dv), dtype=q.dtype, device=dev))
        out.setdefault("dg", torch.empty(tuple(g.shape), dtype=g.dtype, device=dev))
        out.setdefault("dlam", torch.empty((B, T, H), dtype=torch.float32, device=dev))
        if backbone == CCQ_GDN:
            out.setdefault("dbeta", torch.empty((B, T, H), dtype=torch.float32, device=dev))
        workspace, need = _workspace(shape, backbone, True, workspace, dev)
    rc = lib().ccq_fwd_bwd(ctypes.byref(shape), int(backbone), _p(q), _p(k), _p(v), _p(g),
                           _p(beta), _p(lam), _p(dO), _p(out["o"]), _p(out["dq"]),
                           _p(out["dk"]), _p(out["dv"]), _p(out["dg"]), _p(out.get("dbeta")),
                           _p(out["dlam"]), _p(workspace), workspace.numel(), _stream(stream))
    _record(stream, out, workspace, (q, k, v, g, beta, lam, dO))
    if rc != 0:
        raise CcqError("ccq_fwd_bwd", rc)
    return out


def ccq_varlen_workspace_size(shape: Shape, backbone: int, with_bwd: bool = False) -> int:
    return int(lib().ccq_varlen_workspace_size(ctypes.byref(shape), int(backbone),
                                               int(bool(with_bwd))))


def _varlen_shape(backbone, q, v, gate, cu_seqlens, max_len, scale, centered, t0,
                  decay_aligned=False):
    if cu_seqlens.dtype != torch.int32 or cu_seqlens.dim() != 1 or cu_seqlens.numel() < 1:
        raise TypeError("cu_seqlens must be a 1-D int32 tensor of B + 1 offsets")
    if cu_seqlens.device != q.device or not cu_seqlens.is_contiguous():
        raise ValueError("cu_seqlens must be contiguous on the device of q")
    rows, H, dk = q.shape
    B = cu_seqlens.numel() - 1
    gate_dtype = gate.dtype if backbone == CCQ_GLA else q.dtype
    return make_shape(B, max_len, H, dk, v.shape[-1], q.dtype, gate_dtype, scale, centered, t0,
                      decay_aligned=decay_aligned)


def _varlen_ws(shape, backbone, with_bwd, workspace, device):
    need = ccq_varlen_workspace_size(shape, backbone, with_bwd)
    if workspace is None:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=device)
    return workspace


def _varlen_fwd(backbone, q, k, v, gate, beta, lam, cu_seqlens, max_len, S0, C0, mu0, scale,
                centered, t0, want_states, out, workspace, stream, decay_aligned=False):
    rows, H, dk = q.shape
    dv = v.shape[-1]
    dev = q.device
    shape = _varlen_shape(backbone, q, v, gate, cu_seqlens, max_len, scale, centered, t0,
                          decay_aligned)
    B = shape.B
    _check(q, "q", q.shape, q.dtype, dev)
    _check(k, "k", (rows, H, dk), q.dtype, dev)
    _check(v, "v", (rows, H, dv), q.dtype, dev)
    if backbone == CCQ_GLA:
        _check(gate, "g", (rows, H, dk), gate.dtype, dev)
    else:
        if beta is None:
            raise ValueError("beta is required for Gated DeltaNet")
        _check(gate, "logalpha", (rows, H), torch.float32, dev)
        _check(beta, "beta", (rows, H), torch.float32, dev)
    _check(lam, "lam", (rows, H), torch.float32, dev)
    _check(S0, "S0", (B, H, dv, dk), torch.float32, dev)
    _check(C0, "C0", (B, H, dk, dk), torch.float32, dev)
    _check(mu0, "mu0", (B, H, dk), torch.float32, dev)
    out = dict(out or {})
    with _pool(stream):
        out.setdefault("o", torch.empty((rows, H, dv), dtype=q.dtype, device=dev))
        if want_states:
            out.setdefault("ST", torch.empty((B, H, dv, dk), dtype=torch.float32, device=dev))
            out.setdefault("CT", torch.empty((B, H, dk, dk), dtype=torch.float32, device=dev))
            out.setdefault("muT", torch.empty((B, H, dk), dtype=torch.float32, device=dev))
        workspace = _varlen_ws(shape, backbone, False, workspace, dev)
    st = _stream(stream)
    if backbone == CCQ_GLA:
        rc = lib().ccq_gla_fwd_varlen(ctypes.byref(shape), _p(cu_seqlens), _p(q), _p(k), _p(v),
                                      _p(gate), _p(lam), _p(S0), _p(C0), _p(mu0), _p(out["o"]),
                                      _p(out.get("ST")), _p(out.get("CT")), _p(out.get("muT")),
                                      _p(workspace), workspace.numel(), st)
        fn = "ccq_gla_fwd_varlen"
    else:
        rc = lib().ccq_gdn_fwd_varlen(ctypes.byref(shape), _p(cu_seqlens), _p(q), _p(k), _p(v),
                                      _p(gate), _p(beta), _p(lam), _p(S0), _p(C0), _p(mu0),
                                      _p(out["o"]), _p(out.get("ST")), _p(out.get("CT")),
                                      _p(out.get("muT")), _p(workspace), workspace.numel(), st)
        fn = "ccq_gdn_fwd_varlen"
    _record(stream, out, workspace, (cu_seqlens, q, k, v, gate, beta, lam, S0, C0, mu0))
    if rc != 0:
        raise CcqError(fn, rc)
    return out


def ccq_gla_fwd_varlen(q, k, v, g, lam, cu_seqlens, max_len, S0=None, C0=None, mu0=None,
                       scale=1.0, centered=True, t0=0, want_states=True, out=None,
                       workspace=None, stream=None):
    """CCQ-GLA forward on a packed batch: q, k, g [rows,H,dk], v [rows,H,dv], lam
    [rows,H]; sequence b is rows cu_seqlens[b]..cu_seqlens[b+1]-1 (int32 device
    tensor of B + 1 offsets), at most max_len rows long.  Returns dict o
    [rows,H,dv][, ST, CT, muT per sequence]."""
    return _varlen_fwd(CCQ_GLA, q, k, v, g, None, lam, cu_seqlens, max_len, S0, C0, mu0, scale,
                       centered, t0, want_states, out, workspace, stream)


def ccq_gdn_fwd_varlen(q, k, v, logalpha, beta, lam, cu_seqlens, max_len, S0=None, C0=None,
                       mu0=None, scale=1.0, centered=True, t0=0, want_states=True, out=None,
                       workspace=None, stream=None, decay_aligned=False):
    """CCQ-Gated-DeltaNet forward on a packed batch (layout as ccq_gla_fwd_varlen;
    logalpha, beta [rows,H] fp32).  decay_aligned as ccq_gdn_fwd."""
    return _varlen_fwd(CCQ_GDN, q, k, v, logalpha, beta, lam, cu_seqlens, max_len, S0, C0, mu0,
                       scale, centered, t0, want_states, out, workspace, stream, decay_aligned)


def _apart(stream, outs, *inputs):
    """The inputs, those that share memory with one of `outs` as copies (made on the stream
    of the call): the kernels read inputs after they have written outputs."""
    spans = [(o.data_ptr(), o.data_ptr() + o.numel() * o.element_size())
             for o in outs.values() if o is not None]

    def one(t):
        if t is None:
            return None
        a = t.data_ptr()
        b = a + t.numel() * t.element_size()
        if not any(a < end and begin < b for begin, end in spans):
            return t
        with torch.cuda.stream(stream):
            return t.clone()
    return [one(t) for t in inputs]


def ccq_fwd_bwd_varlen(q, k, v, g, lam, dO, cu_seqlens, max_len, scale=1.0, centered=True,
                       out=None, workspace=None, stream=None, backbone=CCQ_GLA, beta=None):
    """Training step on a packed batch (layout as ccq_gla_fwd_varlen; dO [rows,H,dv]).
    Returns the same dict as ccq_fwd_bwd, packed.  Tensors given in `out` may be inputs
    (out=dict(dq=q, ...): those inputs are copied first)."""
    rows, H, dk = q.shape
    dv = v.shape[-1]
    dev = q.device
    shape = _varlen_shape(backbone, q, v, g, cu_seqlens, max_len, scale, centered, 0)
    if backbone == CCQ_GLA:
        _check(g, "g", (rows, H, dk), g.dtype, dev)
    else:
        if beta is None:
            raise ValueError("beta is required for the Gated DeltaNet training step")
        _check(g, "logalpha", (rows, H), torch.float32, dev)
        _check(beta, "beta", (rows, H), torch.float32, dev)
    _check(q, "q", q.shape, q.dtype, dev)
    _check(k, "k", (rows, H, dk), q.dtype, dev)
    _check(v, "v", (rows, H, dv), q.dtype, dev)
    _check(dO, "dO", (rows, H, dv), q.dtype, dev)
    _check(lam, "lam", (rows, H), torch.float32, dev)
    if out:
        q, k, v, g, beta, lam, dO = _apart(stream, out, q, k, v, g, beta, lam, dO)
    out = dict(out or {})
    with _pool(stream):
        out.setdefault("o", torch.empty((rows, H, dv), dtype=q.dtype, device=dev))
        out.setdefault("dq", torch.empty((rows, H, dk), dtype=q.dtype, device=dev))
        out.setdefault("dk", torch.empty((rows, H, dk), dtype=q.dtype, device=dev))
        out.setdefault("dv", torch.empty((rows, H, dv), dtype=q.dtype, device=dev))
        out.setdefault("dg", torch.empty(tuple(g.shape), dtype=g.dtype, device=dev))
        out.setdefault("dlam", torch.empty((rows, H), dtype=torch.float32, device=dev))
        if backbone == CCQ_GDN:
            out.setdefault("dbeta", torch.empty((rows, H), dtype=torch.float32, device=dev))
        workspace = _varlen_ws(shape, backbone, True, workspace, dev)
    rc = lib().ccq_fwd_bwd_varlen(ctypes.byref(shape), int(backbone), _p(cu_seqlens), _p(q),
                                  _p(k), _p(v), _p(g), _p(beta), _p(lam), _p(dO), _p(out["o"]),
                                  _p(out["dq"]), _p(out["dk"]), _p(out["dv"]), _p(out["dg"]),
                                  _p(out.get("dbeta")), _p(out["dlam"]), _p(workspace),
                                  workspace.numel(), _stream(stream))
    _record(stream, out, workspace, (cu_seqlens, q, k, v, g, beta, lam, dO))
    if rc != 0:
        raise CcqError("ccq_fwd_bwd_varlen", rc)
    return out


def ccq_decode_workspace_size(shape: Shape) -> int:
    return int(lib().ccq_decode_workspace_size(ctypes.byref(shape)))


def ccq_decode(q, k, v, gate, lam, S, C, mu, t0, backbone=CCQ_GLA, beta=None, scale=1.0,
               centered=True, out=None, workspace=None, stream=None):
    """One recurrent CCQ step per sequence (Alg. 2) on the cache (S, C, mu), which is
    updated in place.  q, k [B,H,dk] and v [B,H,dv] (one token); GLA gate [B,H,dk],
    Gated DeltaNet log alpha [B,H] fp32 plus beta [B,H] fp32; lam [B,H] fp32;
    S [B,H,dv,dk], C [B,H,dk,dk], mu [B,H,dk] fp32; t0 = tokens already absorbed.
    Returns o [B,H,dv]."""
    B, H, dk = q.shape
    dv = v.shape[-1]
    dev, dt, f32 = q.device, q.dtype, torch.float32
    io = _dt(dt)
    gla = backbone == CCQ_GLA
    if not gla and beta is None:
        raise ValueError("beta is required for Gated DeltaNet")
    if S is None or C is None or mu is None:
        raise ValueError("%s (the cache) is required" % ("S" if S is None else "C" if C is None else "mu"))
    key, val, tok = (B, H, dk), (B, H, dv), (B, H)
    if gla:
        args = ((gate, "g", key, gate.dtype),)
    else:
        args = ((gate, "logalpha", tok, f32), (beta, "beta", tok, f32))
    for t, name, shp, d in ((q, "q", key, dt), (k, "k", key, dt), (v, "v", val, dt),
                            (lam, "lam", tok, f32)) + args + (
            (S, "S", (B, H, dv, dk), f32), (C, "C", (B, H, dk, dk), f32), (mu, "mu", key, f32)):
        if t is None or t.shape != shp or t.dtype != d or t.device != dev or not t.is_contiguous():
            _check(t, name, shp, d, dev)
    if out is None and stream is None:
        o = torch.empty(val, dtype=dt, device=dev)
    elif out is None:
        with _pool(stream):
            o = torch.empty(val, dtype=dt, device=dev)
    else:
        o = out
        _check(o, "o", val, dt, dev)
    shape = Shape(B, 1, H, dk, dv, 64, io, _dt(gate.dtype) if gla else io, float(scale),
                  1 if centered else 0, 0, int(t0))
    if workspace is None:
        need = ccq_decode_workspace_size(shape)
        if need:
            with _pool(stream):
                workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    rc = lib().ccq_decode(shape, int(backbone), q.data_ptr(), _p(k), v.data_ptr(), _p(gate),
                          _p(beta), _p(lam), S.data_ptr(), C.data_ptr(), mu.data_ptr(),
                          o.data_ptr(), _p(workspace),
                          0 if workspace is None else workspace.numel(), _stream(stream))
    if stream is not None:
        _record(stream, o, workspace, (q, k, v, gate, beta, lam, S, C, mu))
    if rc != 0:
        raise CcqError("ccq_decode", rc)
    return o


def ccq_prep(q_raw, k_raw, w_lam, b_lam, out=None, stream=None):
    """Per-head l2 normalisation of raw q, k [B,T,H,dk] and the gate
    lam = sigmoid(w_lam qraw + b_lam) [B,T,H] from the token's query before the head
    split (w_lam [H, H*dk] fp32, b_lam [H] fp32).  Returns dict q, k, lam; pass
    out=dict(q=q_raw, k=k_raw) to normalise in place."""
    B, T, H, dk = q_raw.shape
    dev = q_raw.device
    _check(q_raw, "q_raw", q_raw.shape, q_raw.dtype, dev)
    _check(k_raw, "k_raw", (B, T, H, dk), q_raw.dtype, dev)
    _check(w_lam, "w_lam", (H, H * dk), torch.float32, dev)
    _check(b_lam, "b_lam", (H,), torch.float32, dev)
    out = dict(out or {})
    with _pool(stream):
        out.setdefault("q", torch.empty_like(q_raw))
        out.setdefault("k", torch.empty_like(k_raw))
        out.setdefault("lam", torch.empty((B, T, H), dtype=torch.float32, device=dev))
    shape = make_shape(B, T, H, dk, dk, q_raw.dtype)
    rc = lib().ccq_prep(ctypes.byref(shape), _p(q_raw), _p(k_raw), _p(w_lam), _p(b_lam),
                        _p(out["q"]), _p(out["k"]), _p(out["lam"]), _stream(stream))
    _record(stream, out, (q_raw, k_raw, w_lam, b_lam))
    if rc != 0:
        raise CcqError("ccq_prep", rc)
    return out


def ccq_fwd_raw_workspace_size(shape: Shape, backbone: int) -> int:
    return int(lib().ccq_fwd_raw_workspace_size(ctypes.byref(shape), int(backbone)))


def ccq_fwd_raw(q_raw, k_raw, w_lam, b_lam, v, gate, beta=None, backbone=CCQ_GLA, S0=None, C0=None,
                mu0=None, scale=1.0, centered=True, t0=0, chunk=64, want_states=True,
                want_lam=False, out=None, workspace=None, stream=None):
    """Forward from raw q, k [B,T,H,dk]: the l2 normalisation and the gate
    lam = sigmoid(w_lam qraw + b_lam) (w_lam [H, H*dk], b_lam [H] fp32) folded into the
    forward.  gate: the GLA log-forget gate [B,T,H,dk], or Gated DeltaNet log alpha
    [B,T,H] fp32 with beta [B,T,H] fp32.  Returns dict o[, ST, CT, muT][, lam]."""
    B, T, H, dk = q_raw.shape
    dv = v.shape[-1]
    dev = q_raw.device
    gate_dtype = gate.dtype if backbone == CCQ_GLA else q_raw.dtype
    shape = make_shape(B, T, H, dk, dv, q_raw.dtype, gate_dtype, scale, centered, t0, chunk)
    _check(q_raw, "q_raw", q_raw.shape, q_raw.dtype, dev)
    _check(k_raw, "k_raw", (B, T, H, dk), q_raw.dtype, dev)
    _check(v, "v", (B, T, H, dv), q_raw.dtype, dev)
    _check(w_lam, "w_lam", (H, H * dk), torch.float32, dev)
    _check(b_lam, "b_lam", (H,), torch.float32, dev)
    if backbone == CCQ_GLA:
        _check(gate, "g", (B, T, H, dk), gate.dtype, dev)
    else:
        if beta is None:
            raise ValueError("beta is required for Gated DeltaNet")
        _check(gate, "logalpha", (B, T, H), torch.float32, dev)
        _check(beta, "beta", (B, T, H), torch.float32, dev)
    _check(S0, "S0", (B, H, dv, dk), torch.float32, dev)
    _check(C0, "C0", (B, H, dk, dk), torch.float32, dev)
    _check(mu0, "mu0", (B, H, dk), torch.float32, dev)
    out = dict(out or {})
    with _pool(stream):
        out.setdefault("o", torch.empty((B, T, H, dv), dtype=q_raw.dtype, device=dev))
        if want_states:
            out.setdefault("ST", torch.empty((B, H, dv, dk), dtype=torch.float32, device=dev))
            out.setdefault("CT", torch.empty((B, H, dk, dk), dtype=torch.float32, device=dev))
            out.setdefault("muT", torch.empty((B, H, dk), dtype=torch.float32, device=dev))
        if want_lam:
            out.setdefault("lam", torch.empty((B, T, H), dtype=torch.float32, device=dev))
        need = ccq_fwd_raw_workspace_size(shape, backbone)
        if workspace is None:
            workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
    rc = lib().ccq_fwd_raw(ctypes.byref(shape), int(backbone), _p(q_raw), _p(k_raw), _p(w_lam),
                           _p(b_lam), _p(v), _p(gate), _p(beta), _p(S0), _p(C0), _p(mu0),
                           _p(out["o"]), _p(out.get("ST")), _p(out.get("CT")), _p(out.get("muT")),
                           _p(out.get("lam")), _p(workspace), workspace.numel(), _stream(stream))
    _record(stream, out, workspace, (q_raw, k_raw, w_lam, b_lam, v, gate, beta, S0, C0, mu0))
    if rc != 0:
        raise CcqError("ccq_fwd_raw", rc)
    return out


# ---- The operators around the contraction: the plain gated delta rule, the short
# convolution and the head norm.  Tensors given in `out` are checked like inputs and may
# share no memory with the inputs or each other; a call is made on the tensors' own device.

def _on_gpu(t, name):
    if not t.is_cuda:
        raise ValueError("%s: on %s, expected a GPU tensor" % (name, t.device))


def _outputs(out, want, dev, inputs):
    """The outputs named in `want` (name -> (shape, dtype), or a dense tensor like it), from `out`
    where given."""
    if not out:  # (torch makes a tensor like another in 0.8 us, one of a named shape in 1.4)
        return {n: torch.empty_like(w) if isinstance(w, torch.Tensor) else
                torch.empty(w[0], dtype=w[1], device=dev) for n, w in want.items()}
    extra = set(out) - set(want)
    if extra:
        raise ValueError("out: no output named %s here" % ", ".join(sorted(extra)))
    spans = [_span(t) for t in inputs if t is not None]
    res = {}
    for n, w in want.items():
        shp, dt = (w.shape, w.dtype) if isinstance(w, torch.Tensor) else w
        t = out.get(n)
        if t is None:
            t = torch.empty(shp, dtype=dt, device=dev)
        else:
            _check(t, n, shp, dt, dev)
            a, b = _span(t)
            if any(a < e and s < b for s, e in spans):
                raise ValueError("%s: shares memory with an input or another output" % n)
            spans.append((a, b))
        res[n] = t
    return res


def _span(t):
    """First and one past the last byte that a (possibly strided) tensor covers."""
    if t.numel() == 0:
        return 0, 0
    last = sum((n - 1) * s for n, s in zip(t.shape, t.stride()))
    return t.data_ptr(), t.data_ptr() + (last + 1) * t.element_size()


def _pitch(t, inner, name):
    """Row pitch of a tensor whose last `inner` dims are dense and whose leading dims step
    evenly: a dense tensor, or a slice of a wider one."""
    size = 1
    for n in t.shape[t.dim() - inner:]:
        size *= n
    if t.is_contiguous():
        return size
    want = 1
    for n, s in zip(reversed(t.shape[t.dim() - inner:]), reversed(t.stride()[t.dim() - inner:])):
        if n != 1 and s != want:
            raise ValueError("%s: the channels must be contiguous" % name)
        want *= n
    ld, rows = None, 1
    for n, s in zip(reversed(t.shape[:t.dim() - inner]), reversed(t.stride()[:t.dim() - inner])):
        if n == 1:
            continue
        if ld is None:
            ld = s
        elif s != ld * rows:
            raise ValueError("%s: its tokens must be evenly spaced" % name)
        rows *= n
    if ld is None:
        return size
    if ld < size:
        raise ValueError("%s: its tokens overlap" % name)
    return ld


# The handle of a device's current stream: torch's own accessor of the raw handle where it has
# one (a step of a small batch takes 3 us on the GPU; the Stream object alone takes 3 us to make).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _launch(name, dev, stream, shape, args, ws=None):
    """Calls the library's function `name` with the tensors' device current."""
    if stream is None:
        handle = _raw_stream(dev.index)
    else:
        if stream.device != dev:
            raise ValueError("stream: on %s, the tensors on %s" % (stream.device, dev))
        handle = stream.cuda_stream
    ptrs = [None if t is None else t.data_ptr() for t in args]
    if ws is not None:
        ptrs += [ws.data_ptr(), ws.numel()] if isinstance(ws, torch.Tensor) else [None, 0]
    fn = getattr(_lib or lib(), name)
    if torch.cuda.current_device() == dev.index:
        rc = fn(shape, *ptrs, handle)
    else:
        with torch.cuda.device(dev):
            rc = fn(shape, *ptrs, handle)
    if rc != 0:
        raise CcqError(name, rc)


def _scratch(workspace, need, dev):
    """The caller's workspace or a new one; () where none is needed."""
    if workspace is None:
        return torch.empty(need, dtype=torch.uint8, device=dev) if need else ()
    if workspace.device != dev or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace: a contiguous uint8 tensor on %s is expected" % dev)
    return workspace


def _check_offsets(cu_seqlens, dev):
    if cu_seqlens.dtype != torch.int32 or cu_seqlens.dim() != 1 or cu_seqlens.numel() < 1:
        raise TypeError("cu_seqlens must be a 1-D int32 tensor of B + 1 offsets")
    if cu_seqlens.device != dev or not cu_seqlens.is_contiguous():
        raise ValueError("cu_seqlens must be contiguous on the tensors' device")


def make_delta_shape(B, T, HK, HV, dk, dv, io_dtype, scale=1.0) -> DeltaShape:
    return DeltaShape(int(B), int(T), int(HK), int(HV), int(dk), int(dv), _dt(io_dtype),
                      float(scale))


def ccq_delta_workspace_size(shape: DeltaShape, with_bwd: bool = False) -> int:
    return int(lib().ccq_delta_workspace_size(ctypes.byref(shape), int(bool(with_bwd))))


def _delta_shape(q, k, v, logalpha, beta, cu_seqlens, max_len, scale):
    """Checks the inputs of the chunked forms; returns the shape and the token dims."""
    dims = 4 if cu_seqlens is None else 3
    _on_gpu(q, "q")
    if q.dim() != dims or v.dim() != dims:
        raise ValueError("q and v: %d dims expected" % dims)
    dev, dt = q.device, q.dtype
    HK, dk = q.shape[-2:]
    HV, dv = v.shape[-2:]
    tok = tuple(q.shape[:-2])
    if cu_seqlens is None:
        B, T = tok
    else:
        _check_offsets(cu_seqlens, dev)
        B, T = cu_seqlens.numel() - 1, max_len
    shape = make_delta_shape(B, T, HK, HV, dk, dv, dt, scale)
    _check(q, "q", q.shape, dt, dev)
    _check(k, "k", q.shape, dt, dev)
    _check(v, "v", tok + (HV, dv), dt, dev)
    _check(logalpha, "logalpha", tok + (HV,), torch.float32, dev)
    _check(beta, "beta", tok + (HV,), torch.float32, dev)
    return shape, tok


def _delta_fwd(q, k, v, logalpha, beta, cu_seqlens, max_len, S0, scale, want_states, out,
               workspace, stream):
    shape, tok = _delta_shape(q, k, v, logalpha, beta, cu_seqlens, max_len, scale)
    dev = q.device
    state = (shape.B, shape.HV, shape.dv, shape.dk)
    _check(S0, "S0", state, torch.float32, dev)
    want = {"o": v}
    if want_states:
        want["ST"] = (state, torch.float32)
    with _pool(stream):
        res = _outputs(out, want, dev, (q, k, v, logalpha, beta, S0))
        ws = _scratch(workspace, ccq_delta_workspace_size(shape), dev)
    args = [q, k, v, logalpha, beta, S0, res["o"], res.get("ST")]
    if cu_seqlens is None:
        _launch("ccq_delta_fwd", dev, stream, shape, args, ws)
    else:
        _launch("ccq_delta_fwd_varlen", dev, stream, shape, [cu_seqlens] + args, ws)
    _record(stream, res, ws, args, cu_seqlens)
    return res


def ccq_delta_fwd(q, k, v, logalpha, beta, S0=None, scale=1.0, want_states=True, out=None,
                  workspace=None, stream=None):
    """The gated delta rule without the contraction: q, k [B,T,HK,dk], v [B,T,HV,dv] (value
    head h reads q and k of head h // (HV // HK)), logalpha, beta [B,T,HV] fp32, S0
    [B,HV,dv,dk] fp32.  Returns dict o [B,T,HV,dv][, ST]."""
    return _delta_fwd(q, k, v, logalpha, beta, None, None, S0, scale, want_states, out, workspace,
                      stream)


def ccq_delta_fwd_varlen(q, k, v, logalpha, beta, cu_seqlens, max_len, S0=None, scale=1.0,
                         want_states=True, out=None, workspace=None, stream=None):
    """ccq_delta_fwd on a packed batch: q, k [rows,HK,dk], v [rows,HV,dv], logalpha, beta
    [rows,HV]; sequence b is rows cu_seqlens[b]..cu_seqlens[b+1]-1, at most max_len long."""
    return _delta_fwd(q, k, v, logalpha, beta, cu_seqlens, max_len, S0, scale, want_states, out,
                      workspace, stream)


def _delta_fwd_bwd(q, k, v, logalpha, beta, dO, cu_seqlens, max_len, S0, scale, want_o,
                   want_states, out, workspace, stream):
    shape, tok = _delta_shape(q, k, v, logalpha, beta, cu_seqlens, max_len, scale)
    dev, dt = q.device, q.dtype
    state = (shape.B, shape.HV, shape.dv, shape.dk)
    _check(S0, "S0", state, torch.float32, dev)
    _check(dO, "dO", v.shape, dt, dev)
    gates = tok + (shape.HV,)
    want = {"dq": q, "dk": q, "dv": v, "dlogalpha": (gates, dt), "dbeta": (gates, dt)}
    if want_o:
        want["o"] = v
    if want_states:
        want["ST"] = (state, torch.float32)
    with _pool(stream):
        res = _outputs(out, want, dev, (q, k, v, logalpha, beta, S0, dO))
        ws = _scratch(workspace, ccq_delta_workspace_size(shape, True), dev)
    args = [q, k, v, logalpha, beta, S0, dO, res.get("o"), res.get("ST"), res["dq"], res["dk"],
            res["dv"], res["dlogalpha"], res["dbeta"]]
    if cu_seqlens is None:
        _launch("ccq_delta_fwd_bwd", dev, stream, shape, args, ws)
    else:
        _launch("ccq_delta_fwd_bwd_varlen", dev, stream, shape, [cu_seqlens] + args, ws)
    _record(stream, res, ws, args, cu_seqlens)
    return res


def ccq_delta_fwd_bwd(q, k, v, logalpha, beta, dO, S0=None, scale=1.0, want_o=True,
                      want_states=False, out=None, workspace=None, stream=None):
    """Training step of ccq_delta_fwd: the gradients of sum <dO, o>, in q's dtype.  Returns dict
    dq, dk (summed over the value heads that share them), dv, dlogalpha, dbeta[, o][, ST];
    want_o=False where the forward has been run already.  No gradient flows to S0."""
    return _delta_fwd_bwd(q, k, v, logalpha, beta, dO, None, None, S0, scale, want_o, want_states,
                          out, workspace, stream)


def ccq_delta_fwd_bwd_varlen(q, k, v, logalpha, beta, dO, cu_seqlens, max_len, S0=None, scale=1.0,
                             want_o=True, want_states=False, out=None, workspace=None,
                             stream=None):
    """ccq_delta_fwd_bwd on a packed batch (layout as ccq_delta_fwd_varlen)."""
    return _delta_fwd_bwd(q, k, v, logalpha, beta, dO, cu_seqlens, max_len, S0, scale, want_o,
                          want_states, out, workspace, stream)


def ccq_delta_step(q, k, v, logalpha, beta, S, scale=1.0, out=None, stream=None):
    """The recurrent form for one or a few tokens: q, k [B,T,HK,dk], v [B,T,HV,dv], logalpha,
    beta [B,T,HV] fp32; the state S [B,HV,dv,dk] fp32 is updated in place.  Returns o."""
    _on_gpu(q, "q")
    if q.dim() != 4 or v.dim() != 4:
        raise ValueError("q and v: 4 dims expected")
    if S is None:
        raise ValueError("S (the state) is required")
    B, T, HK, dk = q.shape
    HV, dv = v.shape[2:]
    dev, dt, f32 = q.device, q.dtype, torch.float32
    for t, name, shp, d in ((q, "q", q.shape, dt), (k, "k", q.shape, dt),
                            (v, "v", (B, T, HV, dv), dt), (logalpha, "logalpha", (B, T, HV), f32),
                            (beta, "beta", (B, T, HV), f32), (S, "S", (B, HV, dv, dk), f32)):
        _check(t, name, shp, d, dev)
    if out is None and stream is None:
        o = torch.empty_like(v)
    else:
        with _pool(stream):
            o = _outputs({"o": out}, {"o": v}, dev, (q, k, v, logalpha, beta, S))["o"]
    shape = DeltaShape(B, T, HK, HV, dk, dv, _dt(dt), scale)
    _launch("ccq_delta_step", dev, stream, shape, (q, k, v, logalpha, beta, S, o))
    if stream is not None:
        _record(stream, o, (q, k, v, logalpha, beta, S))
    return o


def _conv_shape(x, w, bias, state0, cu_seqlens, max_len, act):
    dims = 3 if cu_seqlens is None else 2
    _on_gpu(x, "x")
    if x.dim() != dims or w.dim() != 2:
        raise ValueError("x: %d dims, w: 2 dims expected" % dims)
    dev, dt = x.device, x.dtype
    C, W = w.shape
    if x.shape[-1] != C:
        raise ValueError("x: %d channels, w has %d" % (x.shape[-1], C))
    if cu_seqlens is None:
        B, T = x.shape[:2]
    else:
        _check_offsets(cu_seqlens, dev)
        B, T = cu_seqlens.numel() - 1, max_len
    _check(w, "w", (C, W), torch.float32, dev)
    _check(bias, "bias", (C,), torch.float32, dev)
    _check(state0, "state0", (B, W - 1, C), dt, dev)
    return ConvShape(B, int(T), C, W, _dt(dt), int(act), _pitch(x, 1, "x"))


def _conv_fwd(x, w, cu_seqlens, max_len, bias, state0, act, want_state, out, stream):
    shape = _conv_shape(x, w, bias, state0, cu_seqlens, max_len, act)
    dev = x.device
    want = {"y": x if x.is_contiguous() else (tuple(x.shape), x.dtype)}
    if want_state:
        want["stateT"] = ((shape.B, shape.W - 1, shape.C), x.dtype)
    with _pool(stream):
        res = _outputs(out, want, dev, (x, w, bias, state0))
    args = [x, w, bias, state0, res["y"], res.get("stateT")]
    if cu_seqlens is None:
        _launch("ccq_conv_fwd", dev, stream, shape, args)
    else:
        _launch("ccq_conv_fwd_varlen", dev, stream, shape, [cu_seqlens] + args)
    _record(stream, res, args, cu_seqlens)
    return res


def ccq_conv_fwd(x, w, bias=None, state0=None, act=CCQ_ACT_SILU, want_state=False, out=None,
                 stream=None):
    """Short causal convolution of every channel, y = act(bias + sum_j w[:, j] x_{t-W+1+j}):
    x [B,T,C] (dense, or a slice of a wider tensor), w [C,W] fp32 (W = 2, 3, 4), bias [C] fp32,
    state0 [B,W-1,C] the inputs before the first token, oldest first.  Returns dict y[, stateT]."""
    return _conv_fwd(x, w, None, None, bias, state0, act, want_state, out, stream)


def ccq_conv_fwd_varlen(x, w, cu_seqlens, max_len, bias=None, state0=None, act=CCQ_ACT_SILU,
                        want_state=False, out=None, stream=None):
    """ccq_conv_fwd on a packed batch: x [rows,C]; sequence b is rows
    cu_seqlens[b]..cu_seqlens[b+1]-1, at most max_len long."""
    return _conv_fwd(x, w, cu_seqlens, max_len, bias, state0, act, want_state, out, stream)


def _conv_bwd(x, w, dy, cu_seqlens, max_len, bias, state0, dstateT, act, out, workspace, stream):
    shape = _conv_shape(x, w, bias, state0, cu_seqlens, max_len, act)
    dev, dt = x.device, x.dtype
    state = (shape.B, shape.W - 1, shape.C)
    if dy is None:
        raise ValueError("dy is required")
    _check(dy, "dy", x.shape, dt, dev)
    _check(dstateT, "dstateT", state, dt, dev)
    want = {"dx": dy, "dw": w}
    if bias is not None:
        want["dbias"] = bias
    if state0 is not None:
        want["dstate0"] = state0
    with _pool(stream):
        res = _outputs(out, want, dev, (x, w, bias, state0, dy, dstateT))
        ws = _scratch(workspace, int(lib().ccq_conv_workspace_size(shape)), dev)
    args = [x, w, bias, state0, dy, dstateT, res["dx"], res["dw"], res.get("dbias"),
            res.get("dstate0")]
    if cu_seqlens is None:
        _launch("ccq_conv_bwd", dev, stream, shape, args, ws)
    else:
        _launch("ccq_conv_bwd_varlen", dev, stream, shape, [cu_seqlens] + args, ws)
    _record(stream, res, ws, args, cu_seqlens)
    return res


def ccq_conv_bwd(x, w, dy, bias=None, state0=None, dstateT=None, act=CCQ_ACT_SILU, out=None,
                 workspace=None, stream=None):
    """Gradients of ccq_conv_fwd for dy [B,T,C] (and dstateT, the gradient of stateT).  Returns
    dict dx, dw[, dbias][, dstate0]."""
    return _conv_bwd(x, w, dy, None, None, bias, state0, dstateT, act, out, workspace, stream)


def ccq_conv_bwd_varlen(x, w, dy, cu_seqlens, max_len, bias=None, state0=None, dstateT=None,
                        act=CCQ_ACT_SILU, out=None, workspace=None, stream=None):
    """ccq_conv_bwd on a packed batch (layout as ccq_conv_fwd_varlen)."""
    return _conv_bwd(x, w, dy, cu_seqlens, max_len, bias, state0, dstateT, act, out, workspace,
                     stream)


def ccq_conv_step(x, w, state, bias=None, act=CCQ_ACT_SILU, out=None, stream=None):
    """One token per sequence: x [B,C]; state [B,W-1,C] is moved on by the token in place.
    Returns y [B,C]."""
    _on_gpu(x, "x")
    if x.dim() != 2 or w.dim() != 2:
        raise ValueError("x and w: 2 dims expected")
    if state is None:
        raise ValueError("state is required")
    B, C = x.shape
    W = w.shape[1]
    dev, dt = x.device, x.dtype
    _check(w, "w", (C, W), torch.float32, dev)
    _check(bias, "bias", (C,), torch.float32, dev)
    _check(state, "state", (B, W - 1, C), dt, dev)
    dense = x.is_contiguous()
    ld, size = C if dense else _pitch(x, 1, "x"), x.element_size()
    x0, s0 = x.data_ptr(), state.data_ptr()
    s1 = s0 + B * (W - 1) * C * size
    if x0 < s1 and s0 < x0 + B * ld * size:  # (no further than the last token's pitch)
        # the first token that ends behind the state's start, and whether it is there and begins ahead of its end
        i = max(0, (s0 - x0 - C * size) // (ld * size) + 1)
        if i < B and x0 + i * ld * size < s1:
            raise ValueError("state: shares memory with x")
    if out is None and stream is None:
        y = torch.empty_like(x) if dense else torch.empty((B, C), dtype=dt, device=dev)
    else:
        with _pool(stream):
            y = _outputs({"y": out}, {"y": ((B, C), dt)}, dev, (x, w, bias, state))["y"]
    shape = ConvShape(B, 1, C, W, _dt(dt), int(act), ld)
    _launch("ccq_conv_step", dev, stream, shape, (x, w, bias, state, y))
    if stream is not None:
        _record(stream, y, (x, w, bias, state))
    return y


def _norm_shape(x, weight, bias, gate, kind, act, eps):
    _on_gpu(x, "x")
    if x.dim() < 2:
        raise ValueError("x: [..., G, D] expected")
    G, D = x.shape[-2:]
    rows = 1
    for n in x.shape[:-2]:
        rows *= n
    dev, dt = x.device, x.dtype
    shared = weight is not None and weight.dim() == 1
    wshape = (D,) if shared else (G, D)
    _check(weight, "weight", wshape, torch.float32, dev)
    _check(bias, "bias", wshape, torch.float32, dev)
    ldx = ldg = G * D
    if gate is not None:
        if gate.shape != x.shape or gate.dtype != dt or gate.device != dev:
            _check(gate, "gate", x.shape, dt, dev)
        if not gate.is_contiguous():
            ldg = _pitch(gate, 2, "gate")
    if not x.is_contiguous():
        ldx = _pitch(x, 2, "x")
    return NormShape(rows, G, D, _dt(dt), int(kind), int(act), int(shared), float(eps), ldx, ldg)


def ccq_norm_fwd(x, weight=None, bias=None, gate=None, kind=CCQ_NORM_RMS, act=CCQ_ACT_SILU,
                 eps=1e-5, out=None, stream=None):
    """Group norm of every token's heads, channels last: x [..., G, D] (dense, or a slice of a
    wider tensor), each head of each token normalised on its own (kind: CCQ_NORM_GROUP, _RMS,
    _L2), z = n weight + bias with weight, bias [G,D] or, for all heads alike, [D] fp32;
    returns z act(gate) with a gate [..., G, D], else act(z)."""
    shape = _norm_shape(x, weight, bias, gate, kind, act, eps)
    dev = x.device
    if out is None and stream is None:
        y = torch.empty_like(x) if x.is_contiguous() else torch.empty(x.shape, dtype=x.dtype, device=dev)
    else:
        with _pool(stream):
            y = _outputs({"y": out}, {"y": (tuple(x.shape), x.dtype)}, dev, (x, weight, bias, gate))["y"]
    _launch("ccq_norm_fwd", dev, stream, shape, (x, weight, bias, gate, y))
    if stream is not None:
        _record(stream, y, (x, weight, bias, gate))
    return y


def ccq_norm_bwd(x, dy, weight=None, bias=None, gate=None, kind=CCQ_NORM_RMS, act=CCQ_ACT_SILU,
                 eps=1e-5, out=None, workspace=None, stream=None):
    """Gradients of ccq_norm_fwd for dy [..., G, D].  Returns dict dx[, dweight][, dbias][, dgate]."""
    shape = _norm_shape(x, weight, bias, gate, kind, act, eps)
    dev, dt = x.device, x.dtype
    if dy is None:
        raise ValueError("dy is required")
    _check(dy, "dy", x.shape, dt, dev)
    want = {"dx": dy}
    if weight is not None:
        want["dweight"] = weight
    if bias is not None:
        want["dbias"] = bias
    if gate is not None:
        want["dgate"] = dy
    need = int(lib().ccq_norm_workspace_size(shape)) if weight is not None else 0
    with _pool(stream):
        res = _outputs(out, want, dev, (x, dy, weight, bias, gate))
        ws = _scratch(workspace, need, dev)
    _launch("ccq_norm_bwd", dev, stream, shape,
            (x, weight, bias, gate, dy, res["dx"], res.get("dweight"), res.get("dbias"),
             res.get("dgate")), ws)
    _record(stream, res, ws, (x, weight, bias, gate, dy))
    return res
