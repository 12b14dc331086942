"""Thin binding of ``libqdelta.so`` (declared in ``include/qdelta.h``).

Argument marshalling only: torch supplies device memory and the current stream; every step of
the computation runs in the library's CUDA kernels.  The calls that a program makes per step (forward, backward, decode)
marshal natively (``host/*.cpp``), the others through ctypes.  There is no fallback: if the library has
not been built, or a call returns an error code, an exception is raised.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqdelta.so")

QD_F32, QD_BF16 = 0, 1
QD_FWD_SAVE_FOR_BWD, QD_BWD_REUSE_FWD, QD_COEF_LOGITS, QD_NORM_QK, QD_STATE_BF16 = 1, 2, 4, 8, 16
QD_SILU, QD_SOFTPLUS, QD_RMS = 32, 64, 128

EXPORTS = ("qdelta_chunk_workspace_bytes", "qdelta_chunk_fwd", "qdelta_chunk_bwd",
           "qdelta_recurrent_step", "qdelta_workspace_status", "qdelta_status_string",
           "qdelta_profile_enable", "qdelta_profile_stage_count", "qdelta_profile_stage_name",
           "qdelta_profile_read", "qdelta_chunk_fwd_static", "qdelta_chunk_path", "qdelta_chunk_parts",
           "qdelta_recurrent_steps", "qdelta_conv_fwd", "qdelta_conv_steps", "qdelta_conv_workspace_bytes", "qdelta_conv_bwd",
           "qdelta_scan_workspace_bytes", "qdelta_scan_fwd", "qdelta_scan_bwd", "qdelta_scan_steps",
           "qdelta_norm_fwd", "qdelta_norm_workspace_bytes", "qdelta_norm_bwd")


class QdShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("T", ctypes.c_int), ("H", ctypes.c_int), ("dk", ctypes.c_int),
                ("dv", ctypes.c_int), ("chunk", ctypes.c_int), ("dtype", ctypes.c_int)]


class QdScanShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("T", ctypes.c_int), ("D", ctypes.c_int), ("N", ctypes.c_int),
                ("G", ctypes.c_int), ("dtype", ctypes.c_int)]


class QdeltaError(RuntimeError):
    pass


_lib = None
_native = None


def _host():
    """The native marshalling module, which links to libqdelta.so.  Raises if either has not been built."""
    global _native
    if _native is None:
        load()
        try:
            from . import _qdelta_host
        except ImportError as e:
            raise QdeltaError("_qdelta_host.so is not built: run `python -m paper_2606_08804_b200.build` "
                              "(or __graft_entry__.build()); there is no fallback path (%s)" % e) from e
        _qdelta_host.set_error(QdeltaError)
        _native = _qdelta_host
    return _native


def load():
    """Load libqdelta.so (once).  Raises if it is missing: there is no other code path."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise QdeltaError("libqdelta.so is not built: run `python -m paper_2606_08804_b200.build` "
                          "(or __graft_entry__.build()); there is no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    vp, sz, u, i = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_uint, ctypes.c_int
    lib.qdelta_chunk_workspace_bytes.restype = sz
    lib.qdelta_chunk_workspace_bytes.argtypes = [ctypes.POINTER(QdShape), i]
    lib.qdelta_chunk_path.restype = i
    lib.qdelta_chunk_path.argtypes = [ctypes.POINTER(QdShape)]
    lib.qdelta_chunk_parts.restype = i
    lib.qdelta_chunk_parts.argtypes = [ctypes.POINTER(QdShape), i]
    lib.qdelta_chunk_fwd.restype = i
    lib.qdelta_chunk_fwd.argtypes = [ctypes.POINTER(QdShape)] + [vp] * 9 + [vp, sz, u, vp]
    lib.qdelta_chunk_bwd.restype = i
    lib.qdelta_chunk_bwd.argtypes = [ctypes.POINTER(QdShape)] + [vp] * 16 + [vp, sz, u, vp]
    lib.qdelta_chunk_fwd_static.restype = i
    lib.qdelta_chunk_fwd_static.argtypes = [ctypes.POINTER(QdShape)] + [vp] * 9 + [vp, vp]
    lib.qdelta_recurrent_step.restype = i
    lib.qdelta_recurrent_step.argtypes = [i] * 5 + [vp] * 8 + [vp]
    lib.qdelta_recurrent_steps.restype = i
    lib.qdelta_recurrent_steps.argtypes = [i] * 6 + [vp] * 8 + [u, vp]
    ll, f, scan = ctypes.c_longlong, ctypes.c_float, ctypes.POINTER(QdScanShape)
    lib.qdelta_conv_workspace_bytes.restype = sz
    lib.qdelta_conv_workspace_bytes.argtypes = [i] * 5
    lib.qdelta_conv_fwd.argtypes = [i] * 5 + [vp] * 6 + [u, vp]
    lib.qdelta_conv_steps.argtypes = [i] * 5 + [vp] * 5 + [u, vp]
    lib.qdelta_conv_bwd.argtypes = [i] * 5 + [vp] * 11 + [sz, u, vp]
    lib.qdelta_scan_workspace_bytes.restype = sz
    lib.qdelta_scan_workspace_bytes.argtypes = [scan, i]
    lib.qdelta_scan_fwd.argtypes = [scan] + [vp] * 12 + [sz, u, vp]
    lib.qdelta_scan_bwd.argtypes = [scan] + [vp] * 21 + [sz, u, vp]
    lib.qdelta_scan_steps.argtypes = [scan] + [vp] * 10 + [u, vp]
    lib.qdelta_norm_workspace_bytes.restype = sz
    lib.qdelta_norm_workspace_bytes.argtypes = [ll, i, i]
    lib.qdelta_norm_fwd.argtypes = [ll, i, i] + [vp] * 5 + [f, u, vp]
    lib.qdelta_norm_bwd.argtypes = [ll, i, i] + [vp] * 8 + [sz, u, vp]
    lib.qdelta_workspace_status.restype = i
    lib.qdelta_workspace_status.argtypes = [vp, ctypes.POINTER(i), vp]
    lib.qdelta_status_string.restype = ctypes.c_char_p
    lib.qdelta_status_string.argtypes = [i]
    lib.qdelta_profile_enable.restype = i
    lib.qdelta_profile_enable.argtypes = [i]
    lib.qdelta_profile_stage_count.restype = i
    lib.qdelta_profile_stage_name.restype = ctypes.c_char_p
    lib.qdelta_profile_stage_name.argtypes = [i]
    lib.qdelta_profile_read.restype = i
    lib.qdelta_profile_read.argtypes = [i, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_longlong), i]
    _lib = lib
    return lib


def profile_enable(on: bool) -> None:
    """Turn the library's per-kernel CUDA-event timing on or off.  Kernels then run one by one, every sequence in one part."""
    load().qdelta_profile_enable(1 if on else 0)


def profile_read(reset: bool = True) -> dict:
    """{stage name: (total ms, launches)} of everything recorded since the last reset."""
    lib = load()
    out = {}
    for st in range(lib.qdelta_profile_stage_count()):
        ms, n = ctypes.c_double(0), ctypes.c_longlong(0)
        _check(lib.qdelta_profile_read(st, ctypes.byref(ms), ctypes.byref(n), 1 if reset else 0),
               "qdelta_profile_read")
        out[lib.qdelta_profile_stage_name(st).decode()] = (ms.value, n.value)
    return out


def status_string(code: int) -> str:
    return load().qdelta_status_string(int(code)).decode()


def _check(rc, what):
    if rc != 0:
        raise QdeltaError("%s failed: %s (%d)" % (what, status_string(rc), rc))


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return QD_F32
    if t.dtype == torch.bfloat16:
        return QD_BF16
    raise QdeltaError("unsupported dtype %s" % t.dtype)


def _ptr(t, dtype=None, shape=None, name="tensor"):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise QdeltaError("%s must be a contiguous CUDA tensor" % name)
    if dtype is not None and t.dtype != dtype:
        raise QdeltaError("%s must have dtype %s, got %s" % (name, dtype, t.dtype))
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise QdeltaError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    return t.data_ptr()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def make_shape(q, v, chunk) -> QdShape:
    B, T, H, dk = q.shape
    return QdShape(B, T, H, dk, v.shape[-1], int(chunk), _dtype_code(q))


def chunk_workspace_bytes(shape: QdShape, for_backward: bool) -> int:
    n = load().qdelta_chunk_workspace_bytes(ctypes.byref(shape), 1 if for_backward else 0)
    if n == 0:
        raise QdeltaError("unsupported or invalid shape for the chunkwise kernels")
    return int(n)


def chunk_path(shape: QdShape) -> str:
    """Which kernels serve this shape: "tensor_core" (tcgen05) or "fp32" (fp32-accurate products)."""
    r = load().qdelta_chunk_path(ctypes.byref(shape))
    if r < 0:
        raise QdeltaError("unsupported or invalid shape for the chunkwise kernels")
    return "tensor_core" if r == 1 else "fp32"


def chunk_parts(shape: QdShape, backward: bool) -> int:
    """In how many parts a call takes every sequence: the backward, or a forward that returns hT or saves."""
    r = load().qdelta_chunk_parts(ctypes.byref(shape), 1 if backward else 0)
    if r < 0:
        raise QdeltaError("unsupported or invalid shape for the chunkwise kernels")
    return r


def alloc_workspace(shape: QdShape, for_backward: bool, device) -> torch.Tensor:
    return torch.empty(chunk_workspace_bytes(shape, for_backward), dtype=torch.uint8, device=device)


def workspace_status(workspace: torch.Tensor) -> int:
    out = ctypes.c_int(0)
    _check(load().qdelta_workspace_status(workspace.data_ptr(), ctypes.byref(out), _stream()),
           "qdelta_workspace_status")
    return out.value


def chunk_fwd(q, k, v, beta, alpha=None, lam=None, h0=None, chunk=64, save_for_bwd=False,
              workspace=None, o=None, hT=None, want_hT=True, logits=False, norm_qk=False):
    """Chunkwise forward.  Returns (o, hT, workspace).  All tensors live on the GPU.
    logits=True: beta, alpha, lam hold the logits of sigmoid gates (the kernels apply the sigmoid).
    norm_qk=True: q and k are un-normalised, the kernels L2-normalise them per token and head."""
    flags = (QD_FWD_SAVE_FOR_BWD if save_for_bwd else 0) | (QD_COEF_LOGITS if logits else 0) | (QD_NORM_QK if norm_qk else 0)
    return (_native or _host()).chunk_fwd(q, k, v, beta, alpha, lam, h0, int(chunk), workspace, o, hT, bool(want_hT), flags)


def chunk_fwd_static(q, k, v, beta, alpha, lam, h0, o, hT=None, status=None, chunk=64):
    """Forward on the library's built-in scratch array: no workspace, nothing allocated.

    Every output is the caller's: `o` (required), `hT` (optional fp32 final state) and `status`
    (optional int32/uint32 tensor of one element on the GPU that receives the device status word).
    """
    lib = load()
    s = make_shape(q, v, chunk)
    B, T, H, dk, dv, dt = s.B, s.T, s.H, s.dk, s.dv, q.dtype
    if o is None:
        raise QdeltaError("chunk_fwd_static: the output tensor must be supplied (this call allocates nothing)")
    sp = None
    if status is not None:
        if status.numel() != 1 or status.element_size() != 4 or not status.is_cuda:
            raise QdeltaError("chunk_fwd_static: status must be one 32-bit word on the GPU")
        sp = status.data_ptr()
    rc = lib.qdelta_chunk_fwd_static(
        ctypes.byref(s), _ptr(q, dt, (B, T, H, dk), "q"), _ptr(k, dt, (B, T, H, dk), "k"),
        _ptr(v, dt, (B, T, H, dv), "v"), _ptr(beta, dt, (B, T, H), "beta"),
        _ptr(alpha, dt, (B, T, H), "alpha"), _ptr(lam, dt, (B, T, H), "lam"),
        _ptr(h0, torch.float32, (B, H, dk, dv), "h0"), _ptr(o, dt, (B, T, H, dv), "o"),
        _ptr(hT, torch.float32, (B, H, dk, dv), "hT"), sp, _stream())
    _check(rc, "qdelta_chunk_fwd_static")
    torch.autograd.graph.increment_version([t for t in (o, hT, status) if t is not None])
    return o, hT


def chunk_bwd(q, k, v, beta, alpha, lam, h0, dO, dhT=None, chunk=64, workspace=None,
              reuse_fwd=False, out=None, want_dh0=True, logits=False, norm_qk=False):
    """Chunkwise backward.  Returns dict(dq, dk, dv, dbeta, dalpha, dlam, dh0) of GPU tensors.
    logits=True: beta, alpha, lam are logits and dbeta, dalpha, dlam are gradients with respect to them.
    norm_qk=True: q, k are un-normalised and dq, dk are gradients with respect to them."""
    if workspace is None and reuse_fwd:
        raise QdeltaError("reuse_fwd needs the workspace of the forward call")
    flags = (QD_BWD_REUSE_FWD if reuse_fwd else 0) | (QD_COEF_LOGITS if logits else 0) | (QD_NORM_QK if norm_qk else 0)
    return (_native or _host()).chunk_bwd(q, k, v, beta, alpha, lam, h0, int(chunk), dO, dhT, workspace,
                                          out if out is not None else {}, bool(want_dh0), flags)


def recurrent_step(q, k, v, beta, alpha, lam, state, o=None):
    """One decode step; `state` [B,H,dk,dv] fp32 is updated in place.  Returns o [B,H,dv]."""
    return (_native or _host()).recurrent_step(q, k, v, beta, alpha, lam, state, o)


def recurrent_steps(q, k, v, beta, alpha, lam, state, o=None, logits=False, norm_qk=False):
    """S decode tokens per call: q,k [B,S,H,dk], v [B,S,H,dv], coefficients [B,S,H]; `state` [B,H,dk,dv] fp32 is
    updated in place to the state after the last token.  Returns o [B,S,H,dv].  A bf16 `state` selects the
    reduced-precision state option (QD_STATE_BF16)."""
    flags = (QD_COEF_LOGITS if logits else 0) | (QD_NORM_QK if norm_qk else 0)
    return (_native or _host()).recurrent_steps(q, k, v, beta, alpha, lam, state, o, flags)


# ---- operators around the delta rule ------------------------------------------------------------------------------------
# Tensors are contiguous CUDA tensors of one device, bf16 or fp32 (the type of x or u) unless fp32 is said; a call runs on that
# device, in its current stream.  Gradients of parameters are fp32.

def conv_fwd(x, w, bias=None, state=None, silu=False, want_state=True):
    """Short causal convolution per channel.  x [B,T,D], w [D,W] (W = 2, 3, 4), bias [D]; state [B,W-1,D] holds the tokens before
    the first (None: zeros).  silu=True: SiLU of the sum.  Returns (y [B,T,D], the state for the call that goes on from here)."""
    return (_native or _host()).conv_fwd(x, w, bias, state, bool(want_state), QD_SILU if silu else 0)


def conv_bwd(x, w, bias, state, dy, dstate=None, silu=False, want_dstate=None):
    """Backward of conv_fwd: `dstate` is the gradient of the state that it returned.  Returns dict(dx, dw, dbias, dstate), the last
    of the state that it was given (want_dstate: default, if there was one)."""
    want = state is not None if want_dstate is None else bool(want_dstate)
    return (_native or _host()).conv_bwd(x, w, bias, state, dy, dstate, want, QD_SILU if silu else 0)


def conv_steps(x, w, bias, state, y=None, silu=False):
    """S tokens of every sequence, x [B,S,D]: single tokens, and draft tokens.  `state` [B,W-1,D] is updated in place.  Returns y."""
    return (_native or _host()).conv_steps(x, w, bias, state, y, QD_SILU if silu else 0)


def scan_fwd(u, dt, A, Bm, Cm, D=None, z=None, dt_bias=None, h0=None, softplus=False, save_for_bwd=False, workspace=None, want_hT=True):
    """Selective state space scan: h_t = exp(dt_t A) h_{t-1} + dt_t u_t Bm_t, y_t = (<Cm_t, h_t> + D u_t) SiLU(z_t).
    u, dt, z [B,T,D]; A [D,N] (N up to 64), D, dt_bias [D] and h0 [B,D,N] fp32; Bm, Cm [B,T,G,N] serve D / G channels each.
    softplus=True: the step is softplus(dt + dt_bias).  Returns (y, hT [B,D,N] fp32, workspace)."""
    flags = (QD_SOFTPLUS if softplus else 0) | (QD_FWD_SAVE_FOR_BWD if save_for_bwd else 0)
    return (_native or _host()).scan_fwd(u, dt, A, Bm, Cm, D, z, dt_bias, h0, workspace, bool(want_hT), flags)


def scan_bwd(u, dt, A, Bm, Cm, D, z, dt_bias, h0, dy, dhT=None, workspace=None, reuse_fwd=False, softplus=False, want_dh0=None):
    """Backward of scan_fwd; reuse_fwd=True: `workspace` is that of a saving forward of the same inputs.
    Returns dict(du, ddt, dA, dBm, dCm, dD, dz, ddt_bias, dh0); None for those of absent inputs."""
    if workspace is None and reuse_fwd:
        raise QdeltaError("reuse_fwd needs the workspace of the forward call")
    flags = (QD_SOFTPLUS if softplus else 0) | (QD_BWD_REUSE_FWD if reuse_fwd else 0)
    want = h0 is not None if want_dh0 is None else bool(want_dh0)
    return (_native or _host()).scan_bwd(u, dt, A, Bm, Cm, D, z, dt_bias, h0, dy, dhT, workspace, want, flags)


def scan_steps(u, dt, A, Bm, Cm, D, z, dt_bias, state, y=None, softplus=False):
    """S tokens of every sequence, u, dt, z [B,S,D], Bm, Cm [B,S,G,N]: single tokens, and draft tokens.  `state` [B,D,N] fp32 is
    updated in place.  Returns y."""
    return (_native or _host()).scan_steps(u, dt, A, Bm, Cm, D, z, dt_bias, state, y, QD_SOFTPLUS if softplus else 0)


def norm_fwd(x, weight=None, bias=None, eps=1e-5, rms=False, want_stats=True):
    """Layer norm over the last dimension (up to 16384), weight, bias of x's type; rms=True: without the mean.
    Returns (y, stats [2, rows] fp32: mean and reciprocal deviation of every row)."""
    return (_native or _host()).norm_fwd(x, weight, bias, eps, bool(want_stats), QD_RMS if rms else 0)


def norm_bwd(x, weight, dy, stats, rms=False, want_dweight=None, want_dbias=True):
    """Backward of norm_fwd with the `stats` that it returned.  Returns dict(dx, dweight, dbias); None for unwanted ones (dweight:
    wanted if there is a weight)."""
    want = weight is not None if want_dweight is None else bool(want_dweight)
    return (_native or _host()).norm_bwd(x, weight, dy, stats, want, bool(want_dbias), QD_RMS if rms else 0)
