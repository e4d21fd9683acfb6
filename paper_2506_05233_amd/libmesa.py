"""Thin ctypes binding of libmesa (include/libmesa.h).

Argument marshalling only: tensors are checked for device, dtype, shape and
contiguity, then their data pointers and torch's current HIP stream go to the C
ABI.  Every step of the layer runs in libmesa's HIP kernels; there is no
fallback.  Loading fails loudly when the built library is missing.
"""
from __future__ import annotations

import ctypes
import math
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "_lib", "libmesa.so")

MESA_DTYPE_F32 = 0
MESA_DTYPE_BF16 = 1
MESA_DTYPE_Q8 = 2
MESA_PREC_AUTO = 0
MESA_PREC_F32 = 1
MESA_PREC_BF16 = 2
MESA_PREC_BF16X3 = 3
MESA_OK = 0
MESA_ERR_NULL = 1
MESA_ERR_SHAPE = 2
MESA_ERR_UNSUPPORTED = 3
MESA_ERR_ARG = 4
MESA_ERR_WORKSPACE = 5
MESA_ERR_HIP = 6
MESA_ERR_NONFINITE = 7
MESA_MAX_NCG = 1024
MESA_NOALLOC_SCRATCH_BYTES = 64 << 20
MESA_CHECKPOINT_GROUP = 32
MESA_RECURRENCE_BLOCK = 128

EXPORTED = ("mesa_forward", "mesa_forward_ex", "mesa_forward_states", "mesa_forward_solve",
            "mesa_forward_tol", "mesa_forward_workspace_bytes", "mesa_decode_step",
            "mesa_decode_step_tol", "mesa_decode_step_packed", "mesa_pack_state", "mesa_unpack_state",
            "mesa_backward", "mesa_backward_workspace_bytes", "mesa_forward_noalloc",
            "mesa_frontend", "mesa_output_norm",
            "mesa_checkpoint_bytes", "mesa_checkpoint_pack", "mesa_checkpoint_unpack",
            "mesa_recurrence", "mesa_recurrence_workspace_bytes", "mesa_recurrence_step",
            "mesa_recurrence_backward", "mesa_recurrence_backward_workspace_bytes",
            "mesa_frontend_backward", "mesa_frontend_backward_workspace_bytes",
            "mesa_output_norm_backward", "mesa_output_norm_backward_workspace_bytes",
            "mesa_status_string", "mesa_version")

_lib = None


class MesaError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s (status %d)" % (where, status_string(status), status))


def load():
    """Load libmesa.so (built by paper_2506_05233_amd/build.py); raise if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libmesa is not built: %s is missing (run __graft_entry__.build())" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    vp, fp, i64, ci, sz = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_size_t
    lib.mesa_forward_workspace_bytes.argtypes = [i64, i64, i64, i64, i64, ci]
    lib.mesa_forward_workspace_bytes.restype = sz
    lib.mesa_forward.argtypes = [vp, vp, vp, fp, fp, fp, i64, i64, i64, i64, i64, ci, ci, ci, fp, vp, sz, vp]
    lib.mesa_forward.restype = ci
    lib.mesa_forward_ex.argtypes = [vp, vp, vp, fp, fp, fp, i64, i64, i64, i64, i64, ci, ci, ci, ci,
                                    fp, fp, fp, fp, vp, sz, vp]
    lib.mesa_forward_ex.restype = ci
    lib.mesa_forward_states.argtypes = [vp, vp, fp, fp, i64, i64, i64, i64, i64, ci, ci, ci, fp, fp, vp, sz, vp]
    lib.mesa_forward_states.restype = ci
    lib.mesa_forward_solve.argtypes = [vp, vp, vp, fp, fp, fp, i64, i64, i64, i64, i64, ci, ci, ci, ci,
                                       fp, fp, vp, sz, vp]
    lib.mesa_forward_solve.restype = ci
    lib.mesa_decode_step.argtypes = [fp, fp, vp, vp, vp, fp, fp, fp, i64, i64, i64, i64, ci, ci, fp, vp]
    lib.mesa_decode_step.restype = ci
    cf = ctypes.c_float
    lib.mesa_forward_tol.argtypes = [vp, vp, vp, fp, fp, fp, i64, i64, i64, i64, i64, ci, ci, cf, ci, ci,
                                     fp, fp, vp, vp, sz, vp]
    lib.mesa_forward_tol.restype = ci
    lib.mesa_decode_step_tol.argtypes = [fp, fp, vp, vp, vp, fp, fp, fp, i64, i64, i64, i64, ci, ci, cf,
                                         fp, vp, vp]
    lib.mesa_decode_step_tol.restype = ci
    lib.mesa_decode_step_packed.argtypes = [fp, fp, vp, vp, vp, fp, fp, fp, i64, i64, i64, i64, ci, ci, cf,
                                            fp, vp, vp]
    lib.mesa_decode_step_packed.restype = ci
    lib.mesa_pack_state.argtypes = [fp, fp, i64, i64, i64, vp]
    lib.mesa_pack_state.restype = ci
    lib.mesa_unpack_state.argtypes = [fp, fp, i64, i64, i64, vp]
    lib.mesa_unpack_state.restype = ci
    lib.mesa_backward_workspace_bytes.argtypes = [i64, i64, i64, i64, i64]
    lib.mesa_backward_workspace_bytes.restype = sz
    lib.mesa_backward.argtypes = [vp, vp, fp, fp, fp, i64, i64, i64, i64, i64, ci, ci, ci, fp, fp,
                                  fp, fp, fp, fp, fp, fp, vp, sz, vp]
    lib.mesa_backward.restype = ci
    lib.mesa_forward_noalloc.argtypes = [vp, vp, vp, fp, fp, fp, i64, i64, i64, i64, i64, ci, ci, ci, fp, vp]
    lib.mesa_forward_noalloc.restype = ci
    lib.mesa_frontend.argtypes = [vp, vp, vp, fp, fp, fp, fp, fp, fp, cf, cf, i64, i64, i64, i64, i64, ci,
                                   vp, vp, vp, fp, fp, fp, vp]
    lib.mesa_frontend.restype = ci
    lib.mesa_output_norm.argtypes = [fp, fp, cf, i64, i64, i64, i64, ci, vp, vp]
    lib.mesa_output_norm.restype = ci
    lib.mesa_checkpoint_bytes.argtypes = [i64, i64]
    lib.mesa_checkpoint_bytes.restype = sz
    lib.mesa_checkpoint_pack.argtypes = lib.mesa_checkpoint_unpack.argtypes = [vp, i64, i64, i64, ci, vp, vp]
    lib.mesa_checkpoint_pack.restype = lib.mesa_checkpoint_unpack.restype = ci
    lib.mesa_recurrence_workspace_bytes.argtypes = [i64, i64, i64]
    lib.mesa_recurrence_workspace_bytes.restype = sz
    lib.mesa_recurrence.argtypes = [vp, vp, vp, fp, cf, vp, fp, i64, i64, i64, i64, ci, vp, fp, fp, vp, vp, vp, vp, sz, vp]
    lib.mesa_recurrence.restype = ci
    lib.mesa_recurrence_step.argtypes = [fp, vp, vp, vp, fp, cf, vp, i64, i64, i64, ci, fp, vp, vp]
    lib.mesa_recurrence_step.restype = ci
    lib.mesa_recurrence_backward_workspace_bytes.argtypes = [i64, i64, i64]
    lib.mesa_recurrence_backward_workspace_bytes.restype = sz
    lib.mesa_recurrence_backward.argtypes = [vp, vp, vp, fp, cf, vp, fp, vp, fp, i64, i64, i64, i64, ci, ci, i64,
                                             vp, vp, vp, fp, fp, vp, sz, vp]
    lib.mesa_recurrence_backward.restype = ci
    lib.mesa_frontend_backward_workspace_bytes.argtypes = [i64, i64, i64, i64, i64]
    lib.mesa_frontend_backward_workspace_bytes.restype = sz
    lib.mesa_frontend_backward.argtypes = ([vp, vp, vp, fp, fp, fp, fp, fp, fp, cf, cf, i64, i64, i64, i64, i64, ci]
                                           + [fp] * 6 + [ci] + [vp] * 3 + [fp] * 6 + [vp, sz, vp])
    lib.mesa_frontend_backward.restype = ci
    lib.mesa_output_norm_backward_workspace_bytes.argtypes = [i64, i64, i64, i64]
    lib.mesa_output_norm_backward_workspace_bytes.restype = sz
    lib.mesa_output_norm_backward.argtypes = [vp, fp, cf, vp, i64, i64, i64, i64, ci, ci, fp, fp, vp, sz, vp]
    lib.mesa_output_norm_backward.restype = ci
    lib.mesa_status_string.argtypes = [ci]
    lib.mesa_status_string.restype = ctypes.c_char_p
    lib.mesa_version.argtypes = []
    lib.mesa_version.restype = ci
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().mesa_status_string(int(status)).decode()


def version() -> int:
    return load().mesa_version()


def forward_workspace_bytes(batch, heads, seq_len, d_k, d_v, chunk) -> int:
    return load().mesa_forward_workspace_bytes(batch, heads, seq_len, d_k, d_v, chunk)


def bf16_path_available(d_k, d_v, chunk, seq_len=2048) -> bool:
    """Whether MESA_PREC_BF16 (the matrix-core path) supports this shape: a
    zero-batch solve call validates the arguments and launches nothing."""
    st = load().mesa_forward_solve(None, None, None, None, None, None, 0, 1, seq_len, d_k, d_v,
                                   MESA_DTYPE_BF16, 1, chunk, MESA_PREC_BF16, None, None, None, 0,
                                   None)
    return st == MESA_OK


# ---------------------------------------------------------------- torch glue
def _torch():
    import torch
    return torch


def _dtype_code(t):
    torch = _torch()
    if t.dtype == torch.float32:
        return MESA_DTYPE_F32
    if t.dtype == torch.bfloat16:
        return MESA_DTYPE_BF16
    raise TypeError("q, k, v must be float32 or bfloat16, got %s" % t.dtype)


def _check(t, name, shape, dtype=None, device=None):
    torch = _torch()
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.shape == shape and (dtype is None or t.dtype is dtype)
            and (device is None or t.device == device) and t.is_contiguous()):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if device is not None and t.device != device:
        raise ValueError("%s is on %s, expected %s" % (name, t.device, device))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)


def _workspace(workspace, need, device):
    """A caller's workspace, when it is given, on the device and large enough, or a new one.  It
    must be contiguous: a kernel writes the bytes that it counts, one after the other."""
    if need == 0:
        return None
    torch = _torch()
    if workspace is not None:
        if not isinstance(workspace, torch.Tensor):
            raise TypeError("workspace must be a torch.Tensor")
        if workspace.device == device and workspace.numel() * workspace.element_size() >= need:
            if not workspace.is_contiguous():
                raise ValueError("workspace must be contiguous")
            return workspace
    return torch.empty(need, dtype=torch.uint8, device=device)


def _ptr(t):
    return None if t is None else t.data_ptr()


_raw_stream = None


def _stream(device):
    """torch's current HIP stream of the device, as the C ABI takes it."""
    global _raw_stream
    if _raw_stream is None:
        torch = _torch()
        # the handle itself: building a torch.cuda.Stream around it takes longer than a short call
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda index: torch.cuda.current_stream(index).cuda_stream)
    return _raw_stream(device.index)


def forward(q, k, v, gamma, beta, lam, n_cg, chunk=64, precision=MESA_PREC_AUTO, want_qstar=False,
            want_states=False, out=None, workspace=None, eps=None, want_steps=False):
    """Mesa forward over q, k [B,H,T,d_k], v [B,H,T,d_v] (fp32 or bf16, same dtype),
    gamma, beta [B,H,T] fp32, lam [H,d_k] fp32.  Returns out [B,H,T,d_v] fp32, or a
    dict with "out" and, if asked, "qstar" [B,H,T,d_k], "H" [B,H,d_k,d_k], "G" [B,H,d_v,d_k],
    "steps" [B,H,T] int32 (CG iterations per token).
    eps: CG relative tolerance (Alg. 1's |r_k| <= eps |r_0|; n_cg is then the limit),
    through mesa_forward_tol; None or 0 with want_steps False is the fixed-step solve.
    Runs on torch's current stream of q's device."""
    torch = _torch()
    lib = load()
    B, H, T, dk = q.shape
    dv = v.shape[-1]
    dev = q.device
    _check(q, "q", (B, H, T, dk), device=dev)
    _check(k, "k", (B, H, T, dk), q.dtype, dev)
    _check(v, "v", (B, H, T, dv), q.dtype, dev)
    _check(gamma, "gamma", (B, H, T), torch.float32, dev)
    _check(beta, "beta", (B, H, T), torch.float32, dev)
    _check(lam, "lam", (H, dk), torch.float32, dev)
    code = _dtype_code(q)
    if out is None:
        out = torch.empty((B, H, T, dv), dtype=torch.float32, device=dev)
    _check(out, "out", (B, H, T, dv), torch.float32, dev)
    need = lib.mesa_forward_workspace_bytes(B, H, T, dk, dv, chunk)
    workspace = _workspace(workspace, max(need, 1), dev)
    qstar = torch.empty((B, H, T, dk), dtype=torch.float32, device=dev) if want_qstar else None
    if eps is not None or want_steps:
        if want_states:
            raise ValueError("mesa_forward_tol returns no final states")
        steps = torch.empty((B, H, T), dtype=torch.int32, device=dev) if want_steps else None
        st = lib.mesa_forward_tol(_ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(beta), _ptr(lam), B, H,
                                  T, dk, dv, code, int(n_cg), float(eps or 0.0), int(chunk),
                                  int(precision), _ptr(out), _ptr(qstar), _ptr(steps), _ptr(workspace),
                                  workspace.numel() * workspace.element_size(), _stream(dev))
        if st != MESA_OK:
            raise MesaError(st, "mesa_forward_tol")
        res = {"out": out}
        if want_qstar:
            res["qstar"] = qstar
        if want_steps:
            res["steps"] = steps
        return res if (want_qstar or want_steps) else out
    fH = torch.empty((B, H, dk, dk), dtype=torch.float32, device=dev) if want_states else None
    fG = torch.empty((B, H, dv, dk), dtype=torch.float32, device=dev) if want_states else None
    st = lib.mesa_forward_ex(_ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(beta), _ptr(lam), B, H, T,
                             dk, dv, code, int(n_cg), int(chunk), int(precision), _ptr(out),
                             _ptr(qstar), _ptr(fH), _ptr(fG), _ptr(workspace),
                             workspace.numel() * workspace.element_size(), _stream(dev))
    if st != MESA_OK:
        raise MesaError(st, "mesa_forward_ex")
    if not (want_qstar or want_states):
        return out
    res = {"out": out}
    if want_qstar:
        res["qstar"] = qstar
    if want_states:
        res["H"] = fH
        res["G"] = fG
    return res


def frontend(qp, kp, vp, conv_q, conv_k, conv_v, a_gamma, a_beta, theta, gamma_cap=0.9975, l2_eps=1e-6):
    """mesa_frontend: the layer's inputs from the projections (App. E, App. G.5).
    qp, kp [B,T,H,d_k], vp [B,T,H,d_v] (fp32 or bf16, one dtype); conv_q, conv_k
    [H*d_k,4], conv_v [H*d_v,4] or None; a_gamma, a_beta [B,T,H]; theta [H,d_k] (fp32).
    Returns a dict: q, k [B,H,T,d_k], v [B,H,T,d_v] (the projections' dtype), gamma,
    beta [B,H,T], lam [H,d_k] (fp32)."""
    torch = _torch()
    lib = load()
    B, T, H, dk = qp.shape
    dv = vp.shape[-1]
    dev = qp.device
    f32 = torch.float32
    _check(qp, "qp", (B, T, H, dk), device=dev)
    _check(kp, "kp", (B, T, H, dk), qp.dtype, dev)
    _check(vp, "vp", (B, T, H, dv), qp.dtype, dev)
    _check(conv_q, "conv_q", (H * dk, 4), f32, dev)
    _check(conv_k, "conv_k", (H * dk, 4), f32, dev)
    if conv_v is not None:
        _check(conv_v, "conv_v", (H * dv, 4), f32, dev)
    _check(a_gamma, "a_gamma", (B, T, H), f32, dev)
    _check(a_beta, "a_beta", (B, T, H), f32, dev)
    _check(theta, "theta", (H, dk), f32, dev)
    res = {"q": torch.empty((B, H, T, dk), dtype=qp.dtype, device=dev),
           "k": torch.empty((B, H, T, dk), dtype=qp.dtype, device=dev),
           "v": torch.empty((B, H, T, dv), dtype=qp.dtype, device=dev),
           "gamma": torch.empty((B, H, T), dtype=f32, device=dev),
           "beta": torch.empty((B, H, T), dtype=f32, device=dev),
           "lam": torch.empty((H, dk), dtype=f32, device=dev)}
    st = lib.mesa_frontend(_ptr(qp), _ptr(kp), _ptr(vp), _ptr(conv_q), _ptr(conv_k), _ptr(conv_v), _ptr(a_gamma),
                           _ptr(a_beta), _ptr(theta), float(gamma_cap), float(l2_eps), B, H, T, dk, dv,
                           _dtype_code(qp), _ptr(res["q"]), _ptr(res["k"]), _ptr(res["v"]), _ptr(res["gamma"]),
                           _ptr(res["beta"]), _ptr(res["lam"]), _stream(dev))
    if st != MESA_OK:
        raise MesaError(st, "mesa_frontend")
    return res


def output_norm(o, weight, eps=1e-6, out_dtype=None):
    """mesa_output_norm: per-head RMSNorm of the layer output o [B,H,T,d_v] fp32 with
    weight [H,d_v], into [B,T,H,d_v] of out_dtype (torch.bfloat16 by default)."""
    torch = _torch()
    lib = load()
    B, H, T, dv = o.shape
    dev = o.device
    _check(o, "o", (B, H, T, dv), torch.float32, dev)
    _check(weight, "weight", (H, dv), torch.float32, dev)
    out_dtype = torch.bfloat16 if out_dtype is None else out_dtype
    y = torch.empty((B, T, H, dv), dtype=out_dtype, device=dev)
    st = lib.mesa_output_norm(_ptr(o), _ptr(weight), float(eps), B, H, T, dv, _dtype_code(y), _ptr(y),
                              _stream(dev))
    if st != MESA_OK:
        raise MesaError(st, "mesa_output_norm")
    return y


def forward_noalloc(q, k, v, gamma, beta, lam, n_cg, chunk=64, out=None):
    """mesa_forward_noalloc: the forward with the chunk states in the library's own
    fixed device buffer (no workspace; MesaError with MESA_ERR_WORKSPACE when the
    shape needs more than MESA_NOALLOC_SCRATCH_BYTES).  Same inputs as forward();
    returns out [B,H,T,d_v] fp32 (allocated here unless given)."""
    torch = _torch()
    lib = load()
    B, H, T, dk = q.shape
    dv = v.shape[-1]
    dev = q.device
    _check(q, "q", (B, H, T, dk), device=dev)
    _check(k, "k", (B, H, T, dk), q.dtype, dev)
    _check(v, "v", (B, H, T, dv), q.dtype, dev)
    _check(gamma, "gamma", (B, H, T), torch.float32, dev)
    _check(beta, "beta", (B, H, T), torch.float32, dev)
    _check(lam, "lam", (H, dk), torch.float32, dev)
    if out is None:
        out = torch.empty((B, H, T, dv), dtype=torch.float32, device=dev)
    _check(out, "out", (B, H, T, dv), torch.float32, dev)
    st = lib.mesa_forward_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(beta), _ptr(lam), B, H, T,
                                  dk, dv, _dtype_code(q), int(n_cg), int(chunk), _ptr(out), _stream(dev))
    if st != MESA_OK:
        raise MesaError(st, "mesa_forward_noalloc")
    return out


class ForwardPlan:
    """Pre-checked arguments of one forward shape, for repeated calls of the two
    launches (mesa_forward_states, then mesa_forward_solve) on torch's current
    stream.  Holds the output and workspace tensors; used by the benchmark to
    time each launch with events on the launch stream."""

    def __init__(self, q, k, v, gamma, beta, lam, n_cg, chunk=64, precision=MESA_PREC_AUTO):
        torch = _torch()
        self.lib = load()
        B, H, T, dk = q.shape
        dv = v.shape[-1]
        dev = q.device
        _check(q, "q", (B, H, T, dk), device=dev)
        _check(k, "k", (B, H, T, dk), q.dtype, dev)
        _check(v, "v", (B, H, T, dv), q.dtype, dev)
        _check(gamma, "gamma", (B, H, T), torch.float32, dev)
        _check(beta, "beta", (B, H, T), torch.float32, dev)
        _check(lam, "lam", (H, dk), torch.float32, dev)
        self.tensors = (q, k, v, gamma, beta, lam)
        self.dims = (B, H, T, dk, dv)
        self.code = _dtype_code(q)
        self.n_cg, self.chunk, self.precision = int(n_cg), int(chunk), int(precision)
        self.device = dev
        self.out = torch.empty((B, H, T, dv), dtype=torch.float32, device=dev)
        self.ws_bytes = self.lib.mesa_forward_workspace_bytes(B, H, T, dk, dv, chunk)
        self.workspace = torch.empty(max(self.ws_bytes, 1), dtype=torch.uint8, device=dev)

    def states(self):
        q, k, v, gamma, beta, lam = self.tensors
        B, H, T, dk, dv = self.dims
        st = self.lib.mesa_forward_states(_ptr(k), _ptr(v), _ptr(gamma), _ptr(beta), B, H, T, dk, dv,
                                          self.code, self.chunk, self.precision, None, None,
                                          _ptr(self.workspace), self.ws_bytes, _stream(self.device))
        if st != MESA_OK:
            raise MesaError(st, "mesa_forward_states")

    def solve(self):
        q, k, v, gamma, beta, lam = self.tensors
        B, H, T, dk, dv = self.dims
        st = self.lib.mesa_forward_solve(_ptr(q), _ptr(k), _ptr(v), _ptr(gamma), _ptr(beta), _ptr(lam),
                                         B, H, T, dk, dv, self.code, self.n_cg, self.chunk,
                                         self.precision, _ptr(self.out), None, _ptr(self.workspace),
                                         self.ws_bytes, _stream(self.device))
        if st != MESA_OK:
            raise MesaError(st, "mesa_forward_solve")
        return self.out

    def __call__(self):
        self.states()
        return self.solve()


def backward_workspace_bytes(batch, heads, seq_len, d_k, d_v) -> int:
    return load().mesa_backward_workspace_bytes(batch, heads, seq_len, d_k, d_v)


def backward(k, v, gamma, beta, lam, qstar, dout, n_cg, precision=MESA_PREC_AUTO, workspace=None):
    """Gradients of the layer given dout = dL/do [B,H,T,d_v] fp32 and the forward's
    q* [B,H,T,d_k] fp32 (mesa_backward).  k, v [B,H,T,d] fp32 or bf16; gamma, beta
    [B,H,T]; lam [H,d_k].  precision selects the solve for e* (MESA_PREC_F32, or
    MESA_PREC_BF16 on the matrix cores; AUTO: BF16 for bf16 inputs).  Returns a dict
    of fp32 tensors: "dq", "dk" [B,H,T,d_k], "dv" [B,H,T,d_v], "dgamma", "dbeta"
    [B,H,T], "dlam" [H,d_k].
    Runs on torch's current stream of k's device."""
    torch = _torch()
    lib = load()
    B, H, T, dk = k.shape
    dv = v.shape[-1]
    dev = k.device
    _check(k, "k", (B, H, T, dk), device=dev)
    _check(v, "v", (B, H, T, dv), k.dtype, dev)
    _check(gamma, "gamma", (B, H, T), torch.float32, dev)
    _check(beta, "beta", (B, H, T), torch.float32, dev)
    _check(lam, "lam", (H, dk), torch.float32, dev)
    _check(qstar, "qstar", (B, H, T, dk), torch.float32, dev)
    _check(dout, "dout", (B, H, T, dv), torch.float32, dev)
    need = lib.mesa_backward_workspace_bytes(B, H, T, dk, dv)
    workspace = _workspace(workspace, max(need, 1), dev)
    f32 = dict(dtype=torch.float32, device=dev)
    res = {"dq": torch.empty((B, H, T, dk), **f32), "dk": torch.empty((B, H, T, dk), **f32),
           "dv": torch.empty((B, H, T, dv), **f32), "dgamma": torch.empty((B, H, T), **f32),
           "dbeta": torch.empty((B, H, T), **f32), "dlam": torch.empty((H, dk), **f32)}
    st = lib.mesa_backward(_ptr(k), _ptr(v), _ptr(gamma), _ptr(beta), _ptr(lam), B, H, T, dk, dv,
                           _dtype_code(k), int(n_cg), int(precision), _ptr(qstar), _ptr(dout), _ptr(res["dq"]),
                           _ptr(res["dk"]), _ptr(res["dv"]), _ptr(res["dgamma"]), _ptr(res["dbeta"]),
                           _ptr(res["dlam"]), _ptr(workspace), workspace.numel() * workspace.element_size(),
                           _stream(dev))
    if st != MESA_OK:
        raise MesaError(st, "mesa_backward")
    return res


def prefill_states(k, v, gamma, beta, chunk=64, workspace=None):
    """States after the last token only (mesa_forward_ex with out = NULL):
    returns (H [B,H,d_k,d_k], G [B,H,d_v,d_k]) fp32, the input of decode_step.
    workspace: optional device tensor of at least mesa_forward_workspace_bytes,
    scratch that lets the scan of few long sequences run in segments."""
    torch = _torch()
    lib = load()
    B, H, T, dk = k.shape
    dv = v.shape[-1]
    dev = k.device
    _check(k, "k", (B, H, T, dk), device=dev)
    _check(v, "v", (B, H, T, dv), k.dtype, dev)
    _check(gamma, "gamma", (B, H, T), torch.float32, dev)
    _check(beta, "beta", (B, H, T), torch.float32, dev)
    code = _dtype_code(k)
    fH = torch.empty((B, H, dk, dk), dtype=torch.float32, device=dev)
    fG = torch.empty((B, H, dv, dk), dtype=torch.float32, device=dev)
    ws_ptr, ws_bytes = None, 0
    if workspace is not None:
        _check(workspace, "workspace", tuple(workspace.shape), device=dev)
        ws_ptr, ws_bytes = _ptr(workspace), workspace.numel() * workspace.element_size()
    st = lib.mesa_forward_ex(None, _ptr(k), _ptr(v), _ptr(gamma), _ptr(beta), None, B, H, T, dk, dv,
                             code, 0, int(chunk), MESA_PREC_AUTO, None, None, _ptr(fH), _ptr(fG),
                             ws_ptr, ws_bytes, _stream(dev))
    if st != MESA_OK:
        raise MesaError(st, "mesa_forward_ex(states only)")
    return fH, fG


def pack_state(state_H):
    """Full symmetric decode state H [N,H,d_k,d_k] -> packed cyclic diagonals
    [N,H,d_k/2+1,d_k] (mesa_pack_state)."""
    torch = _torch()
    lib = load()
    N, H, dk, _ = state_H.shape
    _check(state_H, "state_H", (N, H, dk, dk), torch.float32, state_H.device)
    hp = torch.empty((N, H, dk // 2 + 1, dk), dtype=torch.float32, device=state_H.device)
    st = lib.mesa_pack_state(_ptr(state_H), _ptr(hp), N, H, dk, _stream(state_H.device))
    if st != MESA_OK:
        raise MesaError(st, "mesa_pack_state")
    return hp


def unpack_state(state_HP):
    """Packed [N,H,d_k/2+1,d_k] -> full symmetric H [N,H,d_k,d_k] (mesa_unpack_state)."""
    torch = _torch()
    lib = load()
    N, H, _, dk = state_HP.shape
    _check(state_HP, "state_HP", (N, H, dk // 2 + 1, dk), torch.float32, state_HP.device)
    h = torch.empty((N, H, dk, dk), dtype=torch.float32, device=state_HP.device)
    st = lib.mesa_unpack_state(_ptr(state_HP), _ptr(h), N, H, dk, _stream(state_HP.device))
    if st != MESA_OK:
        raise MesaError(st, "mesa_unpack_state")
    return h


def decode_step(state_H, state_G, q, k, v, gamma, beta, lam, n_cg, out=None, eps=None, steps_out=None,
                packed=False):
    """One recurrent step, in place on state_H [N,H,d_k,d_k] (or, with packed, the
    cyclic-diagonal form [N,H,d_k/2+1,d_k] of pack_state) and state_G [N,H,d_v,d_k].
    q, k [N,H,d_k], v [N,H,d_v] fp32 or bf16; gamma, beta [N,H]; lam [H,d_k].
    eps / steps_out (int32 [N,H]): CG relative tolerance and iteration counts, through
    mesa_decode_step_tol (or mesa_decode_step_packed).  Returns out [N,H,d_v] fp32."""
    torch = _torch()
    lib = load()
    N, H, dk = q.shape
    dv = v.shape[-1]
    dev = q.device
    _check(state_H, "state_H", (N, H, dk // 2 + 1 if packed else dk, dk), torch.float32, dev)
    _check(state_G, "state_G", (N, H, dv, dk), torch.float32, dev)
    _check(q, "q", (N, H, dk), device=dev)
    _check(k, "k", (N, H, dk), q.dtype, dev)
    _check(v, "v", (N, H, dv), q.dtype, dev)
    _check(gamma, "gamma", (N, H), torch.float32, dev)
    _check(beta, "beta", (N, H), torch.float32, dev)
    _check(lam, "lam", (H, dk), torch.float32, dev)
    if out is None:
        out = torch.empty((N, H, dv), dtype=torch.float32, device=dev)
    _check(out, "out", (N, H, dv), torch.float32, dev)
    if packed:
        if steps_out is not None:
            _check(steps_out, "steps_out", (N, H), torch.int32, dev)
        st = lib.mesa_decode_step_packed(_ptr(state_H), _ptr(state_G), _ptr(q), _ptr(k), _ptr(v),
                                         _ptr(gamma), _ptr(beta), _ptr(lam), N, H, dk, dv, _dtype_code(q),
                                         int(n_cg), float(eps or 0.0), _ptr(out), _ptr(steps_out),
                                         _stream(dev))
        if st != MESA_OK:
            raise MesaError(st, "mesa_decode_step_packed")
        return out
    if eps is not None or steps_out is not None:
        if steps_out is not None:
            _check(steps_out, "steps_out", (N, H), torch.int32, dev)
        st = lib.mesa_decode_step_tol(_ptr(state_H), _ptr(state_G), _ptr(q), _ptr(k), _ptr(v),
                                      _ptr(gamma), _ptr(beta), _ptr(lam), N, H, dk, dv, _dtype_code(q),
                                      int(n_cg), float(eps or 0.0), _ptr(out), _ptr(steps_out),
                                      _stream(dev))
        if st != MESA_OK:
            raise MesaError(st, "mesa_decode_step_tol")
        return out
    st = lib.mesa_decode_step(_ptr(state_H), _ptr(state_G), _ptr(q), _ptr(k), _ptr(v), _ptr(gamma),
                              _ptr(beta), _ptr(lam), N, H, dk, dv, _dtype_code(q), int(n_cg),
                              _ptr(out), _stream(dev))
    if st != MESA_OK:
        raise MesaError(st, "mesa_decode_step")
    return out


# ---------------------------------------------------------------- 8-bit checkpoints
def _row_stride(t, name):
    """Elements between the rows of t [..., width]: its last dimension dense, the leading ones
    one even run of rows."""
    if t.is_contiguous():
        return t.shape[-1]
    shape, stride = t.shape, t.stride()
    if shape[-1] > 1 and stride[-1] != 1:
        raise ValueError("%s must be dense along its last dimension" % name)
    row = span = None
    for n, st in zip(reversed(shape[:-1]), reversed(stride[:-1])):
        if n == 1:
            continue
        if row is None:
            row = st
        elif st != span:
            raise ValueError("%s must have evenly spaced rows" % name)
        span = st * n
    if row is None:
        return shape[-1]
    if row < shape[-1]:
        raise ValueError("%s must not overlap itself" % name)
    return row


def _check_all(dtype, device, *items):
    """_check of several (tensor, name, shape) of one dtype in one go."""
    Tensor = _torch().Tensor
    for t, name, shape in items:
        if not (isinstance(t, Tensor) and t.shape == shape and t.dtype is dtype and t.device == device and t.is_contiguous()):
            _check(t, name, shape, dtype, device)


def _check_rows(t, name, shape, dtype, device):
    """As _check, for a tensor whose rows may be spaced; returns their stride."""
    if not isinstance(t, _torch().Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.shape != shape:
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.device != device:
        raise ValueError("%s is on %s, expected %s" % (name, t.device, device))
    return shape[-1] if t.is_contiguous() else _row_stride(t, name)


def _float_code(dtype, name):
    torch = _torch()
    if dtype is torch.float32:
        return MESA_DTYPE_F32
    if dtype is torch.bfloat16:
        return MESA_DTYPE_BF16
    raise TypeError("%s must be float32 or bfloat16, got %s" % (name, dtype))


def _on_device(t, name):
    if not isinstance(t, _torch().Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    return t.device


def checkpoint_bytes(rows, width) -> int:
    return load().mesa_checkpoint_bytes(rows, width)


class Checkpoint:
    """An 8-bit checkpoint of a tensor of `shape` ([..., width]): the device buffer that
    mesa_checkpoint_pack writes, about 1.03 bytes a value."""

    __slots__ = ("buffer", "shape", "rows", "width")

    def __init__(self, buffer, shape):
        torch = _torch()
        self.shape = shape = tuple(int(n) for n in shape)
        self.rows, self.width = math.prod(shape[:-1]), shape[-1]
        _on_device(buffer, "buffer")
        need = checkpoint_bytes(self.rows, self.width)
        if buffer.dtype != torch.uint8 or not buffer.is_contiguous() or buffer.numel() < need:
            raise ValueError("buffer must be a contiguous uint8 tensor of %d bytes" % need)
        self.buffer = buffer

    @classmethod
    def empty(cls, shape, device):
        """A checkpoint of that shape with nothing in it yet."""
        torch = _torch()
        ck = cls.__new__(cls)
        ck.shape = shape = tuple(shape)
        ck.rows, ck.width = math.prod(shape[:-1]), shape[-1]
        ck.buffer = torch.empty(checkpoint_bytes(ck.rows, ck.width), dtype=torch.uint8, device=device)
        return ck

    @property
    def device(self):
        return self.buffer.device

    @property
    def codes(self):
        """int8 [rows, width]"""
        n = self.rows * self.width
        return self.buffer[:n].view(_torch().int8).view(self.rows, self.width)

    @property
    def exponents(self):
        """uint8 [rows, ceil(width / 32)]: E + 127 of each group, 255 for one that is not finite"""
        at = -(-self.rows * self.width // 16) * 16
        groups = -(-self.width // MESA_CHECKPOINT_GROUP)
        return self.buffer[at:at + self.rows * groups].view(self.rows, groups)


def checkpoint_pack(x):
    """mesa_checkpoint_pack: x [..., width] fp32 or bf16 (rows evenly spaced, so a slice of a
    fused projection will do) as a Checkpoint."""
    lib = load()
    dev = _on_device(x, "x")
    code = _float_code(x.dtype, "x")
    stride = _row_stride(x, "x")
    ck = Checkpoint.empty(x.shape, dev)
    st = lib.mesa_checkpoint_pack(_ptr(x), ck.rows, ck.width, stride, code, _ptr(ck.buffer), _stream(dev))
    if st != MESA_OK:
        raise MesaError(st, "mesa_checkpoint_pack")
    return ck


def checkpoint_unpack(ck, dtype=None, out=None):
    """mesa_checkpoint_unpack: the values of a Checkpoint, as dtype (torch.bfloat16 by default,
    which holds them exactly) or into out (rows evenly spaced)."""
    torch = _torch()
    lib = load()
    dev = ck.device
    if out is None:
        out = torch.empty(ck.shape, dtype=torch.bfloat16 if dtype is None else dtype, device=dev)
    stride = _check_rows(out, "out", ck.shape, out.dtype if dtype is None else dtype, dev)
    st = lib.mesa_checkpoint_unpack(_ptr(ck.buffer), ck.rows, ck.width, stride, _float_code(out.dtype, "out"), _ptr(out),
                                    _stream(dev))
    if st != MESA_OK:
        raise MesaError(st, "mesa_checkpoint_unpack")
    return out


# ---------------------------------------------------------------- the gated recurrence
def _common_stride(x, r, i, shape, dtype, device):
    stride = _check_rows(x, "x", shape, dtype, device)
    if _check_rows(r, "r", shape, dtype, device) != stride or _check_rows(i, "i", shape, dtype, device) != stride:
        raise ValueError("x, r and i must have their rows equally spaced")
    return stride


def recurrence_workspace_bytes(batch, seq_len, width) -> int:
    return load().mesa_recurrence_workspace_bytes(batch, seq_len, width)


def recurrence(x, r, i, theta, decay=8.0, reset=None, h0=None, want_final=False, want_states=False,
               want_checkpoints=False, out=None, workspace=None):
    """mesa_recurrence: the gated linear recurrence over x, r, i [B,T,W] (fp32 or bf16, rows
    evenly spaced alike, e.g. slices of one projection), theta [W] fp32, reset [B,T] uint8 or
    None (a token that starts a document), h0 [B,W] fp32 or None.  Returns y [B,T,W] of x's
    dtype, or a dict with "y" and, if asked, "h" [B,W] fp32 (the state after the last token),
    "states" [B,ceil(T/128),W] fp32 (for recurrence_backward) and the checkpoints "x", "r", "i"
    of the inputs."""
    torch = _torch()
    lib = load()
    dev = _on_device(x, "x")
    B, T, W = x.shape
    f32 = torch.float32
    stride = _common_stride(x, r, i, (B, T, W), x.dtype, dev)
    code = _float_code(x.dtype, "x")
    _check(theta, "theta", (W,), f32, dev)
    if reset is not None:
        _check(reset, "reset", (B, T), torch.uint8, dev)
    if h0 is not None:
        _check(h0, "h0", (B, W), f32, dev)
    if out is None:
        out = torch.empty((B, T, W), dtype=x.dtype, device=dev)
    else:
        _check(out, "out", (B, T, W), x.dtype, dev)
    need = lib.mesa_recurrence_workspace_bytes(B, T, W)
    workspace = _workspace(workspace, need, dev)
    res = {"y": out}
    if want_final:
        res["h"] = torch.empty((B, W), dtype=f32, device=dev)
    if want_states:
        res["states"] = torch.empty((B, -(-T // MESA_RECURRENCE_BLOCK), W), dtype=f32, device=dev)
    kept = (None, None, None)
    if want_checkpoints:
        for n in ("x", "r", "i"):
            res[n] = Checkpoint.empty((B, T, W), dev)
        kept = tuple(res[n].buffer for n in ("x", "r", "i"))
    st = lib.mesa_recurrence(_ptr(x), _ptr(r), _ptr(i), _ptr(theta), float(decay), _ptr(reset), _ptr(h0), B, T, W, stride,
                             code, _ptr(out), _ptr(res.get("h")), _ptr(res.get("states")), _ptr(kept[0]), _ptr(kept[1]),
                             _ptr(kept[2]), _ptr(workspace), need, _stream(dev))
    if st != MESA_OK:
        raise MesaError(st, "mesa_recurrence")
    return res if len(res) > 1 else out


def recurrence_step(state, x, r, i, theta, decay=8.0, reset=None, state_out=None, out=None):
    """mesa_recurrence_step: one token of the recurrence.  state [B,W] fp32, updated in place
    unless state_out is given; x, r, i [B,W] fp32 or bf16 (rows evenly spaced alike); theta [W];
    reset [B] uint8 or None.  Returns y [B,W] of x's dtype."""
    torch = _torch()
    lib = load()
    dev = _on_device(x, "x")
    B, W = x.shape
    stride = _common_stride(x, r, i, (B, W), x.dtype, dev)
    _check_all(torch.float32, dev, (state, "state", (B, W)), (theta, "theta", (W,)))
    if reset is not None:
        _check(reset, "reset", (B,), torch.uint8, dev)
    if state_out is None:
        state_out = state
    elif state_out is not state:
        _check(state_out, "state_out", (B, W), torch.float32, dev)
    if out is None:
        out = torch.empty((B, W), dtype=x.dtype, device=dev)
    else:
        _check(out, "out", (B, W), x.dtype, dev)
    st = lib.mesa_recurrence_step(_ptr(state), _ptr(x), _ptr(r), _ptr(i), _ptr(theta), float(decay), _ptr(reset), B, W,
                                  stride, _float_code(x.dtype, "x"), _ptr(state_out), _ptr(out), _stream(dev))
    if st != MESA_OK:
        raise MesaError(st, "mesa_recurrence_step")
    return out


def recurrence_backward_workspace_bytes(batch, seq_len, width) -> int:
    return load().mesa_recurrence_backward_workspace_bytes(batch, seq_len, width)


def recurrence_backward(x, r, i, theta, states, dy, dfinal=None, decay=8.0, reset=None, out=None, workspace=None):
    """mesa_recurrence_backward: gradients of the recurrence.  x, r, i [B,T,W] as given to
    recurrence(), or the three Checkpoints it kept; states as it returned them; dy [B,T,W]
    fp32 or bf16; dfinal [B,W] fp32 or None (no gradient of the last state).  Returns a dict:
    "dx", "dr", "di" [B,T,W] of dy's dtype (out: three tensors to write them to, rows evenly
    spaced alike, e.g. slices of one gradient), "dtheta" [W] and "dh0" [B,W] fp32."""
    torch = _torch()
    lib = load()
    B, T, W = shape = tuple(x.shape)
    f32 = torch.float32
    if isinstance(x, Checkpoint):
        dev, code, stride = x.device, MESA_DTYPE_Q8, W
        for t, n in ((r, "r"), (i, "i")):
            if not isinstance(t, Checkpoint) or t.shape != shape or t.device != dev:
                raise TypeError("%s must be a Checkpoint of shape %s on %s, as x is" % (n, shape, dev))
        x, r, i = x.buffer, r.buffer, i.buffer
    else:
        dev = _on_device(x, "x")
        code = _float_code(x.dtype, "x")
        stride = _common_stride(x, r, i, shape, x.dtype, dev)
    _check_all(f32, dev, (theta, "theta", (W,)), (states, "states", (B, -(-T // MESA_RECURRENCE_BLOCK), W)))
    _check(dy, "dy", shape, device=dev)
    grad_code = _float_code(dy.dtype, "dy")
    if dfinal is not None:
        _check(dfinal, "dfinal", (B, W), f32, dev)
    if reset is not None:
        _check(reset, "reset", (B, T), torch.uint8, dev)
    if out is None:
        out = (torch.empty_like(dy), torch.empty_like(dy), torch.empty_like(dy))
        grad_stride = W
    else:
        grad_stride = _common_stride(*out, shape, dy.dtype, dev)
    need = lib.mesa_recurrence_backward_workspace_bytes(B, T, W)
    workspace = _workspace(workspace, need, dev)
    res = {"dx": out[0], "dr": out[1], "di": out[2], "dtheta": torch.empty_like(theta),
           "dh0": torch.empty((B, W), dtype=f32, device=dev)}
    st = lib.mesa_recurrence_backward(_ptr(x), _ptr(r), _ptr(i), _ptr(theta), float(decay), _ptr(reset), _ptr(states),
                                      _ptr(dy), _ptr(dfinal), B, T, W, stride, code, grad_code, grad_stride, _ptr(out[0]),
                                      _ptr(out[1]), _ptr(out[2]), _ptr(res["dtheta"]), _ptr(res["dh0"]), _ptr(workspace),
                                      need, _stream(dev))
    if st != MESA_OK:
        raise MesaError(st, "mesa_recurrence_backward")
    return res


# ---------------------------------------------------------------- gradients of the layer's ends
def _held(t, name, shape, dtype, device):
    """A tensor of shape and dtype, or a Checkpoint of that shape: the tensor behind it."""
    if isinstance(t, Checkpoint):
        if dtype is not None or t.shape != tuple(shape) or t.device != device:
            raise TypeError("%s must be held as the others are, with shape %s on %s" % (name, tuple(shape), device))
        return t.buffer
    if dtype is None:
        raise TypeError("%s must be a Checkpoint, as the others are" % name)
    _check(t, name, shape, dtype, device)
    return t


def frontend_backward_workspace_bytes(batch, heads, seq_len, d_k, d_v) -> int:
    return load().mesa_frontend_backward_workspace_bytes(batch, heads, seq_len, d_k, d_v)


def frontend_backward(qp, kp, vp, conv_q, conv_k, conv_v, a_gamma, a_beta, theta, dq, dk, dv, dgamma, dbeta, dlam,
                      gamma_cap=0.9975, l2_eps=1e-6, grad_dtype=None, workspace=None):
    """mesa_frontend_backward: gradients of frontend()'s inputs from those of its outputs (dq,
    dk [B,H,T,d_k], dv [B,H,T,d_v], dgamma, dbeta [B,H,T], dlam [H,d_k]: fp32, as backward()
    returns them).  qp, kp, vp as given to frontend(), or Checkpoints of them; without conv_v vp
    is not read and may be None.  Returns a dict:
    "dqp", "dkp" [B,T,H,d_k], "dvp" [B,T,H,d_v] of grad_dtype (the projections' dtype by default,
    bf16 for Checkpoints), "dconv_q", "dconv_k" [H*d_k,4], "dconv_v" [H*d_v,4] (with conv_v),
    "da_gamma", "da_beta" [B,T,H], "dtheta" [H,d_k] (fp32)."""
    torch = _torch()
    lib = load()
    B, T, H, dk_ = qp.shape
    if vp is None and conv_v is not None:
        raise TypeError("vp must be given with conv_v")
    dv_ = (dv if vp is None else vp).shape[-1]
    f32 = torch.float32
    q8 = isinstance(qp, Checkpoint)
    dev = qp.device if q8 else _on_device(qp, "qp")
    code = MESA_DTYPE_Q8 if q8 else _float_code(qp.dtype, "qp")
    dtype = None if q8 else qp.dtype
    if grad_dtype is None:
        grad_dtype = torch.bfloat16 if q8 else qp.dtype
    qp = _held(qp, "qp", (B, T, H, dk_), dtype, dev)
    kp = _held(kp, "kp", (B, T, H, dk_), dtype, dev)
    if vp is not None:
        vp = _held(vp, "vp", (B, T, H, dv_), dtype, dev)
    gates, outs = (B, T, H), (B, H, T)
    _check_all(f32, dev, (conv_q, "conv_q", (H * dk_, 4)), (conv_k, "conv_k", (H * dk_, 4)), (a_gamma, "a_gamma", gates),
               (a_beta, "a_beta", gates), (theta, "theta", (H, dk_)), (dq, "dq", (B, H, T, dk_)), (dk, "dk", (B, H, T, dk_)),
               (dv, "dv", (B, H, T, dv_)), (dgamma, "dgamma", outs), (dbeta, "dbeta", outs), (dlam, "dlam", (H, dk_)))
    if conv_v is not None:
        _check_all(f32, dev, (conv_v, "conv_v", (H * dv_, 4)))
    like = torch.empty_like     # quicker than torch.empty, and every gradient has its input's shape
    if q8 or vp is None:
        grads = [torch.empty(t, dtype=grad_dtype, device=dev) for t in ((B, T, H, dk_), (B, T, H, dk_), (B, T, H, dv_))]
    else:
        grads = [like(t, dtype=grad_dtype) for t in (qp, kp, vp)]
    res = {"dqp": grads[0], "dkp": grads[1], "dvp": grads[2], "dconv_q": like(conv_q), "dconv_k": like(conv_k)}
    if conv_v is not None:
        res["dconv_v"] = like(conv_v)
    res["da_gamma"], res["da_beta"], res["dtheta"] = like(a_gamma), like(a_beta), like(theta)
    need = lib.mesa_frontend_backward_workspace_bytes(B, H, T, dk_, dv_)
    workspace = _workspace(workspace, need, dev)
    st = lib.mesa_frontend_backward(_ptr(qp), _ptr(kp), _ptr(vp), _ptr(conv_q), _ptr(conv_k), _ptr(conv_v), _ptr(a_gamma),
                                    _ptr(a_beta), _ptr(theta), float(gamma_cap), float(l2_eps), B, H, T, dk_, dv_, code,
                                    _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dgamma), _ptr(dbeta), _ptr(dlam),
                                    _float_code(grad_dtype, "grad_dtype"), _ptr(res["dqp"]), _ptr(res["dkp"]),
                                    _ptr(res["dvp"]), _ptr(res["dconv_q"]), _ptr(res["dconv_k"]), _ptr(res.get("dconv_v")),
                                    _ptr(res["da_gamma"]), _ptr(res["da_beta"]), _ptr(res["dtheta"]), _ptr(workspace), need,
                                    _stream(dev))
    if st != MESA_OK:
        raise MesaError(st, "mesa_frontend_backward")
    return res


def output_norm_backward_workspace_bytes(batch, heads, seq_len, d_v) -> int:
    return load().mesa_output_norm_backward_workspace_bytes(batch, heads, seq_len, d_v)


def output_norm_backward(o, weight, dy, eps=1e-6, workspace=None):
    """mesa_output_norm_backward: gradients of output_norm() from dy [B,T,H,d_v] (fp32 or bf16).
    o [B,H,T,d_v] fp32 as given to it, or a Checkpoint of it; weight [H,d_v].  Returns a dict:
    "do" [B,H,T,d_v] (backward()'s dout) and "dweight" [H,d_v], fp32."""
    torch = _torch()
    lib = load()
    B, H, T, dv_ = o.shape
    f32 = torch.float32
    q8 = isinstance(o, Checkpoint)
    dev = o.device if q8 else _on_device(o, "o")
    o = _held(o, "o", (B, H, T, dv_), None if q8 else f32, dev)
    _check(weight, "weight", (H, dv_), f32, dev)
    _check(dy, "dy", (B, T, H, dv_), device=dev)
    res = {"do": torch.empty((B, H, T, dv_), dtype=f32, device=dev) if q8 else torch.empty_like(o),
           "dweight": torch.empty_like(weight)}
    need = lib.mesa_output_norm_backward_workspace_bytes(B, H, T, dv_)
    workspace = _workspace(workspace, need, dev)
    st = lib.mesa_output_norm_backward(_ptr(o), _ptr(weight), float(eps), _ptr(dy), B, H, T, dv_,
                                       MESA_DTYPE_Q8 if q8 else MESA_DTYPE_F32, _float_code(dy.dtype, "dy"), _ptr(res["do"]),
                                       _ptr(res["dweight"]), _ptr(workspace), need, _stream(dev))
    if st != MESA_OK:
        raise MesaError(st, "mesa_output_norm_backward")
    return res
