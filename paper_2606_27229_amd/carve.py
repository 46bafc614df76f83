"""Thin Python binding of libcarve (C ABI in include/carve.h).

Argument marshalling only: tensors are allocated with PyTorch on the GPU,
their device pointers and the current HIP stream are handed to the C entry
points, and every step of the layer runs in the HIP kernels.  There is no
fallback: if libcarve.so is missing or a tensor is not a contiguous GPU
tensor of the right dtype, the call raises.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcarve.so")

CARVE_F32, CARVE_BF16 = 0, 1
SYMBOLS = ("carve_chunk_fwd", "carve_chunk_bwd", "carve_chunk_fwd_gated", "carve_chunk_bwd_gated",
           "carve_chunk_fwd_sw", "carve_chunk_bwd_sw", "carve_chunk_fwd_act", "carve_chunk_bwd_act",
           "carve_rmsnorm_fwd", "carve_rmsnorm_bwd", "carve_rmsnorm_workspace_size", "carve_rmsnorm_bwd_noalloc",
           "carve_workspace_size", "carve_status_string", "carve_profile_events", "carve_bwd_wait_status",
           "carve_set_ready_wait_limit",
           "carve_gdr_chunk_fwd", "carve_gdr_chunk_bwd", "carve_gdr_step", "carve_gdr_chunk_count",
           "carve_gdr_workspace_size", "carve_block_norm_fwd", "carve_block_norm_bwd",
           "carve_block_norm_workspace_size", "carve_short_conv_fwd", "carve_short_conv_bwd", "carve_short_conv_step",
           "carve_short_conv_workspace_size", "carve_rotary", "carve_ssm_chunk_fwd", "carve_ssm_chunk_bwd",
           "carve_ssm_step", "carve_ssm_chunk_count", "carve_ssm_workspace_size")


class Dims(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int), ("T", ctypes.c_int), ("H", ctypes.c_int), ("Dk", ctypes.c_int),
                ("Dv", ctypes.c_int), ("R", ctypes.c_int), ("L", ctypes.c_int), ("dtype", ctypes.c_int)]


class GdrDims(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int) for n in ("B", "T", "N", "Hk", "Hv", "Dk", "Dv", "dtype")]
                + [("scale", ctypes.c_float)]
                + [(n, ctypes.c_longlong) for n in ("q_batch", "q_token", "q_head", "k_batch", "k_token", "k_head",
                                                    "v_batch", "v_token", "v_head")])


class BlockNormDims(ctypes.Structure):
    _fields_ = ([("rows", ctypes.c_longlong)] + [(n, ctypes.c_int) for n in ("N", "groups", "dtype", "gate_act")]
                + [("eps", ctypes.c_float), ("alpha", ctypes.c_float)]
                + [(n, ctypes.c_longlong) for n in ("y_stride", "gate_stride", "residual_stride")])


class ShortConvDims(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int) for n in ("B", "T", "N", "C", "W", "dtype", "activation")]
                + [(n, ctypes.c_longlong) for n in ("x_batch", "x_token")])


class RotaryDims(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int) for n in ("B", "T", "N", "Hq", "Hk", "D", "rot", "dtype", "interleaved")]
                + [("amplitude", ctypes.c_float)]
                + [(t + n, ctypes.c_longlong) for t in ("q_", "k_", "qo_", "ko_") for n in ("batch", "token", "head")])


class SsmDims(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int) for n in ("B", "T", "N", "G", "H", "P", "S", "dtype", "softplus")]
                + [(n, ctypes.c_longlong) for n in ("x_batch", "x_token", "x_head", "b_batch", "b_token", "b_group",
                                                    "c_batch", "c_token", "c_group", "dt_batch", "dt_token")])


class CarveError(RuntimeError):
    def __init__(self, fn, status, msg):
        super().__init__(f"{fn} failed with status {status}: {msg}")
        self.status = status


_lib = None


def load_library(path: str = LIB_PATH):
    """Load libcarve.so (no GPU needed).  Raises if it has not been built."""
    global _lib
    if _lib is not None and path == LIB_PATH:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} not found: build it with paper_2606_27229_amd.build.build()")
    lib = ctypes.CDLL(path)
    vp, fp, sz = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t
    D = ctypes.POINTER(Dims)
    lib.carve_workspace_size.argtypes = [D, ctypes.c_int]
    lib.carve_workspace_size.restype = sz
    lib.carve_status_string.argtypes = [ctypes.c_int]
    lib.carve_status_string.restype = ctypes.c_char_p
    lib.carve_chunk_fwd.argtypes = [D] + [vp] * 7 + [fp] * 5 + [vp, fp, fp, vp, sz, vp]
    lib.carve_chunk_fwd.restype = ctypes.c_int
    lib.carve_chunk_bwd.argtypes = [D] + [vp] * 7 + [fp] * 5 + [vp, fp] + [vp] * 12 + [vp, sz, vp]
    lib.carve_chunk_bwd.restype = ctypes.c_int
    lib.carve_chunk_fwd_gated.argtypes = [D] + [vp] * 5 + [fp] * 2 + [vp] * 2 + [fp] * 5 + [vp, fp, fp, vp, sz, vp]
    lib.carve_chunk_fwd_gated.restype = ctypes.c_int
    lib.carve_chunk_bwd_gated.argtypes = ([D] + [vp] * 5 + [fp] * 2 + [vp] * 2 + [fp] * 5 + [vp, fp]
                                          + [vp] * 5 + [fp] * 2 + [vp] * 2 + [fp] * 5 + [vp, sz, vp])
    lib.carve_chunk_bwd_gated.restype = ctypes.c_int
    lib.carve_chunk_fwd_sw.argtypes = [D] + [vp] * 4 + [fp, vp, fp, fp, vp, vp, fp, fp, fp, vp, fp, fp, vp, sz, vp]
    lib.carve_chunk_fwd_sw.restype = ctypes.c_int
    lib.carve_chunk_bwd_sw.argtypes = ([D] + [vp] * 4 + [fp, vp, fp, fp, vp, vp, fp, fp, fp, vp, fp]
                                       + [vp] * 4 + [fp, vp, fp, fp, vp, vp, fp, fp, fp, vp, sz, vp])
    lib.carve_chunk_bwd_sw.restype = ctypes.c_int
    lib.carve_chunk_fwd_act.argtypes = lib.carve_chunk_fwd.argtypes
    lib.carve_chunk_fwd_act.restype = ctypes.c_int
    lib.carve_chunk_bwd_act.argtypes = lib.carve_chunk_bwd.argtypes
    lib.carve_chunk_bwd_act.restype = ctypes.c_int
    lib.carve_rmsnorm_fwd.argtypes = [D, vp, fp, ctypes.c_float, vp, vp]
    lib.carve_rmsnorm_fwd.restype = ctypes.c_int
    lib.carve_rmsnorm_bwd.argtypes = [D, vp, fp, ctypes.c_float, vp, vp, fp, vp, sz, vp]
    lib.carve_rmsnorm_bwd.restype = ctypes.c_int
    lib.carve_rmsnorm_bwd_noalloc.argtypes = [D, vp, fp, ctypes.c_float, vp, vp, fp, vp]
    lib.carve_rmsnorm_bwd_noalloc.restype = ctypes.c_int
    lib.carve_rmsnorm_workspace_size.argtypes = [D]
    lib.carve_rmsnorm_workspace_size.restype = sz
    lib.carve_profile_events.argtypes = [ctypes.POINTER(ctypes.c_void_p), ctypes.c_int]
    lib.carve_profile_events.restype = ctypes.c_int
    lib.carve_bwd_wait_status.argtypes = [D, vp, vp, ctypes.POINTER(ctypes.c_int)]
    lib.carve_bwd_wait_status.restype = ctypes.c_int
    lib.carve_set_ready_wait_limit.argtypes = [ctypes.c_int]
    lib.carve_set_ready_wait_limit.restype = ctypes.c_int
    G, N = ctypes.POINTER(GdrDims), ctypes.POINTER(BlockNormDims)
    lib.carve_gdr_chunk_count.argtypes = [G]
    lib.carve_gdr_chunk_count.restype = sz
    lib.carve_gdr_workspace_size.argtypes = [G, ctypes.c_int]
    lib.carve_gdr_workspace_size.restype = sz
    lib.carve_gdr_chunk_fwd.argtypes = [G] + [vp] * 11 + [sz, vp]
    lib.carve_gdr_chunk_fwd.restype = ctypes.c_int
    lib.carve_gdr_chunk_bwd.argtypes = [G] + [vp] * 16 + [sz, vp]
    lib.carve_gdr_chunk_bwd.restype = ctypes.c_int
    lib.carve_gdr_step.argtypes = [G] + [vp] * 6 + [ctypes.c_int] + [vp] * 3
    lib.carve_gdr_step.restype = ctypes.c_int
    lib.carve_block_norm_fwd.argtypes = [N] + [vp] * 9
    lib.carve_block_norm_fwd.restype = ctypes.c_int
    lib.carve_block_norm_workspace_size.argtypes = [N]
    lib.carve_block_norm_workspace_size.restype = sz
    lib.carve_block_norm_bwd.argtypes = [N] + [vp] * 15 + [sz, vp]
    lib.carve_block_norm_bwd.restype = ctypes.c_int
    V, R, S = ctypes.POINTER(ShortConvDims), ctypes.POINTER(RotaryDims), ctypes.POINTER(SsmDims)
    lib.carve_short_conv_fwd.argtypes = [V] + [vp] * 8
    lib.carve_short_conv_bwd.argtypes = [V] + [vp] * 12 + [sz, vp]
    lib.carve_short_conv_step.argtypes = [V] + [vp] * 4 + [ctypes.c_int] + [vp] * 3
    lib.carve_short_conv_workspace_size.argtypes = [V]
    lib.carve_short_conv_workspace_size.restype = sz
    lib.carve_rotary.argtypes = [R] + [vp] * 6 + [ctypes.c_int] + [vp] * 3
    lib.carve_ssm_chunk_count.argtypes = [S]
    lib.carve_ssm_chunk_count.restype = sz
    lib.carve_ssm_workspace_size.argtypes = [S, ctypes.c_int]
    lib.carve_ssm_workspace_size.restype = sz
    lib.carve_ssm_chunk_fwd.argtypes = [S] + [vp] * 13 + [sz, vp]
    lib.carve_ssm_chunk_bwd.argtypes = [S] + [vp] * 20 + [sz, vp]
    lib.carve_ssm_step.argtypes = [S] + [vp] * 8 + [ctypes.c_int] + [vp] * 3
    for name in ("short_conv_fwd", "short_conv_bwd", "short_conv_step", "rotary", "ssm_chunk_fwd", "ssm_chunk_bwd", "ssm_step"):
        getattr(lib, "carve_" + name).restype = ctypes.c_int
    if path == LIB_PATH:
        _lib = lib
    return lib


def status_string(st: int) -> str:
    return load_library().carve_status_string(st).decode()


def profile_events(events) -> None:
    """Arm the next chunk_fwd / chunk_bwd call on this thread to record the
    given torch.cuda.Event objects at its kernel-launch boundaries (measurement
    only).  The events must already exist on the device (record each once)."""
    arr = (ctypes.c_void_p * len(events))(*[e.cuda_event for e in events])
    _check("carve_profile_events", load_library().carve_profile_events(arr, len(events)))


def bwd_wait_status(dims: Dims, workspace, stream=None) -> bool:
    """Whether an adjoint wave's bounded wait for a chunk record ran out in the
    last backward made with this workspace (synchronises the stream)."""
    out = ctypes.c_int(0)
    _check("carve_bwd_wait_status", load_library().carve_bwd_wait_status(
        ctypes.byref(dims), _ptr(workspace, "workspace"), _stream(stream), ctypes.byref(out)))
    return bool(out.value)


def set_ready_wait_limit(polls: int) -> int:
    """Test hook: the bound of the backward's record wait for calls on this
    thread (negative: the default).  Returns the previous bound."""
    return int(load_library().carve_set_ready_wait_limit(int(polls)))


def make_dims(B, T, H, Dk, Dv, R, L, dtype) -> Dims:
    return Dims(B, T, H, Dk, Dv, R, L, CARVE_BF16 if dtype == torch.bfloat16 else CARVE_F32)


def workspace_size(dims: Dims, backward: bool) -> int:
    return int(load_library().carve_workspace_size(ctypes.byref(dims), 1 if backward else 0))


def _ptr(t, name, dtype=None, shape=None):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t.data_ptr()


def _stream(stream):
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def _check(fn, st):
    if st != 0:
        raise CarveError(fn, st, status_string(st))


def chunk_fwd(q, k, v, beta, g, bx, wx, Ub, Uw, Vb, Vw, S0=None, *, L=64, want_chunks=True,
              want_state=True, out=None, stream=None, act=False):
    """Forward of the chunked CARVE layer.

    Shapes: q, k, bx, g [B,T,H,Dk]; v, wx [B,T,H,Dv]; beta [B,T,H]; Ub, Uw [R,Dv];
    Vb [Dk,R]; Vw [Dv,R]; S0 [B,H,Dv,Dk] or None.  Returns (o, S_T, S_chunks).
    ``out`` may hold preallocated {"o", "S_T", "S_chunks"} tensors.  act=True:
    q, k, v are the raw projections and the kernels apply SiLU (+ L2 norm for
    q, k) (carve_chunk_fwd_act).
    """
    lib = load_library()
    B, T, H, Dk = q.shape
    Dv = v.shape[-1]
    R = Ub.shape[0]
    dt = q.dtype
    f32 = torch.float32
    dims = make_dims(B, T, H, Dk, Dv, R, L, dt)
    out = dict(out or {})
    o = out.get("o")
    if o is None:
        o = torch.empty((B, T, H, Dv), dtype=dt, device=q.device)
    S_T = out.get("S_T") if "S_T" in out else (torch.empty((B, H, Dv, Dk), dtype=f32, device=q.device) if want_state else None)
    S_chunks = out.get("S_chunks") if "S_chunks" in out else (
        torch.empty((B, H, T // L, Dv, Dk), dtype=f32, device=q.device) if want_chunks else None)
    fn = "carve_chunk_fwd_act" if act else "carve_chunk_fwd"
    st = getattr(lib, fn)(
        ctypes.byref(dims), _ptr(q, "q", dt, (B, T, H, Dk)), _ptr(k, "k", dt, (B, T, H, Dk)),
        _ptr(v, "v", dt, (B, T, H, Dv)), _ptr(beta, "beta", dt, (B, T, H)), _ptr(g, "g", f32, (B, T, H, Dk)),
        _ptr(bx, "bx", dt, (B, T, H, Dk)), _ptr(wx, "wx", dt, (B, T, H, Dv)),
        _ptr(Ub, "Ub", f32, (R, Dv)), _ptr(Uw, "Uw", f32, (R, Dv)), _ptr(Vb, "Vb", f32, (Dk, R)),
        _ptr(Vw, "Vw", f32, (Dv, R)), _ptr(S0, "S0", f32, (B, H, Dv, Dk)),
        _ptr(o, "o", dt, (B, T, H, Dv)), _ptr(S_T, "S_T", f32), _ptr(S_chunks, "S_chunks", f32),
        None, 0, _stream(stream))
    _check(fn, st)
    return o, S_T, S_chunks


def chunk_bwd(q, k, v, beta, g, bx, wx, Ub, Uw, Vb, Vw, S_chunks, dO, dS_T=None, *, L=64,
              want_dS0=True, out=None, workspace=None, stream=None, act=False):
    """Backward of the chunked CARVE layer for loss <dO, o> + <dS_T, S_T>.

    Returns a dict with dq, dk, dv, dbeta, dg, dbx, dwx, dUb, dUw, dVb, dVw, dS0.
    act=True: the backward of chunk_fwd(act=True) (gradients of the raw q, k, v).
    """
    lib = load_library()
    B, T, H, Dk = q.shape
    Dv = v.shape[-1]
    R = Ub.shape[0]
    dt = q.dtype
    f32 = torch.float32
    dev = q.device
    dims = make_dims(B, T, H, Dk, Dv, R, L, dt)
    res = dict(out or {})
    spec = {"dq": ((B, T, H, Dk), dt), "dk": ((B, T, H, Dk), dt), "dv": ((B, T, H, Dv), dt),
            "dbeta": ((B, T, H), dt), "dg": ((B, T, H, Dk), f32), "dbx": ((B, T, H, Dk), dt),
            "dwx": ((B, T, H, Dv), dt), "dUb": ((R, Dv), f32), "dUw": ((R, Dv), f32),
            "dVb": ((Dk, R), f32), "dVw": ((Dv, R), f32)}
    if want_dS0:
        spec["dS0"] = ((B, H, Dv, Dk), f32)
    for name, (shape, dtype) in spec.items():
        if res.get(name) is None:
            res[name] = torch.empty(shape, dtype=dtype, device=dev)
    ws_bytes = workspace_size(dims, True)
    if workspace is None and ws_bytes:
        workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
    ws_ptr = _ptr(workspace, "workspace") if workspace is not None else None
    ws_len = workspace.numel() * workspace.element_size() if workspace is not None else 0
    fn = "carve_chunk_bwd_act" if act else "carve_chunk_bwd"
    st = getattr(lib, fn)(
        ctypes.byref(dims), _ptr(q, "q", dt, (B, T, H, Dk)), _ptr(k, "k", dt, (B, T, H, Dk)),
        _ptr(v, "v", dt, (B, T, H, Dv)), _ptr(beta, "beta", dt, (B, T, H)), _ptr(g, "g", f32, (B, T, H, Dk)),
        _ptr(bx, "bx", dt, (B, T, H, Dk)), _ptr(wx, "wx", dt, (B, T, H, Dv)),
        _ptr(Ub, "Ub", f32, (R, Dv)), _ptr(Uw, "Uw", f32, (R, Dv)), _ptr(Vb, "Vb", f32, (Dk, R)),
        _ptr(Vw, "Vw", f32, (Dv, R)), _ptr(S_chunks, "S_chunks", f32, (B, H, T // L, Dv, Dk)),
        _ptr(dO, "dO", dt, (B, T, H, Dv)), _ptr(dS_T, "dS_T", f32, (B, H, Dv, Dk)),
        *[_ptr(res[n], n) for n in ("dq", "dk", "dv", "dbeta", "dg", "dbx", "dwx", "dUb", "dUw", "dVb", "dVw")],
        _ptr(res.get("dS0"), "dS0"), ws_ptr, ws_len, _stream(stream))
    _check(fn, st)
    return res


def chunk_fwd_gated(q, k, v, beta, f, A, tau_f, bx, wx, Ub, Uw, Vb, Vw, S0=None, *, L=64,
                    want_chunks=True, want_state=True, out=None, stream=None):
    """Forward with the decay computed in the kernels from its raw logit f
    (g = -exp(A) softplus(f + tau_f)).  f [B,T,H,Dk] has the token dtype; A and
    tau_f are f32 [H,Dk].  Returns (o, S_T, S_chunks)."""
    lib = load_library()
    B, T, H, Dk = q.shape
    Dv = v.shape[-1]
    R = Ub.shape[0]
    dt = q.dtype
    f32 = torch.float32
    dims = make_dims(B, T, H, Dk, Dv, R, L, dt)
    out = dict(out or {})
    o = out.get("o")
    if o is None:
        o = torch.empty((B, T, H, Dv), dtype=dt, device=q.device)
    S_T = out.get("S_T") if "S_T" in out else (torch.empty((B, H, Dv, Dk), dtype=f32, device=q.device) if want_state else None)
    S_chunks = out.get("S_chunks") if "S_chunks" in out else (
        torch.empty((B, H, T // L, Dv, Dk), dtype=f32, device=q.device) if want_chunks else None)
    st = lib.carve_chunk_fwd_gated(
        ctypes.byref(dims), _ptr(q, "q", dt, (B, T, H, Dk)), _ptr(k, "k", dt, (B, T, H, Dk)),
        _ptr(v, "v", dt, (B, T, H, Dv)), _ptr(beta, "beta", dt, (B, T, H)), _ptr(f, "f", dt, (B, T, H, Dk)),
        _ptr(A, "A", f32, (H, Dk)), _ptr(tau_f, "tau_f", f32, (H, Dk)),
        _ptr(bx, "bx", dt, (B, T, H, Dk)), _ptr(wx, "wx", dt, (B, T, H, Dv)),
        _ptr(Ub, "Ub", f32, (R, Dv)), _ptr(Uw, "Uw", f32, (R, Dv)), _ptr(Vb, "Vb", f32, (Dk, R)),
        _ptr(Vw, "Vw", f32, (Dv, R)), _ptr(S0, "S0", f32, (B, H, Dv, Dk)),
        _ptr(o, "o", dt, (B, T, H, Dv)), _ptr(S_T, "S_T", f32), _ptr(S_chunks, "S_chunks", f32),
        None, 0, _stream(stream))
    _check("carve_chunk_fwd_gated", st)
    return o, S_T, S_chunks


def chunk_bwd_gated(q, k, v, beta, f, A, tau_f, bx, wx, Ub, Uw, Vb, Vw, S_chunks, dO, dS_T=None, *, L=64,
                    want_dS0=True, out=None, workspace=None, stream=None):
    """Backward of ``chunk_fwd_gated``: the gradients of ``chunk_bwd`` with dg
    replaced by df (token dtype), dA and dtau ([H,Dk] f32)."""
    lib = load_library()
    B, T, H, Dk = q.shape
    Dv = v.shape[-1]
    R = Ub.shape[0]
    dt = q.dtype
    f32 = torch.float32
    dev = q.device
    dims = make_dims(B, T, H, Dk, Dv, R, L, dt)
    res = dict(out or {})
    spec = {"dq": ((B, T, H, Dk), dt), "dk": ((B, T, H, Dk), dt), "dv": ((B, T, H, Dv), dt),
            "dbeta": ((B, T, H), dt), "df": ((B, T, H, Dk), dt), "dA": ((H, Dk), f32), "dtau": ((H, Dk), f32),
            "dbx": ((B, T, H, Dk), dt), "dwx": ((B, T, H, Dv), dt), "dUb": ((R, Dv), f32),
            "dUw": ((R, Dv), f32), "dVb": ((Dk, R), f32), "dVw": ((Dv, R), f32)}
    if want_dS0:
        spec["dS0"] = ((B, H, Dv, Dk), f32)
    for name, (shape, dtype) in spec.items():
        if res.get(name) is None:
            res[name] = torch.empty(shape, dtype=dtype, device=dev)
    ws_bytes = workspace_size(dims, True)
    if workspace is None and ws_bytes:
        workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
    ws_ptr = _ptr(workspace, "workspace") if workspace is not None else None
    ws_len = workspace.numel() * workspace.element_size() if workspace is not None else 0
    st = lib.carve_chunk_bwd_gated(
        ctypes.byref(dims), _ptr(q, "q", dt, (B, T, H, Dk)), _ptr(k, "k", dt, (B, T, H, Dk)),
        _ptr(v, "v", dt, (B, T, H, Dv)), _ptr(beta, "beta", dt, (B, T, H)), _ptr(f, "f", dt, (B, T, H, Dk)),
        _ptr(A, "A", f32, (H, Dk)), _ptr(tau_f, "tau_f", f32, (H, Dk)),
        _ptr(bx, "bx", dt, (B, T, H, Dk)), _ptr(wx, "wx", dt, (B, T, H, Dv)),
        _ptr(Ub, "Ub", f32, (R, Dv)), _ptr(Uw, "Uw", f32, (R, Dv)), _ptr(Vb, "Vb", f32, (Dk, R)),
        _ptr(Vw, "Vw", f32, (Dv, R)), _ptr(S_chunks, "S_chunks", f32, (B, H, T // L, Dv, Dk)),
        _ptr(dO, "dO", dt, (B, T, H, Dv)), _ptr(dS_T, "dS_T", f32, (B, H, Dv, Dk)),
        *[_ptr(res[n], n) for n in ("dq", "dk", "dv", "dbeta", "df", "dA", "dtau", "dbx", "dwx",
                                    "dUb", "dUw", "dVb", "dVw")],
        _ptr(res.get("dS0"), "dS0"), ws_ptr, ws_len, _stream(stream))
    _check("carve_chunk_bwd_gated", st)
    return res


def chunk_fwd_sw(q, k, v, beta, bx, wx, Ub, Vb, S0=None, *, g=None, f=None, A=None, tau_f=None, L=64,
                 want_chunks=True, want_state=True, out=None, stream=None):
    """Forward with the scalar write gate: wx [B,T,H] (one logit per token and
    head, w = sigmoid(wx) on every value channel), no Uw, Vw.  The decay is g
    (f32 [B,T,H,Dk]) or, with g=None, formed in the kernels from f, A, tau_f.
    Returns (o, S_T, S_chunks)."""
    lib = load_library()
    B, T, H, Dk = q.shape
    Dv = v.shape[-1]
    R = Ub.shape[0]
    dt = q.dtype
    f32 = torch.float32
    dims = make_dims(B, T, H, Dk, Dv, R, L, dt)
    out = dict(out or {})
    o = out.get("o")
    if o is None:
        o = torch.empty((B, T, H, Dv), dtype=dt, device=q.device)
    S_T = out.get("S_T") if "S_T" in out else (torch.empty((B, H, Dv, Dk), dtype=f32, device=q.device) if want_state else None)
    S_chunks = out.get("S_chunks") if "S_chunks" in out else (
        torch.empty((B, H, T // L, Dv, Dk), dtype=f32, device=q.device) if want_chunks else None)
    st = lib.carve_chunk_fwd_sw(
        ctypes.byref(dims), _ptr(q, "q", dt, (B, T, H, Dk)), _ptr(k, "k", dt, (B, T, H, Dk)),
        _ptr(v, "v", dt, (B, T, H, Dv)), _ptr(beta, "beta", dt, (B, T, H)), _ptr(g, "g", f32, (B, T, H, Dk)),
        _ptr(f, "f", dt, (B, T, H, Dk)), _ptr(A, "A", f32, (H, Dk)), _ptr(tau_f, "tau_f", f32, (H, Dk)),
        _ptr(bx, "bx", dt, (B, T, H, Dk)), _ptr(wx, "wx", dt, (B, T, H)),
        _ptr(Ub, "Ub", f32, (R, Dv)), _ptr(Vb, "Vb", f32, (Dk, R)), _ptr(S0, "S0", f32, (B, H, Dv, Dk)),
        _ptr(o, "o", dt, (B, T, H, Dv)), _ptr(S_T, "S_T", f32), _ptr(S_chunks, "S_chunks", f32),
        None, 0, _stream(stream))
    _check("carve_chunk_fwd_sw", st)
    return o, S_T, S_chunks


def chunk_bwd_sw(q, k, v, beta, bx, wx, Ub, Vb, S_chunks, dO, dS_T=None, *, g=None, f=None, A=None, tau_f=None,
                 L=64, want_dS0=True, out=None, workspace=None, stream=None):
    """Backward of ``chunk_fwd_sw``: dq, dk, dv, dbeta, dbx, dwx [B,T,H], dUb,
    dVb, dS0, and dg (g given) or df, dA, dtau (f given)."""
    lib = load_library()
    B, T, H, Dk = q.shape
    Dv = v.shape[-1]
    R = Ub.shape[0]
    dt = q.dtype
    f32 = torch.float32
    dev = q.device
    dims = make_dims(B, T, H, Dk, Dv, R, L, dt)
    res = dict(out or {})
    spec = {"dq": ((B, T, H, Dk), dt), "dk": ((B, T, H, Dk), dt), "dv": ((B, T, H, Dv), dt),
            "dbeta": ((B, T, H), dt), "dbx": ((B, T, H, Dk), dt), "dwx": ((B, T, H), dt),
            "dUb": ((R, Dv), f32), "dVb": ((Dk, R), f32)}
    if f is None:
        spec["dg"] = ((B, T, H, Dk), f32)
    else:
        spec.update({"df": ((B, T, H, Dk), dt), "dA": ((H, Dk), f32), "dtau": ((H, Dk), f32)})
    if want_dS0:
        spec["dS0"] = ((B, H, Dv, Dk), f32)
    for name, (shape, dtype) in spec.items():
        if res.get(name) is None:
            res[name] = torch.empty(shape, dtype=dtype, device=dev)
    ws_bytes = workspace_size(dims, True)
    if workspace is None and ws_bytes:
        workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
    ws_ptr = _ptr(workspace, "workspace") if workspace is not None else None
    ws_len = workspace.numel() * workspace.element_size() if workspace is not None else 0
    st = lib.carve_chunk_bwd_sw(
        ctypes.byref(dims), _ptr(q, "q", dt, (B, T, H, Dk)), _ptr(k, "k", dt, (B, T, H, Dk)),
        _ptr(v, "v", dt, (B, T, H, Dv)), _ptr(beta, "beta", dt, (B, T, H)), _ptr(g, "g", f32, (B, T, H, Dk)),
        _ptr(f, "f", dt, (B, T, H, Dk)), _ptr(A, "A", f32, (H, Dk)), _ptr(tau_f, "tau_f", f32, (H, Dk)),
        _ptr(bx, "bx", dt, (B, T, H, Dk)), _ptr(wx, "wx", dt, (B, T, H)),
        _ptr(Ub, "Ub", f32, (R, Dv)), _ptr(Vb, "Vb", f32, (Dk, R)),
        _ptr(S_chunks, "S_chunks", f32, (B, H, T // L, Dv, Dk)),
        _ptr(dO, "dO", dt, (B, T, H, Dv)), _ptr(dS_T, "dS_T", f32, (B, H, Dv, Dk)),
        *[_ptr(res.get(n), n) for n in ("dq", "dk", "dv", "dbeta", "dg", "df", "dA", "dtau", "dbx", "dwx",
                                        "dUb", "dVb", "dS0")],
        ws_ptr, ws_len, _stream(stream))
    _check("carve_chunk_bwd_sw", st)
    return res


RMSNORM_EPS = 1e-6


def _norm_dims(o):
    B, T, H, Dv = o.shape
    # only B, T, H, Dv and dtype are read by the norm entry points
    return make_dims(B, T, H, Dv, Dv, 1, 1, o.dtype)


def rmsnorm_fwd(o, weight, *, eps=RMSNORM_EPS, out=None, stream=None):
    """Output RMS normalisation of the layer output o [B,T,H,Dv] over each
    token's H*Dv values (Alg. carve_fwd's last step, without W_O):
    y = o / sqrt(mean(o^2) + eps) * weight, weight [H*Dv] f32."""
    lib = load_library()
    B, T, H, Dv = o.shape
    dims = _norm_dims(o)
    y = out if out is not None else torch.empty_like(o)
    st = lib.carve_rmsnorm_fwd(ctypes.byref(dims), _ptr(o, "o", o.dtype, (B, T, H, Dv)),
                               _ptr(weight, "weight", torch.float32, (H * Dv,)), float(eps),
                               _ptr(y, "y", o.dtype, (B, T, H, Dv)), _stream(stream))
    _check("carve_rmsnorm_fwd", st)
    return y


def rmsnorm_bwd(o, weight, dy, *, eps=RMSNORM_EPS, out=None, workspace=None, stream=None):
    """Backward of ``rmsnorm_fwd`` for loss <dy, y>: returns (d_o, dweight)."""
    lib = load_library()
    B, T, H, Dv = o.shape
    dims = _norm_dims(o)
    res = dict(out or {})
    d_o = res.get("d_o")
    if d_o is None:
        d_o = torch.empty_like(o)
    dw = res.get("dweight")
    if dw is None:
        dw = torch.empty((H * Dv,), dtype=torch.float32, device=o.device)
    ws_bytes = int(lib.carve_rmsnorm_workspace_size(ctypes.byref(dims)))
    if workspace is None:
        workspace = torch.empty(max(ws_bytes, 16), dtype=torch.uint8, device=o.device)
    ws_len = workspace.numel() * workspace.element_size()
    st = lib.carve_rmsnorm_bwd(ctypes.byref(dims), _ptr(o, "o", o.dtype, (B, T, H, Dv)),
                               _ptr(weight, "weight", torch.float32, (H * Dv,)), float(eps),
                               _ptr(dy, "dy", o.dtype, (B, T, H, Dv)), _ptr(d_o, "d_o", o.dtype, (B, T, H, Dv)),
                               _ptr(dw, "dweight", torch.float32, (H * Dv,)), _ptr(workspace, "workspace"),
                               ws_len, _stream(stream))
    _check("carve_rmsnorm_bwd", st)
    return d_o, dw


def rmsnorm_bwd_noalloc(o, weight, dy, d_o, dweight, *, eps=RMSNORM_EPS, stream=None):
    """``rmsnorm_bwd`` through the entry point that allocates nothing (its
    scratch is the library's static per-device array): the caller passes the
    outputs d_o (like o) and dweight ([H*Dv] f32)."""
    lib = load_library()
    B, T, H, Dv = o.shape
    dims = _norm_dims(o)
    st = lib.carve_rmsnorm_bwd_noalloc(ctypes.byref(dims), _ptr(o, "o", o.dtype, (B, T, H, Dv)),
                                       _ptr(weight, "weight", torch.float32, (H * Dv,)), float(eps),
                                       _ptr(dy, "dy", o.dtype, (B, T, H, Dv)),
                                       _ptr(d_o, "d_o", o.dtype, (B, T, H, Dv)),
                                       _ptr(dweight, "dweight", torch.float32, (H * Dv,)), _stream(stream))
    _check("carve_rmsnorm_bwd_noalloc", st)
    return d_o, dweight


# ---- the gated delta rule and the norms around a block ------------------------


def _same_device(device, **tensors):
    for name, t in tensors.items():
        if t is None:
            continue
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name} must be a GPU tensor")
        if t.device != device:
            raise ValueError(f"{name} is on {t.device}, expected {device}")


# the current stream's handle of a device (building a Stream object for it takes 2.5 us
# of a 10 us call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _on_stream(call, device, stream):
    """call(stream handle) with the tensors' device current and, with ``stream``
    given, that stream current too, so that what the call allocates belongs to it."""
    if stream is None and device.index == torch.cuda.current_device():
        return call(_raw_stream(device.index))
    if stream is None:
        stream = torch.cuda.current_stream(device)
    if stream.device != device:
        raise ValueError(f"stream is on {stream.device}, the tensors are on {device}")
    with torch.cuda.stream(stream):
        return call(stream.cuda_stream)


def _layout(t):
    """What the checks of a call look at."""
    return None if t is None else (t.shape, t.stride(), t.dtype, t.device)


# layouts that passed a call's checks, and what follows from them alone (the C dims,
# sizes): a call with the same layouts checks nothing else
_checked = {}


def _remember(key, value):
    if len(_checked) >= 512:
        _checked.clear()
    _checked[key] = value
    return value


def _dense_like(t):
    # (a third of the time of torch.empty with its named arguments)
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _out(res, name, like, shape, dtype, device):
    """The pointer of res[name], which is allocated if missing; like: a tensor of its
    shape and type, or None."""
    t = res.get(name)
    if t is not None:
        return _ptr(t, name, dtype, shape)
    res[name] = t = torch.empty(shape, dtype=dtype, device=device) if like is None else _dense_like(like)
    return t.data_ptr()


def _scratch(workspace, nbytes, device):
    if workspace is None:
        workspace = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=device)
    return workspace, _ptr(workspace, "workspace"), workspace.numel() * workspace.element_size()


@functools.lru_cache(maxsize=256)
def _gdr_dims(B, T, N, Hk, Hv, Dk, Dv, dtype, scale, *strides):
    """A reference to the C dims of a call (by sizes and strides alone), its chunk count
    and the workspace sizes of its forward and backward."""
    lib = load_library()
    d = GdrDims(B, T, N, Hk, Hv, Dk, Dv, CARVE_BF16 if dtype == torch.bfloat16 else CARVE_F32, scale, *strides)
    r = ctypes.byref(d)
    return r, int(lib.carve_gdr_chunk_count(r)), int(lib.carve_gdr_workspace_size(r, 0)), int(lib.carve_gdr_workspace_size(r, 1))


def _strides(t):
    # (a dimension of one element may have any stride; none is taken)
    return tuple(s if n > 1 else 0 for n, s in zip(t.shape[:3], t.stride()[:3]))


def _gdr_call(q, k, v, g, beta, scale, offsets):
    """Checks what every entry point takes; returns ((dims, chunks, workspace sizes),
    sequences, the pointers of q, k, v, g, beta)."""
    if scale is not None:
        scale = float(scale)
    try:
        key = ("gdr", scale, _layout(q), _layout(k), _layout(v), _layout(g), _layout(beta), _layout(offsets))
        hit = _checked.get(key)
    except AttributeError:   # (something else than tensors: named below)
        hit = None
    if hit is not None:
        return *hit, (q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr())
    for name, t, dims in (("q", q, 4), ("k", k, 4), ("v", v, 4), ("g", g, 3), ("beta", beta, 3)):
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise TypeError(f"{name} must be a GPU tensor")
        if t.dim() != dims:
            raise ValueError(f"{name} has {t.dim()} dimensions, expected {dims}")
    dt, device = q.dtype, q.device
    if dt not in (torch.bfloat16, torch.float32):
        raise TypeError(f"q must be bfloat16 or float32, got {dt}")
    B, T, Hk, Dk = q.shape
    Hv, Dv = v.shape[2:]
    for name, t, shape in (("k", k, (B, T, Hk, Dk)), ("v", v, (B, T, Hv, Dv))):
        if t.dtype != dt:
            raise TypeError(f"{name} must be {dt}, got {t.dtype}")
        if tuple(t.shape) != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {shape}")
    for name, t in (("q", q), ("k", k), ("v", v)):
        if t.stride(3) != 1 and t.shape[3] > 1:
            raise ValueError(f"{name} must be contiguous in its last dimension")
    _same_device(device, k=k, v=v, g=g, beta=beta, offsets=offsets)
    seqs = B
    if offsets is not None:
        if offsets.dim() != 1 or offsets.numel() < 2:
            raise ValueError("offsets must be one-dimensional, the number of sequences and one")
        seqs = offsets.numel() - 1
    if scale is None:
        scale = Dk ** -0.5
    dims = _gdr_dims(B, T, seqs if offsets is not None else 0, Hk, Hv, Dk, Dv, dt, scale, *_strides(q),
                     *_strides(k), *_strides(v))
    ptrs = (q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(g, "g", torch.float32, (B, T, Hv)),
            _ptr(beta, "beta", dt, (B, T, Hv)))
    return *_remember(key, (dims, seqs)), ptrs


def gdr_chunk_fwd(q, k, v, g, beta, S0=None, *, scale=None, offsets=None, want_chunks=True, want_state=True, out=None,
                  workspace=None, stream=None):
    """Forward of the gated delta rule with a scalar decay, in chunks of 64 tokens:

        S~ = e^g_t S;  u_t = beta_t (v_t - S~ k_t);  S = S~ + u_t k_t^T;  o_t = scale S q_t

    q, k [B,T,Hk,Dk], v [B,T,Hv,Dv] (last dimension contiguous, any strides that are
    multiples of 16 bytes), g [B,T,Hv] f32 (<= 0), beta [B,T,Hv]; value head h reads
    key head h // (Hv // Hk); S0 [B,Hv,Dv,Dk] f32 or None; scale: Dk**-0.5 if None.
    offsets (int32 [n + 1]): the T rows of B = 1 hold n packed sequences, rows
    offsets[i] to offsets[i + 1] each, and states are [n,Hv,Dv,Dk]; rows of no
    sequence are left as they were in a given ``out["o"]``.
    Returns (o, S_T, S_chunks); S_chunks is what ``gdr_chunk_bwd`` needs.  ``out`` may
    hold preallocated {"o", "S_T", "S_chunks"}.
    """
    lib = load_library()
    (dims, chunks, ws_bytes, _), seqs, ptrs = _gdr_call(q, k, v, g, beta, scale, offsets)
    B, T, Hv, Dv = v.shape
    Dk, dt, f32, dev = q.shape[3], q.dtype, torch.float32, q.device
    res = dict(out or {})
    _same_device(dev, S0=S0, workspace=workspace, **res)

    def call(s):
        o = _out(res, "o", v, (B, T, Hv, Dv), dt, dev)
        S_T = _out(res, "S_T", S0, (seqs, Hv, Dv, Dk), f32, dev) if want_state or res.get("S_T") is not None else None
        S_c = _out(res, "S_chunks", None, (chunks, Hv, Dv, Dk), f32, dev) if want_chunks or res.get("S_chunks") is not None else None
        ws, ws_ptr, ws_len = _scratch(workspace, ws_bytes, dev)
        return lib.carve_gdr_chunk_fwd(
            dims, *ptrs, _ptr(S0, "S0", f32, (seqs, Hv, Dv, Dk)), _ptr(offsets, "offsets", torch.int32),
            o, S_T, S_c, ws_ptr, ws_len, s)

    _check("carve_gdr_chunk_fwd", _on_stream(call, dev, stream))
    return res["o"], res.get("S_T"), res.get("S_chunks")


def gdr_chunk_bwd(q, k, v, g, beta, S_chunks, dO, dS_T=None, *, scale=None, offsets=None, want_dS0=True, out=None,
                  workspace=None, stream=None):
    """Backward of ``gdr_chunk_fwd`` for loss <dO, o> + <dS_T, S_T>: a dict with dq,
    dk, dv, dg (f32), dbeta and, with want_dS0, dS0.  dq and dk are sums over the
    value heads of a key head."""
    lib = load_library()
    (dims, chunks, _, ws_bytes), seqs, ptrs = _gdr_call(q, k, v, g, beta, scale, offsets)
    B, T, Hv, Dv = v.shape
    Dk, dt, f32, dev = q.shape[3], q.dtype, torch.float32, q.device
    res = dict(out or {})
    _same_device(dev, S_chunks=S_chunks, dO=dO, dS_T=dS_T, workspace=workspace, **res)

    def call(s):
        outs = [_out(res, name, like, like.shape, like.dtype, dev)
                for name, like in (("dq", q), ("dk", k), ("dv", v), ("dg", g), ("dbeta", beta))]
        dS0 = _out(res, "dS0", dS_T, (seqs, Hv, Dv, Dk), f32, dev) if want_dS0 or res.get("dS0") is not None else None
        ws, ws_ptr, ws_len = _scratch(workspace, ws_bytes, dev)
        return lib.carve_gdr_chunk_bwd(
            dims, *ptrs, _ptr(S_chunks, "S_chunks", f32, (chunks, Hv, Dv, Dk)),
            _ptr(offsets, "offsets", torch.int32), _ptr(dO, "dO", dt, (B, T, Hv, Dv)),
            _ptr(dS_T, "dS_T", f32, (seqs, Hv, Dv, Dk)), *outs, dS0, ws_ptr, ws_len, s)

    _check("carve_gdr_chunk_bwd", _on_stream(call, dev, stream))
    return res


def gdr_step(q, k, v, g, beta, state, slots=None, *, scale=None, out=None, stream=None):
    """The gated delta rule token by token, for decoding: T tokens (one, or several
    at once) for each of B sequences, whose states in the pool ``state``
    [pool,Hv,Dv,Dk] f32 are updated in place.  The state left is that behind the last
    token: to keep only some of T proposed ones, copy the states before the call
    (``state[slots]``), put them back and run the kept tokens again.  Sequence b's state is
    state[slots[b]] (int32 [B]), or state[b] without slots.  A slot outside the
    pool (-1) marks a padding entry, whose output rows are left as they were.  No
    slot may appear twice.  The other arguments are those of ``gdr_chunk_fwd``.
    Returns o [B,T,Hv,Dv] (``out`` if given)."""
    if scale is not None:
        scale = float(scale)
    try:
        key = ("step", scale, _layout(q), _layout(k), _layout(v), _layout(g), _layout(beta), _layout(state),
               _layout(slots), _layout(out))
        dims = _checked.get(key)
    except AttributeError:   # (something else than tensors: named below)
        key = dims = None
    if dims is None:
        (dims, *_), _, _ = _gdr_call(q, k, v, g, beta, scale, None)
        if not isinstance(state, torch.Tensor) or state.dim() != 4:
            raise ValueError("state must be [pool, Hv, Dv, Dk]")
        _ptr(slots, "slots", torch.int32, (v.shape[0],))
        _ptr(state, "state", torch.float32, (state.shape[0], v.shape[2], v.shape[3], q.shape[3]))
        _ptr(out, "out", q.dtype, v.shape)
        _same_device(q.device, state=state, slots=slots, out=out)
        _remember(key, dims)

    def call(s):
        o = _dense_like(v) if out is None else out
        return o, _lib.carve_gdr_step(
            dims, q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), beta.data_ptr(),
            None if slots is None else slots.data_ptr(), state.shape[0], state.data_ptr(), o.data_ptr(), s)

    o, st = _on_stream(call, q.device, stream)
    _check("carve_gdr_step", st)
    return o


GATE_ACTS = {"silu": 1, "sigmoid": 2}


@functools.lru_cache(maxsize=256)
def _block_norm_dims(rows, N, groups, dtype, act, eps, alpha, *strides):
    d = BlockNormDims(rows, N, groups, CARVE_BF16 if dtype == torch.bfloat16 else CARVE_F32, act, eps, alpha, *strides)
    r = ctypes.byref(d)
    return r, int(load_library().carve_block_norm_workspace_size(r))


def _rows(t, name, like=None):
    """t as [rows, N] without a copy, and its row stride."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if like is not None:
        if t.dtype != like.dtype:
            raise TypeError(f"{name} must be {like.dtype}, got {t.dtype}")
        if t.shape != like.shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(like.shape)}")
        if t.device != like.device:
            raise ValueError(f"{name} is on {t.device}, expected {like.device}")
    if t.dim() < 1 or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name} must be contiguous in its last dimension")
    if t.dim() != 2:
        try:
            t = t.view(-1, t.shape[-1]) if t.numel() else t.reshape(0, t.shape[-1])
        except RuntimeError:
            raise ValueError(f"{name}'s rows must have one stride") from None
    return t, (t.stride(0) if t.shape[0] > 1 else 0)


def _block_norm_call(y, weight, groups, gate, gate_act, residual, alpha, scale, next_weight, eps):
    groups, alpha, eps = int(groups), float(alpha), float(eps)
    try:
        key = ("norm", groups, gate_act, alpha, eps, _layout(y), _layout(weight), _layout(gate), _layout(residual),
               _layout(scale), _layout(next_weight))
        hit = _checked.get(key)
    except AttributeError:   # (something else than tensors: named below)
        hit = None
    if hit is not None:
        return *hit, tuple([None if t is None else t.data_ptr() for t in (y, weight, gate, residual, scale, next_weight)])
    yr, ys = _rows(y, "y")
    if y.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"y must be bfloat16 or float32, got {y.dtype}")
    if gate is not None and gate_act not in GATE_ACTS:
        raise ValueError(f"gate_act must be one of {sorted(GATE_ACTS)}, got {gate_act!r}")
    zr, zs = (None, 0) if gate is None else _rows(gate, "gate", y)
    rr, rs = (None, 0) if residual is None else _rows(residual, "residual", y)
    _same_device(y.device, weight=weight, scale=scale, next_weight=next_weight)
    rows, N = yr.shape
    dims, ws_bytes = _block_norm_dims(rows, N, groups, y.dtype, GATE_ACTS[gate_act] if gate is not None else 0,
                                      eps, alpha, ys, zs, rs)
    ptrs = (yr.data_ptr(), _ptr(weight, "weight", torch.float32, (N,)), None if gate is None else zr.data_ptr(),
            None if residual is None else rr.data_ptr(), _ptr(scale, "scale", torch.float32, (N,)),
            _ptr(next_weight, "next_weight", torch.float32, (N,)))
    if weight is None:
        raise TypeError("weight must be a GPU tensor")
    return *_remember(key, (dims, ws_bytes)), ptrs


def block_norm_fwd(y, weight, *, groups=1, gate=None, gate_act="silu", residual=None, alpha=1.0, scale=None,
                   next_weight=None, eps=RMSNORM_EPS, out=None, stream=None):
    """The norm after a block, its gate, its scaled addition to the residual stream
    and the norm before the next block, in one pass over rows y [..., N]:

        n = y / sqrt(mean(y^2) + eps) * weight      (mean over each of ``groups`` groups)
        x = alpha * residual + scale * n * act(gate),   act: "silu" or "sigmoid"
        h = x / sqrt(mean(x^2) + eps) * next_weight

    gate, residual (shape and dtype of y), scale, next_weight (f32 [N]) may be left
    out.  y, gate and residual may be slices of wider rows.  Returns (x, h), h None
    without next_weight.  ``out`` may hold preallocated {"x", "h"}."""
    dims, _, ptrs = _block_norm_call(y, weight, groups, gate, gate_act, residual, alpha, scale, next_weight, eps)
    x, h = (out.get("x"), out.get("h")) if out else (None, None)
    for name, t in (("x", x), ("h", h)):
        if t is not None:
            _ptr(t, name, y.dtype, y.shape)
            _same_device(y.device, **{name: t})

    def call(s):
        xo = _dense_like(y) if x is None else x
        ho = _dense_like(y) if h is None and next_weight is not None else h
        return xo, ho, _lib.carve_block_norm_fwd(dims, *ptrs, xo.data_ptr(), None if ho is None else ho.data_ptr(), s)

    x, h, st = _on_stream(call, y.device, stream)
    _check("carve_block_norm_fwd", st)
    return x, h


def block_norm_bwd(y, weight, dx, dh=None, *, groups=1, gate=None, gate_act="silu", residual=None, alpha=1.0, scale=None,
                   next_weight=None, eps=RMSNORM_EPS, out=None, workspace=None, stream=None):
    """Backward of ``block_norm_fwd`` for loss <dx, x> + <dh, h> (dx may be None where
    dh is given): a dict with dy, dweight and, for each input given, dgate,
    dresidual, dscale, dnext_weight."""
    lib = load_library()
    dims, ws_bytes, ptrs = _block_norm_call(y, weight, groups, gate, gate_act, residual, alpha, scale, next_weight, eps)
    res = dict(out or {})
    dev, shape = y.device, y.shape
    _same_device(dev, dx=dx, dh=dh, workspace=workspace, **res)
    wanted = (("dy", y), ("dgate", gate), ("dresidual", residual), ("dweight", weight), ("dscale", scale),
              ("dnext_weight", next_weight))

    def call(s):
        outs = [_out(res, name, of, of.shape, of.dtype, dev) if of is not None else _ptr(res.get(name), name)
                for name, of in wanted]
        ws, ws_ptr, ws_len = _scratch(workspace, ws_bytes, dev)
        return lib.carve_block_norm_bwd(dims, *ptrs, _ptr(dx, "dx", y.dtype, shape),
                                        _ptr(dh, "dh", y.dtype, shape), *outs, ws_ptr, ws_len, s)

    _check("carve_block_norm_bwd", _on_stream(call, dev, stream))
    return res


# ---- the short causal convolution, rotary positions and the selective state space scan --


def _pointer(t):
    return None if t is None else t.data_ptr()


def _gpu(t, name, dims, dtype=None, device=None):
    """Checks a required tensor by its number of dimensions, type and device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dim() != dims:
        raise ValueError(f"{name} has {t.dim()} dimensions, expected {dims}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")


def _tokens(t, name):
    if t.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"{name} must be bfloat16 or float32, got {t.dtype}")
    return CARVE_BF16 if t.dtype == torch.bfloat16 else CARVE_F32


def _last(t, name):
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name} must be contiguous in its last dimension")


def _count(offsets, B):
    """Sequences, and the N of the C dims."""
    if offsets is None:
        return B, 0
    if not isinstance(offsets, torch.Tensor):
        raise TypeError("offsets must be a GPU tensor")
    if offsets.dim() != 1 or offsets.numel() < 2:
        raise ValueError("offsets must be one-dimensional, the number of sequences and one")
    return offsets.numel() - 1, offsets.numel() - 1


def _steps(t, dims):
    # (a dimension of one element may have any stride; none is taken)
    return [t.stride(i) if t.shape[i] > 1 else 0 for i in range(dims)]


CONV_ACTS = {None: 0, "silu": 1}


def _conv_key(kind, x, weight, bias, past, offsets, activation):
    """The key of a call with these layouts, or None where something is no tensor."""
    try:
        return (kind, activation, _layout(x), _layout(weight), _layout(bias), _layout(past), _layout(offsets))
    except (AttributeError, TypeError):
        return None


def _conv_check(x, weight, bias, past, offsets, activation, past_name, pool=None):
    """Checks what every entry point takes; (reference to the C dims, sequences, workspace bytes)."""
    _gpu(x, "x", 3)
    dt = _tokens(x, "x")
    _last(x, "x")
    B, T, C = x.shape
    _gpu(weight, "weight", 2, torch.float32, x.device)
    W = weight.shape[1]
    _ptr(weight, "weight", torch.float32, (C, W))
    _same_device(x.device, bias=bias, offsets=offsets, **{past_name: past})
    _ptr(bias, "bias", torch.float32, (C,))
    _ptr(offsets, "offsets", torch.int32)
    if activation not in CONV_ACTS:
        raise ValueError(f"activation must be None or 'silu', got {activation!r}")
    seqs, N = _count(offsets, B)
    _ptr(past, past_name, x.dtype, (seqs if pool is None else pool, W - 1, C))
    d = ShortConvDims(B, T, N, C, W, dt, CONV_ACTS[activation], *_steps(x, 2))
    r = ctypes.byref(d)
    return r, seqs, int(load_library().carve_short_conv_workspace_size(r))


def short_conv_fwd(x, weight, x0=None, *, bias=None, activation="silu", offsets=None, want_state=True, out=None, stream=None):
    """The short causal convolution of every channel over its last W inputs:

        y_t = act(bias + sum_j weight[:, j] * x_{t-W+1+j}),   act: "silu" or None

    x [B,T,C] (channels contiguous; it may be a slice of wider rows), weight [C,W] and
    bias [C] f32, W 2 to 4; x0 [B,W-1,C] (x's dtype) or None: the inputs before the first
    row, oldest first.  offsets (int32 [n + 1]): the T rows of B = 1 hold n packed
    sequences, and x0 is [n,W-1,C]; rows of no sequence are left as they were in a given
    ``out["y"]``.  Returns (y, x_T), x_T the last W - 1 inputs.  ``out`` may hold
    preallocated {"y", "x_T"}."""
    lib = load_library()
    key = _conv_key("conv", x, weight, bias, x0, offsets, activation)
    hit = _checked.get(key) or _remember(key, _conv_check(x, weight, bias, x0, offsets, activation, "x0"))
    dims, seqs, _ = hit
    y, x_T = (out.get("y"), out.get("x_T")) if out else (None, None)
    kept = (seqs, weight.shape[1] - 1, x.shape[2])
    for name, t, shape in (("y", y, x.shape), ("x_T", x_T, kept)):
        if t is not None:
            _ptr(t, name, x.dtype, shape)
            _same_device(x.device, **{name: t})

    def call(s):
        yo = _dense_like(x) if y is None else y
        xo = torch.empty(kept, dtype=x.dtype, device=x.device) if x_T is None and want_state else x_T
        return yo, xo, lib.carve_short_conv_fwd(dims, x.data_ptr(), weight.data_ptr(), _pointer(bias), _pointer(x0),
                                                _pointer(offsets), yo.data_ptr(), _pointer(xo), s)

    y, x_T, st = _on_stream(call, x.device, stream)
    _check("carve_short_conv_fwd", st)
    return y, x_T


def short_conv_bwd(x, weight, dy, x0=None, dx_T=None, *, bias=None, activation="silu", offsets=None, want_dx0=None, out=None,
                   workspace=None, stream=None):
    """Backward of ``short_conv_fwd`` for loss <dy, y> + <dx_T, x_T>: a dict with dx,
    dweight (f32), dbias (where bias is given) and dx0 (want_dx0; by default where x0 is
    given)."""
    lib = load_library()
    key = _conv_key("conv", x, weight, bias, x0, offsets, activation)
    hit = _checked.get(key) or _remember(key, _conv_check(x, weight, bias, x0, offsets, activation, "x0"))
    dims, seqs, ws_bytes = hit
    res = dict(out or {})
    dev, kept = x.device, (seqs, weight.shape[1] - 1, x.shape[2])
    _same_device(dev, dy=dy, dx_T=dx_T, workspace=workspace, **res)
    _ptr(dy, "dy", x.dtype, x.shape)
    _ptr(dx_T, "dx_T", x.dtype, kept)
    want = (x0 is not None if want_dx0 is None else want_dx0) or res.get("dx0") is not None

    def call(s):
        dx = _out(res, "dx", x, x.shape, x.dtype, dev)
        dw = _out(res, "dweight", weight, weight.shape, torch.float32, dev)
        db = _out(res, "dbias", bias, bias.shape, torch.float32, dev) if bias is not None else _ptr(res.get("dbias"), "dbias")
        d0 = _out(res, "dx0", x0, kept, x.dtype, dev) if want else None
        ws, ws_ptr, ws_len = _scratch(workspace, ws_bytes, dev)
        return lib.carve_short_conv_bwd(dims, x.data_ptr(), weight.data_ptr(), _pointer(bias), _pointer(x0), _pointer(offsets),
                                        _pointer(dy), _pointer(dx_T), dx, dw, db, d0, ws_ptr, ws_len, s)

    _check("carve_short_conv_bwd", _on_stream(call, dev, stream))
    return res


def short_conv_step(x, weight, state, slots=None, *, bias=None, activation="silu", out=None, stream=None):
    """The short convolution for decoding: T tokens (x [B,T,C]) for each of B sequences,
    whose last inputs in the pool ``state`` [pool,W-1,C] (x's dtype) are updated in place.
    slots as in ``gdr_step``: a slot outside the pool (-1) marks a padding entry, whose
    output rows are left as they were, and no slot may appear twice.  Returns y ("out" if given)."""
    key = _conv_key("conv_step", x, weight, bias, state, slots, activation)
    key = None if key is None else key + (_layout(out) if isinstance(out, torch.Tensor) else out,)
    try:
        hit = _checked.get(key)
    except TypeError:   # (something else than tensors: named below)
        hit = None
    if hit is None:
        load_library()
        if not isinstance(state, torch.Tensor) or state.dim() != 3:
            raise ValueError("state must be [pool, W - 1, C]")
        hit = _conv_check(x, weight, bias, state, None, activation, "state", pool=state.shape[0])
        _ptr(slots, "slots", torch.int32, (x.shape[0],))
        _ptr(out, "out", x.dtype, x.shape)
        _same_device(x.device, slots=slots, out=out)
        _remember(key, hit)

    def call(s):
        y = _dense_like(x) if out is None else out
        return y, _lib.carve_short_conv_step(hit[0], x.data_ptr(), weight.data_ptr(), _pointer(bias), _pointer(slots),
                                             state.shape[0], state.data_ptr(), y.data_ptr(), s)

    y, st = _on_stream(call, x.device, stream)
    _check("carve_short_conv_step", st)
    return y


def rotary_frequencies(rot, base=10000.0, *, stretch=1.0, low=None, high=None, length=None, device="cuda"):
    """Angles a position of the rot / 2 pairs, base^(-2 i / rot), in 64 bits, as
    ``rotary_fwd`` takes them.  stretch: a context ``stretch`` times as long as trained;
    all frequencies are divided by it, or, with length (of the trained context), low and
    high: those that turn less than ``low`` times in it, none that turn more than ``high``
    times, and those between by a part that is linear in their turns."""
    if rot <= 0 or rot % 2:
        raise ValueError(f"rot must be a positive even number, got {rot}")
    if (low is None) != (high is None) or (low is None) != (length is None):
        raise ValueError("low, high and length are given together")
    freq = torch.tensor(float(base), dtype=torch.float64) ** (torch.arange(rot // 2, dtype=torch.float64) * (-2.0 / rot))
    part = torch.ones_like(freq)
    if low is not None:
        if not low < high:
            raise ValueError(f"low must be below high, got {low} and {high}")
        turns = freq * (float(length) / 6.283185307179586)
        part = 1 - ((turns - low) / (high - low)).clamp(0, 1)
    return (freq * (1 - part) + freq / float(stretch) * part).to(device)


def _rotary(q, k, freq, positions, start, offsets, interleaved, amplitude, out, stream, backward, names):
    lib = load_library()
    amplitude, interleaved = float(amplitude), bool(interleaved)
    oq, ok = (out.get("q"), out.get("k")) if out else (None, None)
    try:
        key = ("rotary", interleaved, amplitude, _layout(q), _layout(k), _layout(freq), _layout(positions), _layout(start),
               _layout(offsets), _layout(oq), _layout(ok))
        dims = _checked.get(key)
    except AttributeError:   # (something else than tensors: named below)
        key = dims = None
    if dims is None:
        _gpu(q, names[0], 4)
        dt, dev = _tokens(q, names[0]), q.device
        B, T, Hq, D = q.shape
        if k is not None:
            _gpu(k, names[1], 4, q.dtype, dev)
            if k.shape[:2] != q.shape[:2] or k.shape[3] != D:
                raise ValueError(f"{names[1]} has shape {tuple(k.shape)}, expected {(B, T, 'heads', D)}")
        elif ok is not None:
            raise ValueError(f"out holds k, {names[1]} is not given")
        _gpu(freq, "freq", 1, torch.float64, dev)
        _same_device(dev, positions=positions, start=start, offsets=offsets, freq=freq, **{"out q": oq, "out k": ok})
        seqs, N = _count(offsets, B)
        _ptr(freq, "freq")
        _ptr(positions, "positions", torch.int32, (B, T))
        _ptr(start, "start", torch.int32, (seqs,))
        _ptr(offsets, "offsets", torch.int32)
        strides = []
        for name, t, like in ((names[0], q, None), (names[1], k, None), ("out q", oq, q), ("out k", ok, k)):
            if t is None:
                # (a new tensor: dense)
                n, d = (0, 0) if like is None else like.shape[2:]
                strides += [T * n * d if B > 1 else 0, n * d if T > 1 else 0, d if n > 1 else 0]
                continue
            if like is not None and (t.dtype != like.dtype or t.shape != like.shape):
                raise ValueError(f"{name} must be {tuple(like.shape)} of {like.dtype}")
            _last(t, name)
            strides += _steps(t, 3)
        d = RotaryDims(B, T, N, Hq, 0 if k is None else k.shape[2], D, 2 * freq.numel(), dt, interleaved, amplitude, *strides)
        dims = ctypes.byref(d)
        _remember(key, dims)

    def call(s):
        qo = _dense_like(q) if oq is None else oq
        ko = _dense_like(k) if ok is None and k is not None else ok
        return qo, ko, lib.carve_rotary(dims, q.data_ptr(), _pointer(k), freq.data_ptr(), _pointer(positions), _pointer(start),
                                        _pointer(offsets), backward, qo.data_ptr(), _pointer(ko), s)

    qo, ko, st = _on_stream(call, q.device, stream)
    _check("carve_rotary", st)
    return qo, ko


def rotary_fwd(q, k, freq, *, positions=None, start=None, offsets=None, interleaved=False, amplitude=1.0, out=None, stream=None):
    """Rotary positions of q [B,T,Hq,D] and k [B,T,Hk,D] (k may be None): the pairs of the
    first rot = 2 len(freq) values of every head are turned by position * freq (f64
    [rot / 2], see ``rotary_frequencies``) and multiplied by ``amplitude``; the others are
    kept.  Pairs are values i and i + rot / 2, or with interleaved 2 i and 2 i + 1.

    A row's position is positions[b, t] (int32 [B,T]), or start (int32 [sequences], 0 if
    None) plus its row in its sequence; offsets (int32 [n + 1]) as in ``gdr_chunk_fwd``.
    Returns (q, k) turned.  ``out`` may hold {"q", "k"} to write to, strided or q and k
    themselves (in place)."""
    return _rotary(q, k, freq, positions, start, offsets, interleaved, amplitude, out, stream, 0, ("q", "k"))


def rotary_bwd(dq, dk, freq, *, positions=None, start=None, offsets=None, interleaved=False, amplitude=1.0, out=None, stream=None):
    """Backward of ``rotary_fwd``: from the gradients of its outputs to those of q and k
    (turned the other way).  ``out`` {"q", "k"} as there."""
    return _rotary(dq, dk, freq, positions, start, offsets, interleaved, amplitude, out, stream, 1, ("dq", "dk"))


def _ssm_call(x, dt, A, Bm, Cm, D, dt_bias, softplus, offsets):
    """Checks what every entry point takes; returns (dims, chunks, workspace bytes of
    forward and backward, sequences, the pointers of x, dt, A, Bm, Cm, D, dt_bias)."""
    softplus = bool(softplus)   # (a tensor is read at every call)
    try:
        key = ("ssm", softplus, _layout(x), _layout(dt), _layout(A), _layout(Bm), _layout(Cm), _layout(D), _layout(dt_bias),
               _layout(offsets))
        hit = _checked.get(key)
    except (AttributeError, TypeError):   # (something else than tensors: named below)
        key = hit = None
    if hit is None:
        lib = load_library()
        _gpu(x, "x", 4)
        code, dev = _tokens(x, "x"), x.device
        B, T, H, P = x.shape
        _gpu(dt, "dt", 3, x.dtype, dev)
        if tuple(dt.shape) != (B, T, H):
            raise ValueError(f"dt has shape {tuple(dt.shape)}, expected {(B, T, H)}")
        for name, t in (("Bm", Bm), ("Cm", Cm)):
            _gpu(t, name, 4, x.dtype, dev)
            if t.shape[:2] != x.shape[:2] or t.shape != Bm.shape:
                raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {(B, T, 'groups', 'state')}")
        for name, t in (("x", x), ("dt", dt), ("Bm", Bm), ("Cm", Cm)):
            _last(t, name)
        _gpu(A, "A", 1, torch.float32, dev)
        _same_device(dev, D=D, dt_bias=dt_bias, offsets=offsets)
        for name, t in (("A", A), ("D", D), ("dt_bias", dt_bias)):
            _ptr(t, name, torch.float32, (H,))
        _ptr(offsets, "offsets", torch.int32)
        seqs, N = _count(offsets, B)
        d = SsmDims(B, T, N, Bm.shape[2], H, P, Bm.shape[3], code, softplus, *_steps(x, 3), *_steps(Bm, 3), *_steps(Cm, 3),
                    *_steps(dt, 2))
        r = ctypes.byref(d)
        hit = _remember(key, (r, int(lib.carve_ssm_chunk_count(r)), int(lib.carve_ssm_workspace_size(r, 0)),
                              int(lib.carve_ssm_workspace_size(r, 1)), seqs))
    return *hit, (x.data_ptr(), dt.data_ptr(), A.data_ptr(), Bm.data_ptr(), Cm.data_ptr(), _pointer(D), _pointer(dt_bias))


def ssm_chunk_fwd(x, dt, A, Bm, Cm, S0=None, *, D=None, dt_bias=None, softplus=True, offsets=None, want_chunks=True,
                  want_state=True, out=None, workspace=None, stream=None):
    """Forward of the selective state space scan with a matrix state a head, in chunks of
    64 tokens:

        d_t = softplus(dt_t + dt_bias);  S = e^(d_t A) S + d_t x_t B_t^T;  y_t = S C_t + D x_t

    x [B,T,H,P], Bm, Cm [B,T,G,N] (last dimension contiguous, any strides that are
    multiples of 16 bytes), dt [B,T,H]; A (<= 0), D, dt_bias f32 [H], D and dt_bias may be
    None; head h reads group h // (H // G) of Bm and Cm; S0 [B,H,P,N] f32 or None.
    softplus=False: d_t = dt_t + dt_bias.  offsets (int32 [n + 1]): packed sequences as in
    ``gdr_chunk_fwd``.  Returns (y, S_T, S_chunks); S_chunks is what ``ssm_chunk_bwd``
    needs.  ``out`` may hold preallocated {"y", "S_T", "S_chunks"}."""
    lib = load_library()
    dims, chunks, ws_bytes, _, seqs, ptrs = _ssm_call(x, dt, A, Bm, Cm, D, dt_bias, softplus, offsets)
    H, P, N, f32, dev = x.shape[2], x.shape[3], Bm.shape[3], torch.float32, x.device
    res = dict(out or {})
    _same_device(dev, S0=S0, workspace=workspace, **res)

    def call(s):
        y = _out(res, "y", x, x.shape, x.dtype, dev)
        S_T = _out(res, "S_T", S0, (seqs, H, P, N), f32, dev) if want_state or res.get("S_T") is not None else None
        S_c = _out(res, "S_chunks", None, (chunks, H, P, N), f32, dev) if want_chunks or res.get("S_chunks") is not None else None
        ws, ws_ptr, ws_len = _scratch(workspace, ws_bytes, dev)
        return lib.carve_ssm_chunk_fwd(dims, *ptrs, _ptr(S0, "S0", f32, (seqs, H, P, N)), _pointer(offsets), y, S_T, S_c,
                                       ws_ptr, ws_len, s)

    _check("carve_ssm_chunk_fwd", _on_stream(call, dev, stream))
    return res["y"], res.get("S_T"), res.get("S_chunks")


def ssm_chunk_bwd(x, dt, A, Bm, Cm, S_chunks, dy, dS_T=None, *, D=None, dt_bias=None, softplus=True, offsets=None,
                  want_dS0=True, out=None, workspace=None, stream=None):
    """Backward of ``ssm_chunk_fwd`` for loss <dy, y> + <dS_T, S_T>: a dict with dx, ddt, dA
    (f32), dBm, dCm and, where they are given, dD, ddt_bias (f32), and with want_dS0 dS0.
    dBm and dCm are sums over the heads of a group."""
    lib = load_library()
    dims, chunks, _, ws_bytes, seqs, ptrs = _ssm_call(x, dt, A, Bm, Cm, D, dt_bias, softplus, offsets)
    H, P, N, f32, dev = x.shape[2], x.shape[3], Bm.shape[3], torch.float32, x.device
    res = dict(out or {})
    _same_device(dev, S_chunks=S_chunks, dy=dy, dS_T=dS_T, workspace=workspace, **res)

    def call(s):
        o = {name: _out(res, name, like, like.shape, like.dtype, dev) if like is not None else _ptr(res.get(name), name)
             for name, like in (("dx", x), ("ddt", dt), ("dA", A), ("dBm", Bm), ("dCm", Cm), ("dD", D), ("ddt_bias", dt_bias))}
        dS0 = _out(res, "dS0", dS_T, (seqs, H, P, N), f32, dev) if want_dS0 or res.get("dS0") is not None else None
        ws, ws_ptr, ws_len = _scratch(workspace, ws_bytes, dev)
        return lib.carve_ssm_chunk_bwd(dims, *ptrs, _ptr(S_chunks, "S_chunks", f32, (chunks, H, P, N)), _pointer(offsets),
                                       _ptr(dy, "dy", x.dtype, x.shape), _ptr(dS_T, "dS_T", f32, (seqs, H, P, N)),
                                       *o.values(), dS0, ws_ptr, ws_len, s)

    _check("carve_ssm_chunk_bwd", _on_stream(call, dev, stream))
    return res


def ssm_step(x, dt, A, Bm, Cm, state, slots=None, *, D=None, dt_bias=None, softplus=True, out=None, stream=None):
    """The scan token by token, for decoding: T tokens (one, or several at once) for each
    of B sequences, whose states in the pool ``state`` [pool,H,P,N] f32 are updated in
    place; slots as in ``gdr_step``.  The other arguments are those of ``ssm_chunk_fwd``.
    Returns y [B,T,H,P] (``out`` if given)."""
    softplus = bool(softplus)
    try:
        key = ("ssm_step", softplus, _layout(x), _layout(dt), _layout(A), _layout(Bm), _layout(Cm), _layout(D), _layout(dt_bias),
               _layout(state), _layout(slots), _layout(out))
        dims = _checked.get(key)
    except (AttributeError, TypeError):   # (something else than tensors: named below)
        key = dims = None
    if dims is None:
        dims, *_ = _ssm_call(x, dt, A, Bm, Cm, D, dt_bias, softplus, None)
        if not isinstance(state, torch.Tensor) or state.dim() != 4:
            raise ValueError("state must be [pool, H, P, N]")
        _ptr(slots, "slots", torch.int32, (x.shape[0],))
        _ptr(state, "state", torch.float32, (state.shape[0], x.shape[2], x.shape[3], Bm.shape[3]))
        _ptr(out, "out", x.dtype, x.shape)
        _same_device(x.device, state=state, slots=slots, out=out)
        _remember(key, dims)

    def call(s):
        y = _dense_like(x) if out is None else out
        return y, _lib.carve_ssm_step(dims, x.data_ptr(), dt.data_ptr(), A.data_ptr(), Bm.data_ptr(), Cm.data_ptr(), _pointer(D),
                                      _pointer(dt_bias), _pointer(slots), state.shape[0], state.data_ptr(), y.data_ptr(), s)

    y, st = _on_stream(call, x.device, stream)
    _check("carve_ssm_step", st)
    return y
