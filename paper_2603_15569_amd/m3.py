"""Python binding of libm3 (ctypes): argument marshalling only.

Every step of the path runs in the HIP kernels behind the C ABI declared in
include/m3.h; PyTorch supplies device memory and the current HIP stream.  A call
given another `stream` behaves as under torch.cuda.stream(stream): what it
allocates belongs to that stream, and the inputs have to be ready there.
There is no fallback: when libm3.so is missing or a call fails, an exception
is raised.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libm3.so")

M3_OK, M3_ERR_NULL, M3_ERR_SHAPE, M3_ERR_DTYPE = 0, 1, 2, 3
M3_ERR_UNSUPPORTED, M3_ERR_ALIGN, M3_ERR_WORKSPACE, M3_ERR_HIP = 4, 5, 6, 7
M3_F32, M3_BF16 = 0, 1
M3_SCAN_SPLIT, M3_SCAN_PER_CHUNK, M3_THETA_PER_HEAD = 1, 2, 4
_IO = {torch.float32: M3_F32, torch.bfloat16: M3_BF16}


class M3Dims(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("seqlen", ctypes.c_int64),
                ("nheads", ctypes.c_int64), ("headdim", ctypes.c_int64),
                ("dstate", ctypes.c_int64), ("rank", ctypes.c_int64),
                ("chunk", ctypes.c_int64), ("io", ctypes.c_int32),
                ("flags", ctypes.c_int32), ("a_stride_b", ctypes.c_int64),
                ("a_stride_t", ctypes.c_int64), ("a_stride_h", ctypes.c_int64),
                ("seg_chunks", ctypes.c_int64)]


class M3Prologue(ctypes.Structure):
    """m3_prologue: the block prologue fused into the kernels' input loads,
    and the optional output norm fused into the y store."""
    _fields_ = [("bc_norm", ctypes.c_int32), ("eps", ctypes.c_float),
                ("norm_B", ctypes.c_void_p), ("norm_C", ctypes.c_void_p),
                ("bias_B", ctypes.c_void_p), ("bias_C", ctypes.c_void_p),
                ("w_x", ctypes.c_void_p), ("w_z", ctypes.c_void_p),
                ("out_norm", ctypes.c_int32), ("out_group", ctypes.c_int32),
                ("out_eps", ctypes.c_float), ("out_gain", ctypes.c_void_p)]


M3_OUT_NORM_NONE, M3_OUT_NORM_PRE_GATE, M3_OUT_NORM_POST_GATE = 0, 1, 2


class M3GlrDims(ctypes.Structure):
    """m3_glr_dims: sizes, io dtype and element strides of the gated linear recurrence."""
    _fields_ = ([(n, ctypes.c_int64) for n in ("batch", "seqlen", "width")]
                + [("io", ctypes.c_int32), ("flags", ctypes.c_int32)]
                + [(f"{t}_stride_{a}", ctypes.c_int64) for t in "xriz" for a in "bt"])


class M3FfnDims(ctypes.Structure):
    """m3_ffn_dims: sizes, io dtype, activation and row strides of the feed-forward block."""
    _fields_ = [("tokens", ctypes.c_int64), ("dmodel", ctypes.c_int64), ("dff", ctypes.c_int64),
                ("io", ctypes.c_int32), ("act", ctypes.c_int32), ("x_stride", ctypes.c_int64),
                ("dy_stride", ctypes.c_int64)]


_ACT = {"silu": 0, "gelu": 1}   # M3_ACT_*
GLR_CHUNK = 128             # M3_GLR_CHUNK: tokens between two saved states
M3_ADAMW_8BIT = 1


class M3AdamwTensor(ctypes.Structure):
    """m3_adamw_tensor: one tensor of the optimizer's table."""
    _fields_ = [("p", ctypes.c_void_p), ("g", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("low", ctypes.c_void_p), ("scales", ctypes.c_void_p),
                ("n", ctypes.c_int64), ("decay", ctypes.c_double)]


class M3AdamwConfig(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", ctypes.c_int64), ("seed", ctypes.c_uint64),
                ("device_step", ctypes.c_void_p), ("device_lr", ctypes.c_void_p)]


class M3AdamwPlan(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("groups", ctypes.c_int64), ("bytes", ctypes.c_size_t),
                ("grad_dtype", ctypes.c_int32), ("flags", ctypes.c_int32)]


class M3Error(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"libm3 status {status}: {msg}")
        self.status = status


EXPORTS = ("m3_scan_workspace_bytes", "m3_scan_fwd", "m3_scan_fwd_gated", "m3_scan_fwd_varlen",
           "m3_scan_varlen_workspace_bytes", "m3_scan_varlen_check",
           "m3_step", "m3_step_gated", "m3_scan_check", "m3_set_wait_limit", "m3_scan_fwd_noalloc",
           "m3_scan_fwd_pro", "m3_step_pro", "m3_scan_bwd", "m3_scan_bwd_workspace_bytes",
           "m3_glr_workspace_bytes", "m3_glr_fwd", "m3_glr_bwd", "m3_glr_step", "m3_glr_check",
           "m3_ffn_workspace_bytes", "m3_ffn_fwd", "m3_ffn_bwd", "m3_adamw_plan_make", "m3_adamw_step",
           "m3_status_string", "m3_last_hip_error")
SCRATCH_BYTES = 256 << 20   # M3_SCRATCH_BYTES: the allocation-free scan's fixed workspace
CTL_BYTES = 1280            # M3_CTL_BYTES: a scan workspace's control block (zero before first use)
_lib = None


def lib() -> ctypes.CDLL:
    """Load libm3.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -c 'import __graft_entry__ as g; g.build()'`")
        L = ctypes.CDLL(LIB_PATH)
        vp, dims_p = ctypes.c_void_p, ctypes.POINTER(M3Dims)
        L.m3_scan_workspace_bytes.argtypes = [dims_p]
        L.m3_scan_workspace_bytes.restype = ctypes.c_size_t
        L.m3_scan_fwd.argtypes = [dims_p] + [vp] * 15 + [vp, ctypes.c_size_t, vp]
        L.m3_scan_fwd.restype = ctypes.c_int
        L.m3_scan_fwd_gated.argtypes = [dims_p] + [vp] * 16 + [vp, ctypes.c_size_t, vp]
        L.m3_scan_fwd_gated.restype = ctypes.c_int
        L.m3_scan_fwd_varlen.argtypes = ([dims_p, ctypes.POINTER(ctypes.c_int64)] + [vp] * 16
                                         + [vp, ctypes.c_size_t, vp])
        L.m3_scan_fwd_varlen.restype = ctypes.c_int
        i64p = ctypes.POINTER(ctypes.c_int64)
        L.m3_scan_varlen_workspace_bytes.argtypes = [dims_p, i64p]
        L.m3_scan_varlen_workspace_bytes.restype = ctypes.c_size_t
        L.m3_scan_varlen_check.argtypes = [dims_p, i64p, vp, ctypes.c_size_t,
                                           ctypes.POINTER(ctypes.c_uint32), vp]
        L.m3_scan_varlen_check.restype = ctypes.c_int
        L.m3_step.argtypes = [dims_p] + [vp] * 12 + [vp]
        L.m3_step.restype = ctypes.c_int
        L.m3_step_gated.argtypes = [dims_p] + [vp] * 13 + [vp]
        L.m3_step_gated.restype = ctypes.c_int
        pro_p = ctypes.POINTER(M3Prologue)
        L.m3_scan_fwd_pro.argtypes = [dims_p, pro_p] + [vp] * 16 + [vp, ctypes.c_size_t, vp]
        L.m3_scan_fwd_pro.restype = ctypes.c_int
        L.m3_step_pro.argtypes = [dims_p, pro_p] + [vp] * 13 + [vp]
        L.m3_step_pro.restype = ctypes.c_int
        L.m3_scan_bwd_workspace_bytes.argtypes = [dims_p]
        L.m3_scan_bwd_workspace_bytes.restype = ctypes.c_size_t
        L.m3_scan_bwd.argtypes = [dims_p] + [vp] * 20 + [vp, ctypes.c_size_t, vp]
        L.m3_scan_bwd.restype = ctypes.c_int
        L.m3_scan_fwd_noalloc.argtypes = [dims_p] + [vp] * 15 + [vp]
        L.m3_scan_fwd_noalloc.restype = ctypes.c_int
        L.m3_scan_check.argtypes = [dims_p, vp, ctypes.c_size_t, ctypes.POINTER(ctypes.c_uint32), vp]
        L.m3_scan_check.restype = ctypes.c_int
        glr_p = ctypes.POINTER(M3GlrDims)
        L.m3_glr_workspace_bytes.argtypes = [glr_p]
        L.m3_glr_workspace_bytes.restype = ctypes.c_size_t
        L.m3_glr_fwd.argtypes = [glr_p] + [vp] * 9 + [vp, ctypes.c_size_t, vp]
        L.m3_glr_bwd.argtypes = [glr_p] + [vp] * 14 + [vp, ctypes.c_size_t, vp]
        L.m3_glr_step.argtypes = [glr_p] + [vp] * 7 + [vp]
        L.m3_glr_check.argtypes = [glr_p, vp, ctypes.c_size_t, ctypes.POINTER(ctypes.c_uint32), vp]
        ffn_p = ctypes.POINTER(M3FfnDims)
        L.m3_ffn_workspace_bytes.argtypes = [ffn_p, ctypes.c_int]
        L.m3_ffn_workspace_bytes.restype = ctypes.c_size_t
        L.m3_ffn_fwd.argtypes = [ffn_p] + [vp] * 5 + [vp, ctypes.c_size_t, vp]
        L.m3_ffn_bwd.argtypes = [ffn_p] + [vp] * 9 + [vp, ctypes.c_size_t, vp]
        plan_p = ctypes.POINTER(M3AdamwPlan)
        L.m3_adamw_plan_make.argtypes = [ctypes.POINTER(M3AdamwTensor), ctypes.c_int64, ctypes.c_int32,
                                         ctypes.c_int32, plan_p, vp, ctypes.c_size_t]
        L.m3_adamw_step.argtypes = [ctypes.POINTER(M3AdamwConfig), plan_p, vp, vp, vp]
        for name in ("glr_fwd", "glr_bwd", "glr_step", "glr_check", "ffn_fwd", "ffn_bwd",
                     "adamw_plan_make", "adamw_step"):
            getattr(L, "m3_" + name).restype = ctypes.c_int
        L.m3_set_wait_limit.argtypes = [ctypes.c_uint32]
        L.m3_set_wait_limit.restype = None
        L.m3_status_string.argtypes = [ctypes.c_int]
        L.m3_status_string.restype = ctypes.c_char_p
        L.m3_last_hip_error.argtypes = []
        L.m3_last_hip_error.restype = ctypes.c_int
        _lib = L
    return _lib


def _check(status: int):
    if status != M3_OK:
        msg = lib().m3_status_string(status).decode()
        if status == M3_ERR_HIP:
            msg += f" (hipError {lib().m3_last_hip_error()})"
        raise M3Error(status, msg)


def _p(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("libm3 takes contiguous tensors")
    return t.data_ptr()


# The raw handle of the current stream without a Stream object (half the
# marshalling time of a decode step went into building one), where torch has it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_cur_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None and _cur_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_cur_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _on_stream(stream, call, *args):
    """call(*args) as it runs where `stream` is the current one: what it allocates and
    clears is in that stream's order, not in the caller's.  Its results may be used on
    the caller's stream once that has waited, and freed there."""
    s = stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream))
    here = torch.cuda.current_stream()
    if s.cuda_stream == here.cuda_stream:
        return call(*args)
    with torch.cuda.stream(s):
        out = call(*args)
    results = out.values() if isinstance(out, dict) else out if isinstance(out, tuple) else (out,)
    for r in results:
        for t in r if isinstance(r, tuple) else (r,):     # (a carry is a pair)
            t.record_stream(here)
    return out


def _a_strides(A: torch.Tensor, batch: int, seqlen: int, nheads: int):
    """A is per head [H] or per token [B, L, H] (Mamba-3's data-dependent A)."""
    if A.dim() == 1 and A.shape[0] == nheads:
        return 0, 0, 1
    if A.dim() == 3 and tuple(A.shape) == (batch, seqlen, nheads):
        s = A.stride()
        return s[0], s[1], s[2]
    raise ValueError(f"A must be [H] or [B, L, H], got {tuple(A.shape)}")


def _theta_per_head(theta: Optional[torch.Tensor], nheads: int, dstate: int) -> bool:
    """theta given as per-head frequencies omega [H, N/2] (angle = dt * omega)
    rather than per-token angles."""
    return theta is not None and theta.dim() == 2 and tuple(theta.shape) == (nheads, dstate // 2)


def scan_dims(x: torch.Tensor, Bm: torch.Tensor, chunk: int, A: Optional[torch.Tensor] = None,
              split: bool = False, per_chunk: bool = False, seg: int = 0,
              theta_per_head: bool = False) -> M3Dims:
    batch, seqlen, nheads, rank, headdim = x.shape
    dstate = Bm.shape[-1]
    sb, st, sh = _a_strides(A, batch, seqlen, nheads) if A is not None else (0, 0, 1)
    flags = ((M3_SCAN_SPLIT if split else 0) | (M3_SCAN_PER_CHUNK if per_chunk else 0)
             | (M3_THETA_PER_HEAD if theta_per_head else 0))
    return M3Dims(batch, seqlen, nheads, headdim, dstate, rank, int(chunk),
                  _IO[x.dtype], flags, sb, st, sh, int(seg))


def workspace_bytes(dims: M3Dims) -> int:
    return int(lib().m3_scan_workspace_bytes(ctypes.byref(dims)))


class LookBackTimeout(RuntimeError):
    """A single-pass scan's look-back wait gave up: its y and final state are invalid."""


def scan_check(dims: M3Dims, workspace, stream=None) -> int:
    """m3_scan_check: the number of look-back waits that gave up in the last
    scan run with `dims` on `workspace` (synchronises the stream)."""
    n = ctypes.c_uint32(0)
    wsb = workspace.numel() if workspace is not None else 0
    _check(lib().m3_scan_check(ctypes.byref(dims), _p(workspace), wsb, ctypes.byref(n),
                               _stream(stream)))
    return int(n.value)


def set_wait_limit(polls: int) -> None:
    """m3_set_wait_limit: polls before a look-back wait gives up (0: default)."""
    lib().m3_set_wait_limit(int(polls))


def scan_fwd(x, Bm, Cm, dt, A, lam, theta, D, chunk: int,
             init_state=None, init_carry=None, out=None, workspace=None,
             stream=None, split: bool = False, per_chunk: bool = False, seg: int = 0,
             z=None, check: bool = False
             ) -> Tuple[torch.Tensor, torch.Tensor, Tuple[torch.Tensor, torch.Tensor]]:
    """m3_scan_fwd (m3_scan_fwd_gated when the gate input `z`, shaped like x,
    is given: y o SiLU(z)); `theta` is [B,L,H,N/2] per-token angles, or
    [H,N/2] per-head frequencies omega (M3_THETA_PER_HEAD: angle dt * omega).
    Returns y [B,L,H,R,P], final_state [B,H,N,P] fp32
    and the carry (B_{L-1} [B,H,R,N], X_{L-1} [B,H,R,P]).  `out` may supply
    (y, final_state, carryB, carryX) to write into.  Kernel choice: `split`
    (M3_SCAN_SPLIT, three kernels), `per_chunk` (M3_SCAN_PER_CHUNK, one chunk
    per workgroup), else the segmented kernel with `seg` chunks per
    workgroup (0: library choice).  With `check`, the call synchronises and
    raises LookBackTimeout when a look-back wait gave up (m3_scan_check)."""
    if stream is not None and (out is None or workspace is None):
        return _on_stream(stream, scan_fwd, x, Bm, Cm, dt, A, lam, theta, D, chunk, init_state, init_carry,
                          out, workspace, None, split, per_chunk, seg, z, check)
    d = scan_dims(x, Bm, chunk, A, split, per_chunk, seg,
                  _theta_per_head(theta, x.shape[2], Bm.shape[-1]))
    batch, seqlen, nheads, rank, headdim = x.shape
    dstate = Bm.shape[-1]
    dev = x.device
    if out is None:
        y = torch.empty_like(x)
        fs = torch.empty((batch, nheads, dstate, headdim), dtype=torch.float32, device=dev)
        cB = torch.empty((batch, nheads, rank, dstate), dtype=x.dtype, device=dev)
        cX = torch.empty((batch, nheads, rank, headdim), dtype=x.dtype, device=dev)
    else:
        y, fs, cB, cX = out
    nbytes = workspace_bytes(d)
    if workspace is None and nbytes > 0:
        workspace = torch.zeros(nbytes, dtype=torch.uint8, device=dev)   # control block zero
    icB, icX = (None, None) if init_carry is None else init_carry
    wsb = workspace.numel() if workspace is not None else 0
    if z is None:
        _check(lib().m3_scan_fwd(ctypes.byref(d), _p(x), _p(Bm), _p(Cm), _p(dt), _p(A), _p(lam),
                                 _p(theta), _p(D), _p(init_state), _p(icB), _p(icX), _p(y),
                                 _p(fs), _p(cB), _p(cX), _p(workspace), wsb, _stream(stream)))
    else:
        if z.shape != x.shape or z.dtype != x.dtype:
            raise ValueError("z must have the shape and dtype of x")
        _check(lib().m3_scan_fwd_gated(ctypes.byref(d), _p(x), _p(Bm), _p(Cm), _p(dt), _p(A),
                                       _p(lam), _p(theta), _p(D), _p(z), _p(init_state), _p(icB),
                                       _p(icX), _p(y), _p(fs), _p(cB), _p(cX), _p(workspace), wsb,
                                       _stream(stream)))
    if check:
        n = scan_check(d, workspace, stream)
        if n:
            raise LookBackTimeout(f"{n} look-back wait(s) gave up: y and the final state are invalid")
    return y, fs, (cB, cX)


def scan_fwd_noalloc(x, Bm, Cm, dt, A, lam, theta, D, chunk: int, out,
                     init_state=None, init_carry=None, stream=None, split: bool = False,
                     per_chunk: bool = False, seg: int = 0):
    """m3_scan_fwd_noalloc: the scan with the library's fixed device scratch
    as its workspace (no allocation in the library).  `out` = (y,
    final_state, carryB, carryX) must be given (this call allocates nothing
    either); arguments otherwise as scan_fwd."""
    d = scan_dims(x, Bm, chunk, A, split, per_chunk, seg,
                  _theta_per_head(theta, x.shape[2], Bm.shape[-1]))
    y, fs, cB, cX = out
    icB, icX = (None, None) if init_carry is None else init_carry
    _check(lib().m3_scan_fwd_noalloc(ctypes.byref(d), _p(x), _p(Bm), _p(Cm), _p(dt), _p(A),
                                     _p(lam), _p(theta), _p(D), _p(init_state), _p(icB), _p(icX),
                                     _p(y), _p(fs), _p(cB), _p(cX), _stream(stream)))
    return y, fs, (cB, cX)


def varlen_dims(x, Bm, A, chunk: int, cu, split: bool = False, per_chunk: bool = False,
                seg: int = 0, theta=None) -> M3Dims:
    T, nheads, rank, headdim = x.shape
    dstate = Bm.shape[-1]
    S = len(cu) - 1
    if A.dim() == 1 and A.shape[0] == nheads:
        sb, st, sh = 0, 0, 1
    elif A.dim() == 2 and tuple(A.shape) == (T, nheads):
        sb, (st, sh) = 0, A.stride()
    else:
        raise ValueError(f"A must be [H] or [T, H], got {tuple(A.shape)}")
    ph = theta is not None and _theta_per_head(theta, nheads, dstate)
    flags = ((M3_SCAN_SPLIT if split else 0) | (M3_SCAN_PER_CHUNK if per_chunk else 0)
             | (M3_THETA_PER_HEAD if ph else 0))
    return M3Dims(S, T, nheads, headdim, dstate, rank, int(chunk), _IO[x.dtype], flags, sb, st, sh,
                  int(seg))


def _cu_list(cu_seqlens):
    return [int(v) for v in (cu_seqlens.tolist() if hasattr(cu_seqlens, "tolist") else cu_seqlens)]


def varlen_workspace_bytes(dims: M3Dims, cu_seqlens) -> int:
    """m3_scan_varlen_workspace_bytes: the workspace of the one-launch varlen
    scan (0: it does not apply)."""
    cu = _cu_list(cu_seqlens)
    return int(lib().m3_scan_varlen_workspace_bytes(ctypes.byref(dims), (ctypes.c_int64 * len(cu))(*cu)))


def varlen_check(dims: M3Dims, cu_seqlens, workspace, stream=None) -> int:
    """m3_scan_varlen_check: look-back timeouts of the last varlen call on
    `workspace` (synchronises the stream)."""
    cu = _cu_list(cu_seqlens)
    n = ctypes.c_uint32(0)
    wsb = workspace.numel() if workspace is not None else 0
    _check(lib().m3_scan_varlen_check(ctypes.byref(dims), (ctypes.c_int64 * len(cu))(*cu),
                                      _p(workspace), wsb, ctypes.byref(n), _stream(stream)))
    return int(n.value)


def scan_fwd_varlen(x, Bm, Cm, dt, A, lam, theta, D, chunk: int, cu_seqlens,
                    init_state=None, init_carry=None, z=None, workspace=None, stream=None,
                    split: bool = False, per_chunk: bool = False, seg: int = 0,
                    check: bool = False):
    """m3_scan_fwd_varlen: sequences packed along the token axis, x [T,H,R,P],
    Bm/Cm [T,H,R,N], dt/lam [T,H], theta [T,H,N/2] (or [H,N/2] frequencies),
    A [H] or [T,H]; `cu_seqlens` (S + 1 offsets, host list or tensor).  Returns
    y [T,H,R,P], final_state [S,H,N,P] and the carry ([S,H,R,N], [S,H,R,P]).
    Without a workspace one is allocated (zero-filled) for the one-launch
    scan where that applies, else for the largest sequence."""
    if stream is not None:
        return _on_stream(stream, scan_fwd_varlen, x, Bm, Cm, dt, A, lam, theta, D, chunk, cu_seqlens,
                          init_state, init_carry, z, workspace, None, split, per_chunk, seg, check)
    cu = [int(v) for v in (cu_seqlens.tolist() if hasattr(cu_seqlens, "tolist") else cu_seqlens)]
    T, nheads, rank, headdim = x.shape
    dstate = Bm.shape[-1]
    S = len(cu) - 1
    if A.dim() == 1 and A.shape[0] == nheads:
        sb, st, sh = 0, 0, 1
    elif A.dim() == 2 and tuple(A.shape) == (T, nheads):
        sb, (st, sh) = 0, A.stride()
    else:
        raise ValueError(f"A must be [H] or [T, H], got {tuple(A.shape)}")
    flags = ((M3_SCAN_SPLIT if split else 0) | (M3_SCAN_PER_CHUNK if per_chunk else 0)
             | (M3_THETA_PER_HEAD if _theta_per_head(theta, nheads, dstate) else 0))
    d = M3Dims(S, T, nheads, headdim, dstate, rank, int(chunk), _IO[x.dtype], flags, sb, st, sh,
               int(seg))
    dev = x.device
    y = torch.empty_like(x)
    fs = torch.empty((S, nheads, dstate, headdim), dtype=torch.float32, device=dev)
    cB = torch.empty((S, nheads, rank, dstate), dtype=x.dtype, device=dev)
    cX = torch.empty((S, nheads, rank, headdim), dtype=x.dtype, device=dev)
    if workspace is None:
        one = varlen_workspace_bytes(d, cu)
        if one == 0:
            longest = max([cu[i + 1] - cu[i] for i in range(S)] + [0])
            d1 = M3Dims(1, longest, nheads, headdim, dstate, rank, int(chunk), _IO[x.dtype], flags,
                        0, st, sh, int(seg))
            one = workspace_bytes(d1)
        workspace = torch.zeros(max(one, 16), dtype=torch.uint8, device=dev)
    icB, icX = (None, None) if init_carry is None else init_carry
    cu_arr = (ctypes.c_int64 * len(cu))(*cu)
    _check(lib().m3_scan_fwd_varlen(ctypes.byref(d), cu_arr, _p(x), _p(Bm), _p(Cm), _p(dt), _p(A),
                                    _p(lam), _p(theta), _p(D), _p(z), _p(init_state), _p(icB),
                                    _p(icX), _p(y), _p(fs), _p(cB), _p(cX), _p(workspace),
                                    workspace.numel(), _stream(stream)))
    if check:
        n = varlen_check(d, cu, workspace, stream)
        if n:
            raise LookBackTimeout(f"{n} look-back wait(s) gave up: y and the final state are invalid")
    return y, fs, (cB, cX)


@functools.lru_cache(maxsize=256)
def _step_dims(xs, bs, dtype, ash, ast, theta_per_head):
    """The dims of a decode step by shapes, strides and dtype (a decode loop
    makes the same ones for every token; the library only reads them)."""
    batch, nheads, rank, headdim = xs
    if len(ash) == 1 and ash[0] == nheads:
        sb, sh = 0, 1
    elif len(ash) == 2 and tuple(ash) == (batch, nheads):
        sb, sh = ast
    else:
        raise ValueError(f"A must be [H] or [B, H], got {tuple(ash)}")
    return M3Dims(batch, 1, nheads, headdim, bs[-1], rank, 1, _IO[dtype],
                  M3_THETA_PER_HEAD if theta_per_head else 0, sb, 0, sh, 0)


def step_dims(x_t: torch.Tensor, B_t: torch.Tensor, A: torch.Tensor,
              theta_per_head: bool = False) -> M3Dims:
    d = _step_dims(x_t.shape, B_t.shape, x_t.dtype, A.shape, A.stride(), bool(theta_per_head))
    return M3Dims.from_buffer_copy(d)   # (the caller's own)


def step(state, carry, x_t, B_t, C_t, dt_t, A, lam_t, theta_t, D, y=None, stream=None, z=None):
    """m3_step (m3_step_gated when the gate input `z`, shaped like x_t, is
    given: y_t o SiLU(z_t); `theta_t` [B,H,N/2] angles or [H,N/2] frequencies
    omega, as in scan_fwd): advances `state` [B,H,N,P] and `carry`
    (B [B,H,R,N], X [B,H,R,P]) in place by one token; returns y_t [B,H,R,P]."""
    if stream is not None and y is None:
        return _on_stream(stream, step, state, carry, x_t, B_t, C_t, dt_t, A, lam_t, theta_t, D, None, None, z)
    xs, bs = x_t.shape, B_t.shape
    d = _step_dims(xs, bs, x_t.dtype, A.shape, A.stride(), _theta_per_head(theta_t, xs[1], bs[-1]))
    if y is None:
        y = torch.empty_like(x_t)
    cB, cX = carry
    if z is None:
        _check(lib().m3_step(ctypes.byref(d), _p(state), _p(cB), _p(cX), _p(x_t), _p(B_t),
                             _p(C_t), _p(dt_t), _p(A), _p(lam_t), _p(theta_t), _p(D), _p(y),
                             _stream(stream)))
    else:
        if z.shape != x_t.shape or z.dtype != x_t.dtype:
            raise ValueError("z must have the shape and dtype of x_t")
        _check(lib().m3_step_gated(ctypes.byref(d), _p(state), _p(cB), _p(cX), _p(x_t), _p(B_t),
                                   _p(C_t), _p(dt_t), _p(A), _p(lam_t), _p(theta_t), _p(D), _p(z),
                                   _p(y), _stream(stream)))
    return y


def prologue(bc_norm: bool = False, eps: float = 1e-6, norm_B=None, norm_C=None, bias_B=None,
             bias_C=None, w_x=None, w_z=None, out_norm: int = M3_OUT_NORM_NONE,
             out_group: int = 0, out_eps: float = 1e-6, out_gain=None) -> M3Prologue:
    """An m3_prologue over fp32 device tables: gains and biases [H,R,N],
    w_x / w_z [H,R,P] (None: not applied); the output norm (M3_OUT_NORM_*)
    over groups of out_group channels with gain out_gain [H,R,P] (None:
    ones)."""
    for t in (norm_B, norm_C, bias_B, bias_C, w_x, w_z, out_gain):
        if t is not None and t.dtype != torch.float32:
            raise ValueError("prologue tables are fp32")
    return M3Prologue(1 if bc_norm else 0, float(eps), _p(norm_B), _p(norm_C), _p(bias_B),
                      _p(bias_C), _p(w_x), _p(w_z), int(out_norm), int(out_group),
                      float(out_eps), _p(out_gain))


def scan_fwd_pro(x, Bm, Cm, dt, A, lam, theta, D, chunk: int, pro: M3Prologue, rank: int,
                 z=None, init_state=None, init_carry=None, out=None, workspace=None,
                 stream=None, check: bool = False, seg: int = 0):
    """m3_scan_fwd_pro: the scan with the block prologue `pro` applied to the
    raw B', C' [B,L,H,R,N] and to x (X' [B,L,H,P] when pro.w_x is set, else
    [B,L,H,R,P]) and z as they are read.  Returns y [B,L,H,R,P], the final
    state and the carry (the prologue's B_{L-1}, X_{L-1}).  `seg` is the
    dims' seg_chunks (0: chosen at launch; at least the chunk count: one
    segment per slice, the warp-specialised kernel where it is built)."""
    if stream is not None and (out is None or workspace is None):
        return _on_stream(stream, scan_fwd_pro, x, Bm, Cm, dt, A, lam, theta, D, chunk, pro, rank, z,
                          init_state, init_carry, out, workspace, None, check, seg)
    batch, seqlen, nheads = x.shape[:3]
    headdim, dstate = x.shape[-1], Bm.shape[-1]
    if tuple(Bm.shape) != (batch, seqlen, nheads, rank, dstate):
        raise ValueError("B must be [B, L, H, R, N]")
    sb, st, sh = _a_strides(A, batch, seqlen, nheads)
    flags = M3_THETA_PER_HEAD if _theta_per_head(theta, nheads, dstate) else 0
    d = M3Dims(batch, seqlen, nheads, headdim, dstate, rank, int(chunk), _IO[x.dtype], flags,
               sb, st, sh, int(seg))
    dev = x.device
    if out is None:
        y = torch.empty((batch, seqlen, nheads, rank, headdim), dtype=x.dtype, device=dev)
        fs = torch.empty((batch, nheads, dstate, headdim), dtype=torch.float32, device=dev)
        cB = torch.empty((batch, nheads, rank, dstate), dtype=x.dtype, device=dev)
        cX = torch.empty((batch, nheads, rank, headdim), dtype=x.dtype, device=dev)
    else:
        y, fs, cB, cX = out
    nbytes = workspace_bytes(d)
    if workspace is None and nbytes > 0:
        workspace = torch.zeros(nbytes, dtype=torch.uint8, device=dev)   # control block zero
    icB, icX = (None, None) if init_carry is None else init_carry
    wsb = workspace.numel() if workspace is not None else 0
    _check(lib().m3_scan_fwd_pro(ctypes.byref(d), ctypes.byref(pro), _p(x), _p(Bm), _p(Cm),
                                 _p(dt), _p(A), _p(lam), _p(theta), _p(D), _p(z),
                                 _p(init_state), _p(icB), _p(icX), _p(y), _p(fs), _p(cB), _p(cX),
                                 _p(workspace), wsb, _stream(stream)))
    if check:
        n = scan_check(d, workspace, stream)
        if n:
            raise LookBackTimeout(f"{n} look-back wait(s) gave up: y and the final state are invalid")
    return y, fs, (cB, cX)


def step_pro(state, carry, x_t, B_t, C_t, dt_t, A, lam_t, theta_t, D, pro: M3Prologue,
             z=None, y=None, stream=None):
    """m3_step_pro: one decode step with the block prologue; x_t (z) is
    [B,H,P] when pro.w_x (pro.w_z) is set.  Returns y_t [B,H,R,P]."""
    if stream is not None and y is None:
        return _on_stream(stream, step_pro, state, carry, x_t, B_t, C_t, dt_t, A, lam_t, theta_t, D, pro, z)
    batch, nheads, rank, dstate = B_t.shape
    headdim = x_t.shape[-1]
    if A.dim() == 1 and A.shape[0] == nheads:
        sb, sh = 0, 1
    elif A.dim() == 2 and tuple(A.shape) == (batch, nheads):
        sb, sh = A.stride()
    else:
        raise ValueError(f"A must be [H] or [B, H], got {tuple(A.shape)}")
    flags = M3_THETA_PER_HEAD if _theta_per_head(theta_t, nheads, dstate) else 0
    d = M3Dims(batch, 1, nheads, headdim, dstate, rank, 1, _IO[x_t.dtype], flags, sb, 0, sh, 0)
    if y is None:
        y = torch.empty((batch, nheads, rank, headdim), dtype=x_t.dtype, device=x_t.device)
    cB, cX = carry
    _check(lib().m3_step_pro(ctypes.byref(d), ctypes.byref(pro), _p(state), _p(cB), _p(cX),
                             _p(x_t), _p(B_t), _p(C_t), _p(dt_t), _p(A), _p(lam_t), _p(theta_t),
                             _p(D), _p(z), _p(y), _stream(stream)))
    return y


def scan_bwd(x, Bm, Cm, dt, A, lam, theta, D, dy, chunk: int, dfinal=None, init_state=None,
             want_dinit: bool = False, workspace=None, stream=None):
    """m3_scan_bwd: gradients of J = <dy, y> + <dfinal, final_state> for the
    scan of these inputs.  Returns a dict: dx, dB, dC (io dtype), ddt, dlam,
    dtheta, dD, dA ([H] for a per-head A, [B,L,H] for a per-token A) and
    dinit (when `want_dinit`)."""
    if stream is not None:
        return _on_stream(stream, scan_bwd, x, Bm, Cm, dt, A, lam, theta, D, dy, chunk, dfinal, init_state,
                          want_dinit, workspace)
    d = scan_dims(x, Bm, chunk, A)
    batch, seqlen, nheads, rank, headdim = x.shape
    dstate = Bm.shape[-1]
    dev = x.device
    f32 = dict(dtype=torch.float32, device=dev)
    out = dict(dx=torch.empty_like(x), dB=torch.empty_like(Bm), dC=torch.empty_like(Cm),
               ddt=torch.empty((batch, seqlen, nheads), **f32),
               dlam=torch.empty((batch, seqlen, nheads), **f32),
               dtheta=torch.empty((batch, seqlen, nheads, dstate // 2), **f32),
               dD=torch.empty((nheads,), **f32),
               dA=torch.empty((nheads,) if A.dim() == 1 else (batch, seqlen, nheads), **f32))
    dinit = torch.empty((batch, nheads, dstate, headdim), **f32) if want_dinit else None
    if dinit is not None:
        out["dinit"] = dinit
    nbytes = int(lib().m3_scan_bwd_workspace_bytes(ctypes.byref(d)))
    if workspace is None:
        workspace = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=dev)
    _check(lib().m3_scan_bwd(ctypes.byref(d), _p(x), _p(Bm), _p(Cm), _p(dt), _p(A), _p(lam),
                             _p(theta), _p(D), _p(init_state), _p(dy), _p(dfinal),
                             _p(out["dx"]), _p(out["dB"]), _p(out["dC"]), _p(out["ddt"]),
                             _p(out["dA"]), _p(out["dlam"]), _p(out["dtheta"]), _p(out["dD"]),
                             _p(dinit), _p(workspace), workspace.numel(), _stream(stream)))
    return out


# ---------------------------------------------------------------------------
# Gated linear recurrence
# ---------------------------------------------------------------------------

def _meta(t: Optional[torch.Tensor]):
    """What the checks of a tensor go by (a call's checks are kept by it: a program
    makes the same ones again and again)."""
    return None if t is None else (t.shape, t.dtype, t.get_device(), t.stride())


def _empty(t: torch.Tensor) -> torch.Tensor:
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _dense(name: str, t, shape, dtype, dev) -> None:
    """Raises unless the tensor of meta `t` (None: there is none) is contiguous, of
    this shape, type and device."""
    if t is None:
        return
    step, dense = 1, True
    for n, st in zip(reversed(t[0]), reversed(t[3])):
        dense = dense and (n == 1 or st == step)
        step *= n
    if tuple(t[0]) != tuple(shape) or t[1] is not dtype or t[2] != dev or not (dense or step == 0):
        raise ValueError(f"{name} must be contiguous {dtype} {tuple(shape)} on the device of x")


def _on_gpu(x) -> None:
    if x[2] < 0:
        raise ValueError("libm3 takes tensors of a GPU")


def _work(t: torch.Tensor, x: torch.Tensor):
    """A workspace's address and bytes."""
    if t.dtype is not torch.uint8 or t.get_device() != x.get_device() or not t.is_contiguous():
        raise ValueError("a workspace is contiguous bytes (torch.uint8) on the device of x")
    return t.data_ptr(), t.numel()


@functools.lru_cache(maxsize=256)
def _glr_dims(x, r, i, z) -> M3GlrDims:
    """The dims of a recurrence by the tensors' metas, checked (the library only reads
    them)."""
    shape, dtype = x[0], x[1]
    if dtype not in _IO:
        raise ValueError("x must be fp32 or bf16")
    if len(shape) not in (2, 3):
        raise ValueError(f"x must be [B, L, D] or [B, D], got {tuple(shape)}")
    strides = []
    for name, t in (("x", x), ("r", r), ("i", i), ("z", z)):
        if t is None:
            strides += [0, 0]
            continue
        if t[:3] != x[:3]:
            raise ValueError(f"{name} must have the shape, dtype and device of x")
        if shape[-1] > 1 and t[3][-1] != 1:
            raise ValueError(f"{name}: libm3 takes channels next to each other (channel stride 1)")
        # (a stride over one element is never walked, whatever torch reports)
        st = [t[3][k] if shape[k] > 1 else 0 for k in range(len(shape) - 1)]
        strides += [st[0], st[1] if len(st) > 1 else 0]
    return M3GlrDims(shape[0], 1 if len(shape) == 2 else shape[1], shape[-1], _IO[dtype], 0, *strides)


@functools.lru_cache(maxsize=256)
def _glr_call(x, r, i, z, A, like, states, *state) -> M3GlrDims:
    """The dims of a call on x [B, L, D] (a step: [B, D]), and the checks of its other
    tensors: A [D], one like x, the saved states, and states [B, D]."""
    d, dev = _glr_dims(x, r, i, z), x[2]
    _dense("A", A, (d.width,), torch.float32, dev)
    _dense("y or dy", like, x[0], x[1], dev)
    _dense("states", states, (d.batch, -(-d.seqlen // GLR_CHUNK), d.width), torch.float32, dev)
    for t in state:
        _dense("a state or its gradient", t, (d.batch, d.width), torch.float32, dev)
    _on_gpu(x)
    return d


def glr_dims(x, r=None, i=None, z=None) -> M3GlrDims:
    """The dims of a recurrence over x [B, L, D] (a step: [B, D]) with gates r and i
    and the output gate z."""
    return M3GlrDims.from_buffer_copy(_glr_dims(_meta(x), _meta(r), _meta(i), _meta(z)))   # (the caller's own)


def glr_workspace(x, r=None, i=None, z=None) -> torch.Tensor:
    """A workspace (zero-filled) for glr_fwd and glr_bwd of these inputs: keep it for
    further calls, one at a time."""
    n = int(lib().m3_glr_workspace_bytes(ctypes.byref(glr_dims(x, r, i, z))))
    return torch.zeros(max(n, 16), dtype=torch.uint8, device=x.device)


def glr_check(x, r, i, workspace, z=None, stream=None) -> int:
    """m3_glr_check: look-back waits that gave up in the last call on `workspace`
    (synchronises the stream)."""
    n = ctypes.c_uint32(0)
    _check(lib().m3_glr_check(ctypes.byref(glr_dims(x, r, i, z)), _p(workspace), workspace.numel(),
                              ctypes.byref(n), _stream(stream)))
    return int(n.value)


def glr_fwd(x, r, i, A, z=None, init_state=None, save_states: bool = False, out=None,
            workspace=None, stream=None):
    """m3_glr_fwd: h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigmoid(i_t) x_t with
    log a_t = A sigmoid(r_t), y = h, or h o SiLU(z).  x, r, i, z [B, L, D] (bf16 or
    fp32, channels next to each other, any batch and token strides), A [D] fp32.
    Returns y [B, L, D], final_state [B, D] fp32 and, with `save_states`, the states
    that glr_bwd takes.  `out` may supply (y, final_state)."""
    if stream is not None and (out is None or workspace is None or save_states):
        return _on_stream(stream, glr_fwd, x, r, i, A, z, init_state, save_states, out, workspace)
    y, fs = (None, None) if out is None else out
    B, L, D = x.shape
    d = _glr_call(_meta(x), _meta(r), _meta(i), _meta(z), _meta(A), _meta(y), None, _meta(init_state), _meta(fs))
    if out is None:
        y, fs = _empty(x), A.new_empty((B, D))
    states = A.new_empty((B, -(-L // GLR_CHUNK), D)) if save_states else None
    if workspace is None:
        workspace = glr_workspace(x, r, i, z)
    _check(lib().m3_glr_fwd(ctypes.byref(d), x.data_ptr(), r.data_ptr(), i.data_ptr(), A.data_ptr(), _ptr(z),
                            _ptr(init_state), y.data_ptr(), fs.data_ptr(), _ptr(states), *_work(workspace, x),
                            _stream(stream)))
    return (y, fs, states) if save_states else (y, fs)


def glr_bwd(x, r, i, A, states, dy, z=None, dfinal=None, want_dinit: bool = False,
            workspace=None, stream=None):
    """m3_glr_bwd: gradients of J = <dy, y> + <dfinal, final_state>, from the forward's
    inputs and the states it saved.  Returns a dict: dx, dr, di (dz) in the io dtype,
    dA [D] fp32 and, with `want_dinit`, dinit [B, D] fp32."""
    if stream is not None:
        return _on_stream(stream, glr_bwd, x, r, i, A, states, dy, z, dfinal, want_dinit, workspace)
    B, _, D = x.shape
    if states is None or dy is None:
        raise ValueError("glr_bwd takes the forward's states and dy")
    d = _glr_call(_meta(x), _meta(r), _meta(i), _meta(z), _meta(A), _meta(dy), _meta(states), _meta(dfinal))
    out = {k: _empty(x)
           for k in (("dx", "dr", "di") if z is None else ("dx", "dr", "di", "dz"))}
    out["dA"] = A.new_empty((D,))
    if want_dinit:
        out["dinit"] = A.new_empty((B, D))
    if workspace is None:
        workspace = glr_workspace(x, r, i, z)
    _check(lib().m3_glr_bwd(ctypes.byref(d), x.data_ptr(), r.data_ptr(), i.data_ptr(), A.data_ptr(), _ptr(z),
                            states.data_ptr(), dy.data_ptr(), _ptr(dfinal), out["dx"].data_ptr(),
                            out["dr"].data_ptr(), out["di"].data_ptr(), _ptr(out.get("dz")),
                            out["dA"].data_ptr(), _ptr(out.get("dinit")), *_work(workspace, x),
                            _stream(stream)))
    return out


def glr_step(state, x, r, i, A, z=None, y=None, stream=None):
    """m3_glr_step: one token, x, r, i, z [B, D]; advances `state` [B, D] fp32 in
    place and returns y [B, D]."""
    if stream is not None and y is None:
        return _on_stream(stream, glr_step, state, x, r, i, A, z)
    if x.dim() != 2:
        raise ValueError(f"x must be [B, D], got {tuple(x.shape)}")
    d = _glr_call(_meta(x), _meta(r), _meta(i), _meta(z), _meta(A), _meta(y), None, _meta(state))
    if y is None:
        y = _empty(x)
    _check(lib().m3_glr_step(ctypes.byref(d), state.data_ptr(), x.data_ptr(), r.data_ptr(), i.data_ptr(),
                             A.data_ptr(), _ptr(z), y.data_ptr(), _stream(stream)))
    return y


# ---------------------------------------------------------------------------
# Gated feed-forward block
# ---------------------------------------------------------------------------

@functools.lru_cache(maxsize=256)
def _ffn_dims(x, Wg, Wu, Wd, y, dy, act) -> M3FfnDims:
    """The dims of a block by the tensors' metas, checked."""
    shape, dtype, dev = x[:3]
    if dtype not in _IO:
        raise ValueError("x must be fp32 or bf16")
    if act not in _ACT:
        raise ValueError(f"act must be one of {sorted(_ACT)}")
    D, F = shape[-1], Wg[0][0]
    for name, t, want in (("Wg", Wg, (F, D)), ("Wu", Wu, (F, D)), ("Wd", Wd, (D, F))):
        _dense(name, t, want, dtype, dev)
    _dense("y", y, shape, dtype, dev)
    rows = []
    for name, t in (("x", x), ("dy", dy)):
        if t is None:
            rows.append(D)
            continue
        if t[:3] != x[:3]:
            raise ValueError(f"{name} must have the shape, dtype and device of x")
        st = t[3]
        if D > 1 and st[-1] != 1:
            raise ValueError(f"{name}: libm3 takes channels next to each other (channel stride 1)")
        # [..., D] as rows of one stride (a stride over one element is never walked)
        dims = [(n, st[k]) for k, n in enumerate(shape[:-1]) if n > 1]
        for (_, outer), (n, inner) in zip(dims, dims[1:]):
            if outer != n * inner:
                raise ValueError(f"{name}: rows must lie at one stride")
        rows.append(dims[-1][1] if dims else D)
    T = 1
    for n in shape[:-1]:
        T *= n
    _on_gpu(x)
    return M3FfnDims(T, D, F, _IO[dtype], _ACT[act], *rows)


M3_FFN_BACKWARD, M3_FFN_ANY_WEIGHTS = 1, 2


def ffn_workspace(x, Wg, backward: bool = False, any_weights: bool = False) -> torch.Tensor:
    """A workspace for ffn_fwd (ffn_bwd with `backward`, which serves both) of x
    [..., D] and Wg [F, D]: keep it for further calls, one at a time.  `any_weights`: with
    room for copies of weights that do not start on 16 bytes (made at every call)."""
    d = _ffn_dims(_meta(x), _meta(Wg), None, None, None, None, "silu")
    n = int(lib().m3_ffn_workspace_bytes(ctypes.byref(d), (M3_FFN_BACKWARD if backward else 0)
                                         | (M3_FFN_ANY_WEIGHTS if any_weights else 0)))
    return torch.empty(max(n, 16), dtype=torch.uint8, device=x.device)


def _off_16(*weights) -> bool:
    return any(w.data_ptr() % 16 for w in weights)


def ffn_fwd(x, Wg, Wu, Wd, act: str = "silu", out=None, workspace=None, stream=None):
    """m3_ffn_fwd: y = (act(x Wg^T) o (x Wu^T)) Wd^T; x [..., D] (rows at one stride), Wg
    and Wu [F, D], Wd [D, F], bf16 or fp32; act "silu" or "gelu" (tanh form).  Returns
    y, shaped like x, contiguous."""
    if stream is not None and (out is None or workspace is None):
        return _on_stream(stream, ffn_fwd, x, Wg, Wu, Wd, act, out, workspace)
    d = _ffn_dims(_meta(x), _meta(Wg), _meta(Wu), _meta(Wd), _meta(out), None, act)
    y = out if out is not None else _empty(x)
    if workspace is None:
        workspace = ffn_workspace(x, Wg, any_weights=_off_16(Wg, Wu, Wd))
    _check(lib().m3_ffn_fwd(ctypes.byref(d), x.data_ptr(), Wg.data_ptr(), Wu.data_ptr(), Wd.data_ptr(),
                            y.data_ptr(), *_work(workspace, x), _stream(stream)))
    return y


def ffn_bwd(x, Wg, Wu, Wd, dy, act: str = "silu", workspace=None, stream=None):
    """m3_ffn_bwd: gradients of J = <dy, y> from the forward's inputs (g and u are formed
    again).  Returns a dict: dx (shaped like x), dWg, dWu, dWd, in the io dtype."""
    if stream is not None:
        return _on_stream(stream, ffn_bwd, x, Wg, Wu, Wd, dy, act, workspace)
    d = _ffn_dims(_meta(x), _meta(Wg), _meta(Wu), _meta(Wd), None, _meta(dy), act)
    out = dict(dx=_empty(x), dWg=_empty(Wg), dWu=_empty(Wu), dWd=_empty(Wd))
    if workspace is None:
        workspace = ffn_workspace(x, Wg, backward=True, any_weights=_off_16(Wg, Wu, Wd))
    _check(lib().m3_ffn_bwd(ctypes.byref(d), x.data_ptr(), Wg.data_ptr(), Wu.data_ptr(), Wd.data_ptr(),
                            dy.data_ptr(), out["dx"].data_ptr(), out["dWg"].data_ptr(), out["dWu"].data_ptr(),
                            out["dWd"].data_ptr(), *_work(workspace, x), _stream(stream)))
    return out


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------

class AdamWTable:
    """The tensors of an optimizer step as m3_adamw_step takes them (built by
    adamw_table; holds them, so that their memory stays)."""

    def __init__(self, plan, table, tensors):
        self.plan, self.table, self.tensors = plan, table, tensors


def adamw_table(params, grads, exp_avg, exp_avg_sq, weight_decay=0.0, low=None, scales=None):
    """A table of tensors for adamw_step, built once while they stay where they are:
    lists of fp32 params, of grads (fp32 or bf16) and of the states, shaped like the
    params; `weight_decay` a number or one per tensor; `low` bf16 copies of the params
    to write.  The states are fp32, or with `scales` (fp32 [ceil(n / 256), 2] each)
    torch.float8_e4m3fn: e4m3 codes of m and of sqrt(v).  Zeros are the first step's
    states."""
    n = len(params)
    decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * n
    lists = [grads, exp_avg, exp_avg_sq, decay] + [v for v in (low, scales) if v is not None]
    if n == 0 or any(len(v) != n for v in lists):
        raise ValueError("adamw_table takes lists of one length")
    eight = scales is not None
    state = torch.float8_e4m3fn if eight else torch.float32
    gtype, dev = grads[0].dtype, params[0].device
    if gtype not in _IO:
        raise ValueError("gradients are fp32 or bf16")
    array = (M3AdamwTensor * n)()
    for k in range(n):
        p = params[k]
        want = [("param", p, torch.float32), ("gradient", grads[k], gtype), ("exp_avg", exp_avg[k], state),
                ("exp_avg_sq", exp_avg_sq[k], state)]
        if low is not None:
            want.append(("low", low[k], torch.bfloat16))
        for name, t, dtype in want:
            if t.dtype != dtype or t.shape != p.shape or t.device != dev:
                raise ValueError(f"tensor {k}: {name} must be {dtype} {tuple(p.shape)} on {dev}")
        if eight and (scales[k].dtype != torch.float32 or scales[k].device != dev
                      or tuple(scales[k].shape) != (-(-p.numel() // 256), 2)):
            raise ValueError(f"tensor {k}: scales must be fp32 [ceil(n / 256), 2]")
        array[k] = M3AdamwTensor(_p(p), _p(grads[k]), _p(exp_avg[k]), _p(exp_avg_sq[k]),
                                 _p(low[k]) if low is not None else None,
                                 _p(scales[k]) if eight else None, p.numel(), float(decay[k]))
    plan, make = M3AdamwPlan(), lib().m3_adamw_plan_make
    args = (array, n, _IO[gtype], M3_ADAMW_8BIT if eight else 0, ctypes.byref(plan))
    _check(make(*args, None, 0))
    host = torch.zeros(max(plan.bytes, 16), dtype=torch.uint8)
    _check(make(*args, host.data_ptr(), host.numel()))
    held = (list(params), list(grads), list(exp_avg), list(exp_avg_sq), low and list(low),
            scales and list(scales))
    return AdamWTable(plan, host.to(dev), held)


def _device_number(name: str, v, dtype, table: AdamWTable):
    """The address of a number on the device (None: it is one of the host's)."""
    if not isinstance(v, torch.Tensor) or v.get_device() < 0:
        return None
    if v.dtype is not dtype or v.numel() != 1 or v.get_device() != table.table.get_device():
        raise ValueError(f"{name} is a number of the host, or one of {dtype} on the device")
    return v.data_ptr()


def adamw_step(table: AdamWTable, step, lr, betas=(0.9, 0.999), eps: float = 1e-8,
               grad_scale=None, seed: int = 0, stream=None) -> None:
    """m3_adamw_step: one AdamW step (the `step`-th, from 1) over the table's tensors, in
    place.  `grad_scale` is a device scalar that every gradient is multiplied by (None:
    1); `seed` feeds the 8-bit states' stochastic rounding: another for every step.

    A captured step keeps `step`, `lr` and `seed`.  For one that goes on from replay to
    replay give `step` as an int64 tensor of one element on the device, which the program
    or the graph advances (the rounding's seed is then seed + step), and `lr`, where
    it changes, as a float64 one."""
    if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1
                                   or grad_scale.get_device() != table.table.get_device()):
        raise ValueError("grad_scale is one fp32 number on the device")
    if table.table.get_device() < 0:
        raise ValueError("libm3 takes tensors of a GPU")
    at, rate = _device_number("step", step, torch.int64, table), _device_number("lr", lr, torch.float64, table)
    c = M3AdamwConfig(0.0 if rate else float(lr), float(betas[0]), float(betas[1]), float(eps),
                      0 if at else int(step), int(seed) & (2 ** 64 - 1), at, rate)
    _check(lib().m3_adamw_step(ctypes.byref(c), ctypes.byref(table.plan), table.table.data_ptr(),
                               None if grad_scale is None else grad_scale.data_ptr(), _stream(stream)))
