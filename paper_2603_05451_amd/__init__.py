"""MI355X-native fused attention (forward + backward): thin Python binding of libattn.so.

Argument marshalling only: every step of the path runs in the HIP kernels behind the C ABI
declared in include/attn.h.  PyTorch supplies device memory and streams.  There is no CPU
or eager fallback: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import array
import ctypes
import math
import os
from functools import lru_cache
from typing import NamedTuple

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libattn.so")
_lib = None
_native = None          # _binding: the well-formed calls, marshalled natively (csrc/binding.cpp); loaded with the library

ATTN_OK, ATTN_EINVAL, ATTN_EUNSUPPORTED, ATTN_ELAUNCH = 0, -1, -2, -3


class AttnError(RuntimeError):
    def __init__(self, code: int, text: str):
        super().__init__(f"libattn error {code}: {text}")
        self.code = code


def lib():
    """Load libattn.so (built in-tree by build.py); fail loudly when it is absent."""
    global _lib, _native
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} not found: run `python -m paper_2603_05451_amd.build` "
                              "(hipcc --offload-arch=gfx950); there is no fallback path")
        # PyTorch ships its own HIP runtime (same SONAME as the system one).  Load torch first
        # so that libattn.so binds to the runtime that owns torch's streams and allocations;
        # two HIP runtimes in one process cannot launch on each other's streams.
        import torch  # noqa: F401
        L = ctypes.CDLL(LIB_PATH)
        vp, i, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
        L.attn_fwd.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, f, i, vp]
        L.attn_fwd.restype = i
        L.attn_fwd_ex.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, i, f, i, vp]
        L.attn_fwd_ex.restype = i
        L.attn_bwd.argtypes = [vp] * 9 + [i, i, i, i, i, f, i, vp, sz, vp]
        L.attn_bwd.restype = i
        L.attn_bwd_ex.argtypes = [vp] * 9 + [i, i, i, i, i, i, f, i, vp, sz, vp]
        L.attn_bwd_ex.restype = i
        L.attn_bwd_phases.argtypes = [vp] * 9 + [i, i, i, i, i, i, f, i, vp, sz, vp, i]
        L.attn_bwd_phases.restype = i
        L.attn_bwd_noalloc.argtypes = [vp] * 9 + [i, i, i, i, i, i, f, i, vp]
        L.attn_bwd_noalloc.restype = i
        L.attn_bwd_workspace_bytes.argtypes = [i] * 6
        L.attn_bwd_workspace_bytes.restype = sz
        L.attn_fwd_dtype.argtypes = [i, vp, vp, vp, vp, vp, i, i, i, i, i, i, f, i, vp]
        L.attn_fwd_dtype.restype = i
        L.attn_bwd_dtype.argtypes = [i] + [vp] * 9 + [i, i, i, i, i, i, f, i, vp, sz, vp]
        L.attn_bwd_dtype.restype = i
        L.attn_varlen_fwd_dtype.argtypes = [i] + [vp] * 7 + [i] * 7 + [f, i, vp, sz, vp]
        L.attn_varlen_fwd_dtype.restype = i
        L.attn_varlen_bwd_dtype.argtypes = [i] + [vp] * 11 + [i] * 7 + [f, i, vp, sz, vp]
        L.attn_varlen_bwd_dtype.restype = i
        L.attn_varlen_workspace_bytes.argtypes = [i] * 8
        L.attn_varlen_workspace_bytes.restype = sz
        sp = ctypes.POINTER(AttnStrides)
        L.attn_strided_workspace_bytes.argtypes = [i] * 8
        L.attn_strided_workspace_bytes.restype = sz
        L.attn_fwd_strided.argtypes = [i] + [vp, sp] * 4 + [vp] + [i] * 7 + [f, i, vp, sz, vp]
        L.attn_fwd_strided.restype = i
        L.attn_bwd_strided.argtypes = [i] + [vp, sp] * 5 + [vp] + [vp, sp] * 3 + [i] * 7 + [f, i, vp, sz, vp]
        L.attn_bwd_strided.restype = i
        # the same two for this module's own calls, with the addresses that _with_strides makes
        L.strides_by_address = []
        for fn in ("attn_fwd_strided", "attn_bwd_strided"):
            own = L[fn]                     # (indexing gives a function object of its own)
            own.argtypes = [vp if t is sp else t for t in getattr(L, fn).argtypes]
            own.restype = i
            L.strides_by_address.append(own)
        L.attn_varlen_plan.argtypes = [vp, vp] + [i] * 7 + [vp, sz, vp]
        L.attn_varlen_plan.restype = i
        L.attn_varlen_fwd.argtypes = [vp] * 7 + [i] * 7 + [f, i, vp, sz, vp]
        L.attn_varlen_fwd.restype = i
        L.attn_varlen_bwd.argtypes = [vp] * 11 + [i] * 7 + [f, i, vp, sz, vp]
        L.attn_varlen_bwd.restype = i
        rp, cp = ctypes.POINTER(AttnRope), ctypes.POINTER(AttnCacheLayout)
        L.attn_rope_fwd.argtypes = [i, rp] + [vp, sp] * 4 + [i] * 5 + [vp]
        L.attn_rope_fwd.restype = i
        L.attn_rope_workspace_bytes.argtypes = [i] * 5
        L.attn_rope_workspace_bytes.restype = sz
        L.attn_rope_bwd.argtypes = [i, rp] + [vp, sp] * 6 + [vp, vp] + [i] * 5 + [vp, sz, vp]
        L.attn_rope_bwd.restype = i
        L.attn_cache_write.argtypes = [i, cp, vp, sp, vp, sp, vp, i, vp]
        L.attn_cache_write.restype = i
        L.attn_cache_read.argtypes = [i, cp, vp, i, vp, vp, vp]
        L.attn_cache_read.restype = i
        L.attn_cache_workspace_bytes.argtypes = [cp, i, i, i, i]
        L.attn_cache_workspace_bytes.restype = sz
        L.attn_cache_fwd.argtypes = [i, cp, vp, sp, vp, sp, vp, vp, i, vp, i, i, i, f, i, vp, sz, vp]
        L.attn_cache_fwd.restype = i
        L.attn_cache_chunk_workspace_bytes.argtypes = [cp, i, i, i, i]
        L.attn_cache_chunk_workspace_bytes.restype = sz
        L.attn_cache_chunk_fwd.argtypes = [i, cp, vp, sp, vp, sp, vp, vp, i, vp, vp, i, i, i, f, i, vp, sz, vp]
        L.attn_cache_chunk_fwd.restype = i
        L.attn_cache_weigh_workspace_bytes.argtypes = [cp, i, i, i, i, i]
        L.attn_cache_weigh_workspace_bytes.restype = sz
        L.attn_cache_weigh.argtypes = [i, cp, vp, sp, vp, vp, vp, i, vp, vp, i, i, i, f, i, i, vp, sz, vp]
        L.attn_cache_weigh.restype = i
        L.attn_cache_evict_workspace_bytes.argtypes = [cp, i, i]
        L.attn_cache_evict_workspace_bytes.restype = sz
        L.attn_cache_evict.argtypes = [cp, vp, vp, i, vp, vp, i, i, vp, vp, sz, vp]
        L.attn_cache_evict.restype = i
        L.attn_exp2_emulated.argtypes = [vp, vp, sz, i, vp]
        L.attn_exp2_emulated.restype = i
        L.attn_strerror.argtypes = [i]
        L.attn_strerror.restype = ctypes.c_char_p
        L.attn_version.restype = i
        try:
            from . import _binding
        except ImportError as e:
            raise ImportError(f"{_HERE}/_binding.so is missing or does not load ({e}): run `python -m paper_2603_05451_amd.build`; "
                              "there is no fallback path") from e
        address = lambda f: ctypes.cast(f, ctypes.c_void_p).value
        _binding.bind(*(address(f) for f in (L.attn_fwd_dtype, L.attn_bwd_phases, L.attn_bwd_dtype, L.attn_bwd_workspace_bytes, L.attn_varlen_fwd_dtype,
                                             L.attn_varlen_bwd_dtype, L.attn_varlen_workspace_bytes, L.attn_fwd_strided, L.attn_bwd_strided,
                                             L.attn_strided_workspace_bytes, L.attn_rope_fwd, L.attn_rope_bwd, L.attn_rope_workspace_bytes,
                                             L.attn_cache_write, L.attn_cache_read, L.attn_cache_fwd, L.attn_cache_workspace_bytes,
                                             L.attn_cache_chunk_fwd, L.attn_cache_chunk_workspace_bytes, L.attn_cache_weigh,
                                             L.attn_cache_weigh_workspace_bytes, L.attn_cache_evict, L.attn_cache_evict_workspace_bytes)),
                      torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream, torch.nn.Parameter)
        _native = _binding
        _lib = L                # last: another thread that finds it set uses both
    return _lib


def _call():
    if _native is None:
        lib()
    return _native


def _done(r):
    """Outputs of a native call, or its error."""
    if type(r) is int:
        _check(r)
    return r


def attn_strerror(code: int) -> str:
    return lib().attn_strerror(int(code)).decode()


def attn_version() -> int:
    return int(lib().attn_version())


def _check(rc: int):
    if rc != ATTN_OK:
        raise AttnError(rc, attn_strerror(rc))


# Well-formed calls go through _binding (the first lines of each function below: None means that it left the call alone).
# The Python text after them takes the rest -- tensor subclasses, numbers that are no floats, tables kept in a workspace -- and
# says what is wrong with a call that is refused.
def _stream(stream):
    """Raw hipStream_t of `stream`, or of the current device's current stream."""
    if stream is not None:
        return stream.cuda_stream
    import torch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


ATTN_BF16, ATTN_F16 = 0, 1


def _dtype_code(t):
    """ATTN_BF16 / ATTN_F16 for a tensor's element type."""
    import torch
    if t.dtype == torch.bfloat16:
        return ATTN_BF16
    if t.dtype == torch.float16:
        return ATTN_F16
    raise ValueError(f"unsupported element type {t.dtype}: bf16 or fp16")


def _dev(t, name, shape, dtype):
    """Device address of a contiguous CUDA tensor of that element type and shape."""
    if not (t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} CUDA tensor")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t.data_ptr()


def _dev_lse(lse, shape, axes):
    import torch
    if not (lse.is_cuda and lse.dtype == torch.float32 and lse.is_contiguous() and lse.shape == shape):
        raise ValueError(f"lse must be a contiguous fp32 CUDA tensor [{axes}]")
    return lse.data_ptr()


@lru_cache(maxsize=256)
def _bytes(size_function, *sizes):
    """What a size function of the library says, asked once per set of plain integers (of tensor shapes: not what a
    caller of the public functions passes, which may compare equal and be refused, or change its value)."""
    return getattr(lib(), size_function)(*sizes)


def attn_bwd_workspace_bytes(B, H, Hkv, N, d_qk, d_v) -> int:
    return int(lib().attn_bwd_workspace_bytes(B, H, Hkv, N, d_qk, d_v))


def attn_fwd(q, k, v, scale, causal, o=None, lse=None, stream=None):
    """q [B,N,H,d_qk], k [B,N,Hkv,d_qk], v [B,N,Hkv,d_v] bf16 (or all fp16) on the GPU ->
    (o [B,N,H,d_v] of the same type, lse [B,H,N] fp32).  Outputs are allocated with torch unless
    passed in."""
    r = (_native or _call()).fwd(q, k, v, scale, causal, o, lse, stream)
    if r is not None:
        return _done(r)
    import torch
    B, N, H, dqk = q.shape
    Hkv, dv = k.shape[2], v.shape[3]
    code = _dtype_code(q)
    if o is None:
        o = torch.empty((B, N, H, dv), dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
    lse_p, dt = _dev_lse(lse, (B, H, N), "B,H,N"), q.dtype
    _check(lib().attn_fwd_dtype(code, _dev(q, "q", q.shape, dt), _dev(k, "k", (B, N, Hkv, dqk), dt),
                                _dev(v, "v", (B, N, Hkv, dv), dt), _dev(o, "o", (B, N, H, dv), dt), lse_p,
                                B, H, Hkv, N, dqk, dv, float(scale), int(bool(causal)), _stream(stream)))
    return o, lse


def attn_varlen_workspace_bytes(B, total_q, total_k, H, Hkv, d_qk, d_v, backward) -> int:
    return int(lib().attn_varlen_workspace_bytes(B, total_q, total_k, H, Hkv, d_qk, d_v, int(bool(backward))))


def attn_varlen_plan(cu_seqlens, total_q, total_k, H, Hkv, d_qk, d_v, workspace, cu_seqlens_k=None, stream=None):
    """Fills the tile tables of a backward-sized workspace once; later attn_varlen_fwd / attn_varlen_bwd
    calls on it may pass cu_seqlens=None and B=<number of sequences> to reuse them."""
    B = cu_seqlens.numel() - 1
    if cu_seqlens_k is None:
        cu_seqlens_k = cu_seqlens
    _check(lib().attn_varlen_plan(_dev_cu(cu_seqlens, B), _dev_cu(cu_seqlens_k, B, "cu_seqlens_k"), B, total_q, total_k,
                                  H, Hkv, d_qk, d_v, workspace.data_ptr(), workspace.numel(), _stream(stream)))


def _dev_cu(cu, B, name="cu_seqlens"):
    import torch
    if cu is None:
        return None
    if not (cu.is_cuda and cu.dtype == torch.int32 and cu.is_contiguous() and cu.shape == (B + 1,)):
        raise ValueError(f"{name} must be a contiguous int32 CUDA tensor [B+1]")
    return cu.data_ptr()


def attn_varlen_fwd(q, k, v, cu_seqlens, scale, causal, o=None, lse=None, workspace=None, stream=None,
                    cu_seqlens_k=None, B=None):
    """Packed variable-length batch: q [Tq,H,d_qk], k [Tk,Hkv,d_qk], v [Tk,Hkv,d_v] bf16 (or all fp16),
    cu_seqlens [B+1] int32 (query rows; also the key rows unless cu_seqlens_k is given), all on the
    GPU -> (o [Tq,H,d_v], lse [H,Tq] fp32)."""
    r = (_native or _call()).varlen_fwd(q, k, v, cu_seqlens, scale, causal, o, lse, workspace, stream, cu_seqlens_k)
    if r is not None:
        return _done(r)
    import torch
    T, H, dqk = q.shape
    Tk, Hkv, dv = k.shape[0], k.shape[1], v.shape[2]
    if cu_seqlens is None:       # tables kept in `workspace` by attn_varlen_plan or an earlier call
        if B is None or workspace is None:
            raise ValueError("cu_seqlens=None needs B and the workspace that holds the tables")
    else:
        B = cu_seqlens.numel() - 1
        if cu_seqlens_k is None:
            cu_seqlens_k = cu_seqlens
    if o is None:
        o = torch.empty((T, H, dv), dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty((H, T), dtype=torch.float32, device=q.device)
    lse_p, dt = _dev_lse(lse, (H, T), "H,Tq"), q.dtype
    if workspace is None:
        need = _bytes("attn_varlen_workspace_bytes", B, T, Tk, H, Hkv, dqk, dv, 0)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    _check(lib().attn_varlen_fwd_dtype(
        _dtype_code(q), _dev(q, "q", q.shape, dt), _dev(k, "k", (Tk, Hkv, dqk), dt), _dev(v, "v", (Tk, Hkv, dv), dt),
        _dev(o, "o", (T, H, dv), dt), lse_p, _dev_cu(cu_seqlens, B), _dev_cu(cu_seqlens_k, B, "cu_seqlens_k"),
        B, T, Tk, H, Hkv, dqk, dv, float(scale), int(bool(causal)), workspace.data_ptr(), workspace.numel(),
        _stream(stream)))
    return o, lse


def attn_varlen_bwd(q, k, v, o, d_o, lse, cu_seqlens, scale, causal, dq=None, dk=None, dv=None, workspace=None,
                    stream=None, cu_seqlens_k=None, B=None):
    """Backward of attn_varlen_fwd: returns (dq [Tq,H,d_qk], dk [Tk,Hkv,d_qk], dv [Tk,Hkv,d_v])."""
    r = (_native or _call()).varlen_bwd(q, k, v, o, d_o, lse, cu_seqlens, scale, causal, dq, dk, dv, workspace, stream, cu_seqlens_k)
    if r is not None:
        return _done(r)
    import torch
    T, H, dqk = q.shape
    Tk, Hkv, dv_ = k.shape[0], k.shape[1], v.shape[2]
    if cu_seqlens is None:       # tables kept in `workspace` by attn_varlen_plan or an earlier backward call
        if B is None or workspace is None:
            raise ValueError("cu_seqlens=None needs B and the workspace that holds the tables")
    else:
        B = cu_seqlens.numel() - 1
        if cu_seqlens_k is None:
            cu_seqlens_k = cu_seqlens
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    if workspace is None:
        need = _bytes("attn_varlen_workspace_bytes", B, T, Tk, H, Hkv, dqk, dv_, 1)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    lse_p, dt = _dev_lse(lse, (H, T), "H,Tq"), q.dtype
    _check(lib().attn_varlen_bwd_dtype(
        _dtype_code(q), _dev(q, "q", q.shape, dt), _dev(k, "k", (Tk, Hkv, dqk), dt), _dev(v, "v", (Tk, Hkv, dv_), dt),
        _dev(o, "o", (T, H, dv_), dt), _dev(d_o, "d_o", (T, H, dv_), dt), lse_p, _dev(dq, "dq", (T, H, dqk), dt),
        _dev(dk, "dk", (Tk, Hkv, dqk), dt), _dev(dv, "dv", (Tk, Hkv, dv_), dt), _dev_cu(cu_seqlens, B),
        _dev_cu(cu_seqlens_k, B, "cu_seqlens_k"), B, T, Tk, H, Hkv, dqk, dv_, float(scale), int(bool(causal)),
        workspace.data_ptr(), workspace.numel(), _stream(stream)))
    return dq, dk, dv


class AttnStrides(ctypes.Structure):
    """attn_strides_t of include/attn.h: element strides of the batch, token and head axes."""
    _fields_ = [("batch", ctypes.c_longlong), ("row", ctypes.c_longlong), ("head", ctypes.c_longlong)]


def _view(t, name, shape, dtype, strides):
    """Address of a [B, N, heads, d] view with a contiguous head dim; appends its strides to `strides`."""
    if not (t.is_cuda and t.dtype == dtype and t.dim() == 4 and (t.stride(3) == 1 or t.shape[3] == 1)):
        raise ValueError(f"{name} must be a 4-d {dtype} CUDA tensor with a contiguous last axis")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    strides.extend(t.stride()[:3])
    return t.data_ptr()


def _with_strides(pointers, strides):
    """pointer, attn_strides_t*, pointer, ... for the C ABI.  `strides` (three numbers per pointer, the layout of
    AttnStrides) has to outlive the call."""
    at = strides.buffer_info()[0]
    return [x for i, p in enumerate(pointers) for x in (p, at + 24 * i)]


def attn_strided_workspace_bytes(B, H, Hkv, Nq, Nk, d_qk, d_v, backward) -> int:
    return int(lib().attn_strided_workspace_bytes(B, H, Hkv, Nq, Nk, d_qk, d_v, int(bool(backward))))


def attn_fwd_strided(q, k, v, scale, causal, o=None, lse=None, workspace=None, stream=None):
    """attn_fwd on views: q [B,Nq,H,d_qk], k [B,Nk,Hkv,d_qk], v [B,Nk,Hkv,d_v] of any strides (the
    last axis contiguous), e.g. x.permute(0, 2, 1, 3) of a [B,H,N,d] tensor; any Nq, Nk >= 1 (under a
    causal mask the last query sees the last key, Nk >= Nq).  o may be a view too (default: a new
    contiguous [B,Nq,H,d_v]); lse [B,H,Nq] fp32 contiguous."""
    r = (_native or _call()).fwd_strided(q, k, v, scale, causal, o, lse, workspace, stream)
    if r is not None:
        return _done(r)
    import torch
    B, N, H, dqk = q.shape
    Nk, Hkv, dv = k.shape[1], k.shape[2], v.shape[3]
    if o is None:
        o = torch.empty((B, N, H, dv), dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty((B, H, N), dtype=torch.float32, device=q.device)
    lse_p, dt = _dev_lse(lse, (B, H, N), "B,H,Nq"), q.dtype
    if workspace is None:
        need = _bytes("attn_strided_workspace_bytes", B, H, Hkv, N, Nk, dqk, dv, 0)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    st = array.array("q")
    ptrs = (_view(q, "q", (B, N, H, dqk), dt, st), _view(k, "k", (B, Nk, Hkv, dqk), dt, st),
            _view(v, "v", (B, Nk, Hkv, dv), dt, st), _view(o, "o", (B, N, H, dv), dt, st))
    _check(lib().strides_by_address[0](_dtype_code(q), *_with_strides(ptrs, st), lse_p, B, H, Hkv, N, Nk, dqk, dv, float(scale),
                                  int(bool(causal)), workspace.data_ptr(), workspace.numel(), _stream(stream)))
    return o, lse


def attn_bwd_strided(q, k, v, o, d_o, lse, scale, causal, dq=None, dk=None, dv=None, workspace=None, stream=None):
    """Backward of attn_fwd_strided; every tensor may be a view.  Gradients default to new
    contiguous tensors shaped like q, k and v."""
    r = (_native or _call()).bwd_strided(q, k, v, o, d_o, lse, scale, causal, dq, dk, dv, workspace, stream)
    if r is not None:
        return _done(r)
    import torch
    B, N, H, dqk = q.shape
    Nk, Hkv, dv_ = k.shape[1], k.shape[2], v.shape[3]
    dq = torch.empty((B, N, H, dqk), dtype=q.dtype, device=q.device) if dq is None else dq
    dk = torch.empty((B, Nk, Hkv, dqk), dtype=q.dtype, device=q.device) if dk is None else dk
    dv = torch.empty((B, Nk, Hkv, dv_), dtype=q.dtype, device=q.device) if dv is None else dv
    lse_p, dt = _dev_lse(lse, (B, H, N), "B,H,Nq"), q.dtype
    if workspace is None:
        need = _bytes("attn_strided_workspace_bytes", B, H, Hkv, N, Nk, dqk, dv_, 1)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    st = array.array("q")
    ptrs = (_view(q, "q", (B, N, H, dqk), dt, st), _view(k, "k", (B, Nk, Hkv, dqk), dt, st),
            _view(v, "v", (B, Nk, Hkv, dv_), dt, st), _view(o, "o", (B, N, H, dv_), dt, st),
            _view(d_o, "d_o", (B, N, H, dv_), dt, st), _view(dq, "dq", (B, N, H, dqk), dt, st),
            _view(dk, "dk", (B, Nk, Hkv, dqk), dt, st), _view(dv, "dv", (B, Nk, Hkv, dv_), dt, st))
    a = _with_strides(ptrs, st)
    _check(lib().strides_by_address[1](_dtype_code(q), *a[:10], lse_p, *a[10:], B, H, Hkv, N, Nk, dqk, dv_, float(scale),
                                  int(bool(causal)), workspace.data_ptr(), workspace.numel(), _stream(stream)))
    return dq, dk, dv


def attn_exp2_emulated(x, degree, y=None, stream=None):
    """y = 2^x elementwise on the GPU: polynomial emulation of degree 3/4/5, or 0 = v_exp_f32."""
    import torch
    if not (x.is_cuda and x.dtype == torch.float32 and x.is_contiguous()):
        raise ValueError("x must be a contiguous fp32 CUDA tensor")
    y = torch.empty_like(x) if y is None else y
    _check(lib().attn_exp2_emulated(x.data_ptr(), y.data_ptr(), x.numel(), int(degree), _stream(stream)))
    return y


ATTN_BWD_PREPARE, ATTN_BWD_DKDV, ATTN_BWD_DQ, ATTN_BWD_ALL = 1, 2, 4, 7


def attn_bwd(q, k, v, o, do, lse, scale, causal, dq=None, dk=None, dv=None, workspace=None,
             stream=None, phases=ATTN_BWD_ALL):
    """Gradients dq, dk, dv (bf16, layouts of q, k, v) from do, the forward's o and lse.
    phases != ATTN_BWD_ALL maps to attn_bwd_phases (per-kernel timing only)."""
    r = (_native or _call()).bwd(q, k, v, o, do, lse, scale, causal, dq, dk, dv, workspace, stream, phases)
    if r is not None:
        return _done(r)
    import torch
    B, N, H, dqk = q.shape
    Hkv, dvd = k.shape[2], v.shape[3]
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    need = _bytes("attn_bwd_workspace_bytes", B, H, Hkv, N, dqk, dvd)
    if need == 0:
        _check(lib().attn_bwd_ex(*([None] * 9), B, H, Hkv, N, dqk, dvd, float(scale), 0, None, 0, None)
               or ATTN_EINVAL)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    code, dt = _dtype_code(q), q.dtype
    args = (_dev(q, "q", q.shape, dt), _dev(k, "k", (B, N, Hkv, dqk), dt), _dev(v, "v", (B, N, Hkv, dvd), dt),
            _dev(o, "o", (B, N, H, dvd), dt), _dev(do, "do", (B, N, H, dvd), dt), lse.data_ptr(),
            _dev(dq, "dq", q.shape, dt), _dev(dk, "dk", k.shape, dt), _dev(dv, "dv", v.shape, dt),
            B, H, Hkv, N, dqk, dvd, float(scale), int(bool(causal)), workspace.data_ptr(),
            workspace.numel() * workspace.element_size(), _stream(stream))
    if code == ATTN_BF16:
        rc = lib().attn_bwd_phases(*args, int(phases))
    elif phases == ATTN_BWD_ALL:
        rc = lib().attn_bwd_dtype(code, *args)
    else:
        raise ValueError("per-kernel phases are exposed for bf16 only")
    _check(rc)
    return dq, dk, dv


ATTN_NOALLOC_MAX_ROWS = 1 << 20


def attn_bwd_noalloc(q, k, v, o, do, lse, scale, causal, dq, dk, dv, stream=None):
    """attn_bwd with the library's built-in workspace (bf16; B * H * N <= ATTN_NOALLOC_MAX_ROWS).
    The caller passes every output: nothing is allocated, here or in the library."""
    B, N, H, dqk = q.shape
    Hkv, dvd = k.shape[2], v.shape[3]
    if _dtype_code(q) != ATTN_BF16:
        raise ValueError("attn_bwd_noalloc takes bf16 tensors")
    dt = q.dtype
    _check(lib().attn_bwd_noalloc(_dev(q, "q", q.shape, dt), _dev(k, "k", (B, N, Hkv, dqk), dt),
                                  _dev(v, "v", (B, N, Hkv, dvd), dt), _dev(o, "o", (B, N, H, dvd), dt),
                                  _dev(do, "do", (B, N, H, dvd), dt), lse.data_ptr(), _dev(dq, "dq", q.shape, dt),
                                  _dev(dk, "dk", k.shape, dt), _dev(dv, "dv", v.shape, dt), B, H, Hkv, N, dqk, dvd,
                                  float(scale), int(bool(causal)), _stream(stream)))
    return dq, dk, dv


# ---- rotary positions and head norms; the quantised cache

class AttnRope(ctypes.Structure):
    """attn_rope_t of include/attn.h."""
    _fields_ = [("freqs", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("positions_batch", ctypes.c_longlong),
                ("rot", ctypes.c_int), ("offset", ctypes.c_int), ("interleaved", ctypes.c_int), ("amplitude", ctypes.c_float),
                ("norm", ctypes.c_int), ("eps", ctypes.c_float), ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p)]


class AttnCacheLayout(ctypes.Structure):
    """attn_cache_t of include/attn.h."""
    _fields_ = [("k", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("pages", ctypes.c_int), ("page", ctypes.c_int), ("Hkv", ctypes.c_int), ("d_qk", ctypes.c_int), ("d_v", ctypes.c_int),
                ("bits", ctypes.c_int)]


def _here(t, name, dtype, stream):
    """Refuses a tensor of another type or device than the call's kernels run with."""
    import torch
    if not (t.is_cuda and t.dtype == dtype):
        raise ValueError(f"{name} must be a {dtype} CUDA tensor")
    device = torch.cuda.current_device()
    if t.device.index != device or (stream is not None and stream.device.index != device):
        raise ValueError(f"{name} is on {t.device}, the stream on {t.device if stream is None else stream.device}, the current device is {device}: "
                         "a call's tensors and stream belong to the current device")


def _scratch(t, stream):
    import torch
    _here(t, "workspace", torch.uint8, stream)
    if not t.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 CUDA tensor")


def _empty(shape, dtype, device, stream):
    """A new tensor of the call's stream: what a call makes and drops is used again behind it on that stream, not on the current one."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _rows(t, name, dtype, stream, shape=None):
    """A [B, N, heads, d] or packed [T, heads, d] view as a 4-d one."""
    _here(t, name, dtype, stream)
    if t.dim() not in (3, 4) or (t.stride(-1) != 1 and t.shape[-1] != 1):
        raise ValueError(f"{name} must be a [B, N, heads, d] or [T, heads, d] tensor with a contiguous last axis")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t if t.dim() == 4 else t.unsqueeze(0)


def _strides(t):
    return None if t is None else ctypes.byref(AttnStrides(t.stride(0) if t.shape[0] > 1 else 0, t.stride(1) if t.shape[1] > 1 else 0,
                                                           t.stride(2) if t.shape[2] > 1 else 0))


def _address(t):
    return None if t is None else t.data_ptr()


def _rope(x, y, freqs, positions, interleaved, offset, amplitude, eps, q_weight, k_weight, stream):
    """attn_rope_t for rows x (4-d, of q) and y (of k, or None)."""
    import torch
    dt, (B, N, _, d) = x.dtype, x.shape
    _here(freqs, "freqs", torch.float32, stream)
    if freqs.dim() != 1 or not freqs.is_contiguous():
        raise ValueError("freqs must be a contiguous fp32 CUDA tensor [rot / 2]")
    batch = 0
    if positions is not None:
        _here(positions, "positions", torch.int32, stream)
        if not positions.is_contiguous() or positions.shape not in ((N,), (B, N)):
            raise ValueError(f"positions must be a contiguous int32 CUDA tensor [{N}] or [{B}, {N}]")
        batch = N if positions.dim() == 2 else 0
    if eps is None and (q_weight is not None or k_weight is not None):
        raise ValueError("weights without eps: eps asks for the norms")
    for w, name, there in ((q_weight, "q_weight", True), (k_weight, "k_weight", y is not None)):
        if w is not None:
            _here(w, name, dt, stream)
            if not there or w.shape != (d,) or not w.is_contiguous():
                raise ValueError(f"{name} must be a contiguous {dt} CUDA tensor [{d}]" + ("" if there else ", and there is no k"))
    return AttnRope(freqs.data_ptr(), _address(positions), batch, 2 * freqs.shape[0], int(offset), int(bool(interleaved)), float(amplitude),
                    int(eps is not None), 0.0 if eps is None else float(eps), _address(q_weight), _address(k_weight))


def attn_rope_freqs(rot, base=10000.0, factor=1.0, original=None, low=1.0, high=32.0, device="cuda"):
    """The rot / 2 frequencies (radians per position, fp32) of rotary positions: base^(-2i / rot).  For contexts `factor` times longer
    than the trained ones: without `original` every frequency is divided by factor (positions are interpolated); with the trained
    length in `original` by parts (Peng et al. 2023, "YaRN", Sec. 3.2): frequencies that turn more than `high` times within it stay, those
    that turn less than `low` times are divided, linearly in the number of turns between."""
    import torch
    if rot <= 0 or rot % 2 or not (base > 0 and factor > 0):
        raise ValueError("rot must be even and positive, base and factor positive")
    f = float(base) ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if original is None:
        f = f / factor
    else:
        if not (original > 0 and high > low):
            raise ValueError("original must be positive and high above low")
        stay = ((original * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        f = f * (stay + (1 - stay) / factor)
    return f.float().to(device)


def attn_rope_fwd(q, k, freqs, positions=None, interleaved=False, offset=0, amplitude=1.0, eps=None, q_weight=None, k_weight=None,
                  q_out=None, k_out=None, stream=None):
    """Rotary positions of q [B,N,H,d] and k [B,N,Hkv,d] (or packed [T,H,d], [T,Hkv,d]; views with a contiguous last axis; k may be None),
    bf16 or fp16, with root-mean-square norms of their heads in front if `eps` is given (weights [d], or None: ones).  freqs [rot/2] fp32
    (attn_rope_freqs): the rotated dims are offset ... offset + rot - 1, paired i with i + rot/2 or, interleaved, neighbours.
    positions: int32 [N], [B,N] ([T] for packed tokens), or None: 0 ... N-1.  -> (q_out, k_out), new contiguous tensors unless
    passed in; an output may be its input."""
    r = (_native or _call()).rope_fwd(q, k, freqs, positions, interleaved, offset, amplitude, eps, q_weight, k_weight, q_out, k_out, stream)
    if r is not None:
        return _done(r)
    x = _rows(q, "q", q.dtype, stream)
    code, dt = _dtype_code(q), q.dtype
    y = None if k is None else _rows(k, "k", dt, stream, (*q.shape[:-2], k.shape[-2], q.shape[-1]))
    if k is None and k_out is not None:
        raise ValueError("k_out without k")
    rope = _rope(x, y, freqs, positions, interleaved, offset, amplitude, eps, q_weight, k_weight, stream)
    if q_out is None:
        q_out = _empty(q.shape, dt, q.device, stream)
    if k is not None and k_out is None:
        k_out = _empty(k.shape, dt, q.device, stream)
    xo = _rows(q_out, "q_out", dt, stream, q.shape)
    yo = None if k is None else _rows(k_out, "k_out", dt, stream, k.shape)
    B, N, H, d = x.shape
    _check(lib().attn_rope_fwd(code, ctypes.byref(rope), x.data_ptr(), _strides(x), _address(y), _strides(y), xo.data_ptr(), _strides(xo),
                               _address(yo), _strides(yo), B, N, H, 0 if y is None else y.shape[2], d, _stream(stream)))
    return q_out, k_out


def attn_rope_workspace_bytes(B, N, H, Hkv, d) -> int:
    return int(lib().attn_rope_workspace_bytes(B, N, H, Hkv, d))


def attn_rope_bwd(dq, dk, freqs, positions=None, interleaved=False, offset=0, amplitude=1.0, eps=None, q=None, k=None, q_weight=None,
                  k_weight=None, dq_in=None, dk_in=None, workspace=None, stream=None):
    """Backward of attn_rope_fwd: dq and dk are the gradients of its outputs (dk None where k was); q and k, its inputs, are needed
    with norms (eps) only.  -> (dq_in, dk_in, dq_weight, dk_weight): the gradients of q and k, and of the weights in fp32 [d]
    (None where there are no weights)."""
    r = (_native or _call()).rope_bwd(dq, dk, freqs, positions, interleaved, offset, amplitude, eps, q_weight, k_weight, q, k, dq_in, dk_in,
                                      workspace, stream)
    if r is not None:
        return _done(r)
    g = _rows(dq, "dq", dq.dtype, stream)
    code, dt = _dtype_code(dq), dq.dtype
    h = None if dk is None else _rows(dk, "dk", dt, stream, (*dq.shape[:-2], dk.shape[-2], dq.shape[-1]))
    x = y = None
    if eps is not None:
        if q is None or (k is None) != (dk is None):
            raise ValueError("with norms the backward pass needs q and k")
        x = _rows(q, "q", dt, stream, dq.shape)
        y = None if dk is None else _rows(k, "k", dt, stream, dk.shape)
    if dk is None and dk_in is not None:
        raise ValueError("dk_in without dk")
    rope = _rope(g, h, freqs, positions, interleaved, offset, amplitude, eps, q_weight, k_weight, stream)
    import torch
    dq_in = _empty(dq.shape, dt, dq.device, stream) if dq_in is None else dq_in
    dk_in = _empty(dk.shape, dt, dq.device, stream) if dk_in is None and dk is not None else dk_in
    gi = _rows(dq_in, "dq_in", dt, stream, dq.shape)
    hi = None if dk is None else _rows(dk_in, "dk_in", dt, stream, dk.shape)
    B, N, H, d = g.shape
    Hkv = 0 if h is None else h.shape[2]
    dqw = None if q_weight is None else _empty((d,), torch.float32, dq.device, stream)
    dkw = None if k_weight is None else _empty((d,), torch.float32, dq.device, stream)
    if workspace is None:
        if dqw is not None or dkw is not None:
            workspace = _empty((max(_bytes("attn_rope_workspace_bytes", B, N, H, Hkv, d), 256),), torch.uint8, dq.device, stream)
    else:
        _scratch(workspace, stream)
    _check(lib().attn_rope_bwd(code, ctypes.byref(rope), g.data_ptr(), _strides(g), _address(h), _strides(h), _address(x), _strides(x),
                               _address(y), _strides(y), gi.data_ptr(), _strides(gi), _address(hi), _strides(hi), _address(dqw), _address(dkw),
                               B, N, H, Hkv, d, _address(workspace), 0 if workspace is None else workspace.numel(), _stream(stream)))
    return dq_in, dk_in, dqw, dkw


class AttnCache(NamedTuple):
    """A paged cache in 4 or 8 bits (the formats: include/attn.h): codes k [pages, Hkv, page, d_qk * bits / 8] and v, scale bytes k_scale
    [pages, Hkv, page, d_qk / 32] and v_scale; uint8, contiguous, on the GPU.  attn_cache_new makes one."""
    k: object
    k_scale: object
    v: object
    v_scale: object


def attn_cache_new(pages, page, Hkv, d_qk, d_v, bits=4, device="cuda"):
    """A cache of zeros: `pages` pages of `page` tokens (a power of two, 16 ... 65536)."""
    import torch
    if bits not in (4, 8):
        raise ValueError("a cache holds 4 or 8 bits")
    new = lambda width: torch.zeros(pages, Hkv, page, width, dtype=torch.uint8, device=device)
    return AttnCache(new(d_qk * bits // 8), new(d_qk // 32), new(d_v * bits // 8), new(d_v // 32))


def _cache(cache, stream):
    import torch
    lead = cache[0].shape[:3]
    for t, name in zip(cache, AttnCache._fields):
        _here(t, "cache." + name, torch.uint8, stream)
        if t.dim() != 4 or t.shape[:3] != lead or not t.is_contiguous():
            raise ValueError(f"cache.{name} must be a contiguous uint8 CUDA tensor [pages, Hkv, page, ...]")
    d = [32 * cache[i].shape[3] for i in (1, 3)]
    bits = 8 if cache[0].shape[3] == d[0] else 4
    if cache[0].shape[3] != d[0] * bits // 8 or cache[2].shape[3] != d[1] * bits // 8:
        raise ValueError("the codes of a cache are as wide as its scales say in 4 or 8 bits")
    return AttnCacheLayout(*(t.data_ptr() for t in cache), lead[0], lead[2], lead[1], *d, bits)


def _indexes(t, name, shape, stream):
    import torch
    _here(t, name, torch.int32, stream)
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 CUDA tensor {list(shape)}")
    return t.data_ptr()


def attn_cache_write(k, v, slots, cache, stream=None):
    """Quantises k [T,Hkv,d_qk] and v [T,Hkv,d_v] (bf16 or fp16; views with a contiguous last axis) into slots int32 [T] of the cache
    (page * tokens-per-page + token in the page; negative or past the cache: the row is skipped; the others all different)."""
    r = (_native or _call()).cache_write(k, v, slots, cache, stream)
    if r is not None:
        return _check(r)
    layout = _cache(cache, stream)
    code, dt, T = _dtype_code(k), k.dtype, k.shape[0]
    if k.dim() != 3 or v.dim() != 3:
        raise ValueError("k and v must be [T, Hkv, d] tensors")
    x = _rows(k, "k", dt, stream, (T, layout.Hkv, layout.d_qk))
    y = _rows(v, "v", dt, stream, (T, layout.Hkv, layout.d_v))
    _check(lib().attn_cache_write(code, ctypes.byref(layout), x.data_ptr(), _strides(x), y.data_ptr(), _strides(y),
                                  _indexes(slots, "slots", (T,), stream), T, _stream(stream)))


def attn_cache_read(slots, cache, dtype, k=None, v=None, stream=None):
    """The rows at slots int32 [T] as bf16 or fp16 -> (k [T,Hkv,d_qk], v [T,Hkv,d_v]); zeros where a slot is negative or past the cache,
    infinite where a value is beyond the type's range (include/attn.h: numbers near its end that were rounded up)."""
    import torch
    if dtype is torch.bfloat16 or dtype is torch.float16:
        r = (_native or _call()).cache_read(slots, cache, dtype is torch.float16, k, v, stream)
        if r is not None:
            return _done(r)
    layout = _cache(cache, stream)
    T = slots.shape[0] if slots.dim() == 1 else 0
    at = _indexes(slots, "slots", (T,), stream)
    shapes = [(T, layout.Hkv, layout.d_qk), (T, layout.Hkv, layout.d_v)]
    k, v = (_empty(s, dtype, slots.device, stream) if t is None else t for t, s in zip((k, v), shapes))
    code = _dtype_code(k)
    for t, name, s in zip((k, v), "kv", shapes):
        _here(t, name, dtype, stream)
        _dev(t, name, s, dtype)
    _check(lib().attn_cache_read(code, ctypes.byref(layout), at, T, k.data_ptr(), v.data_ptr(), _stream(stream)))
    return k, v


def attn_cache_workspace_bytes(cache, B, Nq, H, table_width) -> int:
    return int(lib().attn_cache_workspace_bytes(ctypes.byref(_cache(cache, None)), B, Nq, H, table_width))


def attn_cache_fwd(q, cache, block_table, lens, scale, causal, o=None, lse=None, workspace=None, stream=None):
    """Attention of q [B,Nq,H,d_qk] (a view with a contiguous last axis) over a paged cache: sequence b has lens[b] keys (int32 [B]), key j
    in page block_table[b, j // page] (int32 [B,width]); under the causal mask the last query sees the last key.
    -> (o [B,Nq,H,d_v], lse [B,H,Nq] fp32); a query without a visible key has o = 0 and lse = -inf."""
    r = (_native or _call()).cache_fwd(q, cache, block_table, lens, scale, causal, o, lse, workspace, stream)
    if r is not None:
        return _done(r)
    import torch
    layout = _cache(cache, stream)
    code, dt = _dtype_code(q), q.dtype
    if q.dim() != 4:
        raise ValueError("q must be a [B, Nq, H, d] tensor")
    B, Nq, H, d = q.shape
    x = _rows(q, "q", dt, stream, (B, Nq, H, layout.d_qk))
    width = block_table.shape[1] if block_table.dim() == 2 else 0
    table, keys = _indexes(block_table, "block_table", (B, width), stream), _indexes(lens, "lens", (B,), stream)
    if o is None:
        o = _empty((B, Nq, H, layout.d_v), dt, q.device, stream)
    if lse is None:
        lse = _empty((B, H, Nq), torch.float32, q.device, stream)
    y = _rows(o, "o", dt, stream, (B, Nq, H, layout.d_v))
    _here(lse, "lse", torch.float32, stream)
    lse_p = _dev_lse(lse, (B, H, Nq), "B,H,Nq")
    if workspace is None:
        need = lib().attn_cache_workspace_bytes(ctypes.byref(layout), B, Nq, H, width)
        workspace = _empty((max(need, 256),), torch.uint8, q.device, stream)
    else:
        _scratch(workspace, stream)
    _check(lib().attn_cache_fwd(code, ctypes.byref(layout), x.data_ptr(), _strides(x), y.data_ptr(), _strides(y), lse_p, table, width, keys,
                                B, Nq, H, float(scale), int(bool(causal)), workspace.data_ptr(), workspace.numel(), _stream(stream)))
    return o, lse


def attn_cache_chunk_workspace_bytes(cache, B, T, H, table_width) -> int:
    return int(lib().attn_cache_chunk_workspace_bytes(ctypes.byref(_cache(cache, None)), B, T, H, table_width))


def attn_cache_chunk_fwd(q, cache, block_table, cu_seqlens, lens, scale, causal, o=None, lse=None, workspace=None, stream=None):
    """Attention of chunks of new tokens over a paged cache: q [T,H,d_qk] (a view with a contiguous last axis) holds the queries of sequence b in rows
    cu_seqlens[b] ... cu_seqlens[b+1] - 1 (int32 [B+1]); lens int32 [B] counts its keys (the chunk's own among them, written before), key j in page
    block_table[b, j // page] (int32 [B,width]); under the causal mask a sequence's last query sees its last key.
    -> (o [T,H,d_v], lse [H,T] fp32); a query without a visible key has o = 0 and lse = -inf, rows of no sequence are not touched (unspecified in new
    tensors)."""
    r = (_native or _call()).cache_chunk_fwd(q, cache, block_table, cu_seqlens, lens, scale, causal, o, lse, workspace, stream)
    if r is not None:
        return _done(r)
    import torch
    layout = _cache(cache, stream)
    code, dt = _dtype_code(q), q.dtype
    if q.dim() != 3:
        raise ValueError("q must be a [T, H, d] tensor")
    T, H, _ = q.shape
    x = _rows(q, "q", dt, stream, (T, H, layout.d_qk))
    B, width = block_table.shape if block_table.dim() == 2 else (0, 0)
    table, keys = _indexes(block_table, "block_table", (B, width), stream), _indexes(lens, "lens", (B,), stream)
    cu = _indexes(cu_seqlens, "cu_seqlens", (B + 1,), stream)
    if o is None:
        o = _empty((T, H, layout.d_v), dt, q.device, stream)
    if lse is None:
        lse = _empty((H, T), torch.float32, q.device, stream)
    y = _rows(o, "o", dt, stream, (T, H, layout.d_v))
    _here(lse, "lse", torch.float32, stream)
    lse_p = _dev_lse(lse, (H, T), "H,T")
    if workspace is None:
        workspace = _empty((max(lib().attn_cache_chunk_workspace_bytes(ctypes.byref(layout), B, T, H, width), 256),), torch.uint8, q.device, stream)
    else:
        _scratch(workspace, stream)
    _check(lib().attn_cache_chunk_fwd(code, ctypes.byref(layout), x.data_ptr(), _strides(x), y.data_ptr(), _strides(y), lse_p, table, width, cu, keys,
                                      B, T, H, float(scale), int(bool(causal)), workspace.data_ptr(), workspace.numel(), _stream(stream)))
    return o, lse


def attn_cache_weights(cache):
    """Weights of a cache's rows for attn_cache_weigh and attn_cache_evict: zeros, fp32 [pages, Hkv, page]."""
    import torch
    return torch.zeros(cache[0].shape[:3], dtype=torch.float32, device=cache[0].device)


def _weights(weights, layout, stream):
    import torch
    _here(weights, "weights", torch.float32, stream)
    return _dev(weights, "weights", (layout.pages, layout.Hkv, layout.page), torch.float32)


def attn_cache_weigh_workspace_bytes(cache, B, Nq, H, table_width, packed) -> int:
    return int(lib().attn_cache_weigh_workspace_bytes(ctypes.byref(_cache(cache, None)), B, Nq, H, table_width, int(bool(packed))))


def attn_cache_weigh(q, lse, weights, cache, block_table, lens, scale, causal, cu_seqlens=None, fresh=False, workspace=None, stream=None):
    """Adds to weights (fp32 [pages,Hkv,page], attn_cache_weights) the attention weight that each key of the sequences had from the queries of an
    attn_cache_chunk_fwd call (q [T,H,d_qk], its lse [H,T], its cu_seqlens) or an attn_cache_fwd call (q [B,Nq,H,d_qk], its lse [B,H,Nq], no
    cu_seqlens), summed over queries and the heads of a KV head's group; the other arguments are that call's.  fresh: the last keys, as many as the
    sequence has queries, are the call's own, their weights are set and not added to.  -> weights"""
    r = (_native or _call()).cache_weigh(q, lse, weights, cache, block_table, lens, scale, causal, cu_seqlens, fresh, workspace, stream)
    if r is not None:
        _check(r)
        return weights
    import torch
    layout = _cache(cache, stream)
    code, dt = _dtype_code(q), q.dtype
    if q.dim() != (4 if cu_seqlens is None else 3):
        raise ValueError("q must be a [T, H, d] tensor with cu_seqlens, a [B, Nq, H, d] tensor without")
    x = _rows(q, "q", dt, stream, (*q.shape[:-1], layout.d_qk))
    B, width = block_table.shape if block_table.dim() == 2 else (0, 0)
    table, keys = _indexes(block_table, "block_table", (B, width), stream), _indexes(lens, "lens", (B,), stream)
    N, H = q.shape[-3], q.shape[-2]
    if cu_seqlens is None and q.shape[0] != B:
        raise ValueError(f"q has {q.shape[0]} sequences, block_table {B}")
    cu = None if cu_seqlens is None else _indexes(cu_seqlens, "cu_seqlens", (B + 1,), stream)
    _here(lse, "lse", torch.float32, stream)
    lse_p = _dev_lse(lse, (B, H, N), "B,H,Nq") if cu is None else _dev_lse(lse, (H, N), "H,T")
    if workspace is None:
        need = lib().attn_cache_weigh_workspace_bytes(ctypes.byref(layout), B, N, H, width, int(cu is not None))
        workspace = _empty((max(need, 256),), torch.uint8, q.device, stream)
    else:
        _scratch(workspace, stream)
    _check(lib().attn_cache_weigh(code, ctypes.byref(layout), x.data_ptr(), _strides(x), lse_p, _weights(weights, layout, stream), table, width, cu, keys,
                                  B, N, H, float(scale), int(bool(causal)), int(bool(fresh)), workspace.data_ptr(), workspace.numel(), _stream(stream)))
    return weights


def attn_cache_evict_workspace_bytes(cache, B, table_width) -> int:
    return int(lib().attn_cache_evict_workspace_bytes(ctypes.byref(_cache(cache, None)), B, table_width))


def attn_cache_evict(weights, cache, block_table, lens, keep, recent, lens_out=None, workspace=None, stream=None):
    """Cuts the sequences of a paged cache down to keep[b] rows (int32 [B]), for every KV head by itself: the last `recent` stay and, of the others, those
    of greatest weight.  Rows and weights are moved in place to the sequence's first keep[b] places (which goes where: include/attn.h); the pages
    behind them are free.  -> lens_out int32 [B], min(lens, keep) (not lens itself)"""
    r = (_native or _call()).cache_evict(weights, cache, block_table, lens, keep, recent, lens_out, workspace, stream)
    if r is not None:
        return _done(r)
    import torch
    layout = _cache(cache, stream)
    B, width = block_table.shape if block_table.dim() == 2 else (0, 0)
    table, keys = _indexes(block_table, "block_table", (B, width), stream), _indexes(lens, "lens", (B,), stream)
    w, k = _weights(weights, layout, stream), _indexes(keep, "keep", (B,), stream)
    if lens_out is None:
        lens_out = _empty((B,), torch.int32, lens.device, stream)
    out = _indexes(lens_out, "lens_out", (B,), stream)
    if workspace is None:
        workspace = _empty((max(lib().attn_cache_evict_workspace_bytes(ctypes.byref(layout), B, width), 256),), torch.uint8, lens.device, stream)
    else:
        _scratch(workspace, stream)
    _check(lib().attn_cache_evict(ctypes.byref(layout), w, table, width, keys, k, int(recent), B, out, workspace.data_ptr(), workspace.numel(),
                                  _stream(stream)))
    return lens_out
