"""Binding of libserq.so: argument marshalling only, through ctypes; the calls of a layer's pass go through the extension
module `_fastcall` (csrc/fastcall.cpp) where their arguments are plain tensors and ints, and through ctypes otherwise.

Every function has the name of the C entry point it calls (include/serq.h).
PyTorch supplies device memory and the current stream; no arithmetic of the
method happens in Python.  If the shared library is missing the import of
this module's `lib()` raises -- there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libserq.so")
FASTCALL_PATH = os.path.join(_HERE, "_fastcall.so")

F32, F16, BF16, I4, F8 = 0, 1, 2, 3, 4
PATH_AUTO, PATH_SKINNY, PATH_MFMA = 0, 1, 2

_DT = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}

# name -> (restype, argtypes): mirrors include/serq.h declaration by declaration
_vp, _i, _i64, _sz = C.c_void_p, C.c_int, C.c_int64, C.c_size_t
SIGNATURES = {
    "serq_version": (_i, []),
    "serq_strerror": (C.c_char_p, [_i]),
    "serq_packed_act_bytes": (_sz, [_i64, _i64, _i]),
    "serq_packed_weight_bytes": (_sz, [_i64, _i64]),
    "serq_packed_lowrank_bytes": (_sz, [_i64, _i]),
    "serq_packed_lowrank_q4_bytes": (_sz, [_i64, _i]),
    "serq_workspace_bytes": (_sz, [_i64, _i64, _i64, _i, _i]),
    "serq_workspace_init": (_i, [_vp, _sz, _vp]),
    "serq_pack_weights": (_i, [_vp, _i, _vp, _vp, _i64, _i64, _i, _vp, _vp, _vp, _vp, _vp, _i, _vp, _vp]),
    "serq_pack_lowrank": (_i, [_vp, _i, _i64, _i, _vp, _vp]),
    "serq_unpack_lowrank": (_i, [_vp, _i64, _i, _vp, _vp]),
    "serq_pack_lowrank_q4": (_i, [_vp, _i, _i64, _i, _vp, _vp]),
    "serq_unpack_lowrank_q4": (_i, [_vp, _i64, _i, _vp, _vp, _vp]),
    "serq_unpack_weights": (_i, [_vp, _i64, _i64, _vp, _vp]),
    "serq_unpack_act": (_i, [_vp, _i, _i64, _i64, _vp, _vp]),
    "serq_quantize_act": (_i, [_vp, _i, _vp, _i64, _i64, _i64, _i, _vp, _vp, _vp]),
    "serq_swiglu_quantize_act": (_i, [_vp, _vp, _i, _vp, _i64, _i64, _i64, _i64, _i, _vp, _vp, _vp]),
    "serq_mx_swiglu_quantize_act": (_i, [_vp, _vp, _i, _vp, _i64, _i64, _i64, _i64, _vp, _vp, _vp]),
    "serq_linear": (_i, [_vp, _vp, _i, _vp, _vp, _i, _i, _vp, _i, _i64, _i64, _i64, _vp, _i, _i64,
                         _vp, _sz, _i, _vp]),
    "serq_linear_noalloc": (_i, [_vp, _vp, _i, _vp, _vp, _i, _i, _vp, _i, _i64, _i64, _i64, _vp, _i, _i64, _i, _vp]),
    "serq_gemm_i32": (_i, [_vp, _i, _vp, _i64, _i64, _i64, _vp, _i64, _vp, _sz, _i, _vp]),
    "serq_mx_act_scale_bytes": (_sz, [_i64, _i64]),
    "serq_mx_weight_scale_bytes": (_sz, [_i64, _i64]),
    "serq_mx_quantize_act": (_i, [_vp, _i, _vp, _i64, _i64, _i64, _vp, _vp, _vp]),
    "serq_mx_pack_weights": (_i, [_vp, _i, _vp, _vp, _i64, _i64, _i, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "serq_mx_unpack_weights": (_i, [_vp, _vp, _i64, _i64, _vp, _vp, _vp]),
    "serq_mx_unpack_act": (_i, [_vp, _vp, _i64, _i64, _vp, _vp, _vp]),
    "serq_mx_workspace_bytes": (_sz, [_i64, _i64, _i64]),
    "serq_mx_linear": (_i, [_vp, _vp, _vp, _vp, _i, _i, _vp, _vp, _i64, _i64, _i64, _vp, _i, _i64, _vp, _sz, _i, _vp]),
    "serq_g128_scale_bytes": (_sz, [_i64, _i64]),
    "serq_quantize_act_asym": (_i, [_vp, _i, _vp, _i64, _i64, _i64, _i, _vp, _vp, _vp, _vp]),
    "serq_g128_pack_weights": (_i, [_vp, _i, _vp, _vp, _i64, _i64, _i, _vp, _vp, _vp, _vp, _vp, _vp, _i, _vp, _vp]),
    "serq_g128_unpack_scales": (_i, [_vp, _i64, _i64, _vp, _vp]),
    "serq_g128_linear": (_i, [_vp, _vp, _vp, _i, _vp, _vp, _vp, _i, _i, _vp, _i, _i64, _i64, _i64, _vp, _i, _i64, _i, _vp]),
    "serq_rmsnorm_quantize_act": (_i, [_vp, _vp, _i, _vp, C.c_float, _i64, _i64, _i64, _i64, _vp, _i64, _i, _vp, _vp, _vp]),
    "serq_rmsnorm_quantize_act_asym": (_i, [_vp, _vp, _i, _vp, C.c_float, _i64, _i64, _i64, _i64, _vp, _i64, _i, _vp, _vp, _vp, _vp]),
    "serq_mx_rmsnorm_quantize_act": (_i, [_vp, _vp, _i, _vp, C.c_float, _i64, _i64, _i64, _i64, _vp, _i64, _vp, _vp, _vp]),
    "serq_fp6_weight_bytes": (_sz, [_i64, _i64]),
    "serq_fp6_act_bytes": (_sz, [_i64, _i64]),
    "serq_fp6_pack_weights": (_i, [_vp, _i64, _i64, _vp, _vp]),
    "serq_fp6_pack_act": (_i, [_vp, _i64, _i64, _vp, _vp]),
    "serq_proto_gemm_i32": (_i, [_vp, _vp, _i, _i64, _i64, _i64, _vp, _i64, _vp]),
    "serq_kv_append": (_i, [_vp, _i64, _i64, _i, _vp, _i64, _i64, _vp, _i64, _i64, _i, _vp, _vp, _i64, _i, _i, _vp, _vp, _vp,
                            _vp, _i64, _i64, _vp]),
    "serq_kv_append_norm": (_i, [_vp, _i64, _i64, _i, _vp, _i64, _i64, _vp, _i64, _i64, _i, _vp, _vp, C.c_float, _vp, _vp, _i64, _i, _i, _vp,
                                 _vp, _vp, _vp, _i64, _i64, _vp]),
    "serq_paged_attn": (_i, [_vp, _i64, _i64, _i, _i, _vp, _vp, _i, _i64, C.c_float, _i, _vp, _i64, _i64, _vp, _vp, _sz, _vp]),
    "serq_paged_attn_mod": (_i, [_vp, _i64, _i64, _i, _i, _vp, _vp, _i, _i64, C.c_float, _i, _vp, _vp, _i64, _i64, _vp, _vp, _sz, _vp]),
    "serq_paged_attn_workspace_bytes": (_sz, [_i64, _i, _i, _i64, _i, _i, _i]),
    "serq_bench_mfma_peak": (_i, [_vp, _i, _i, _vp, _vp]),
    "serq_bench_mfma_fp4_peak": (_i, [_vp, _i, _i, _vp, _vp]),
    "serq_bench_read": (_i, [_vp, _sz, _i, _vp, _vp]),
}

_lib = None
_fast = None            # the extension module, bound to _lib
_fast_error = None      # why there is none

# the entry points it calls, in the order of its bind()
_FAST = ["serq_quantize_act", "serq_swiglu_quantize_act", "serq_mx_quantize_act", "serq_mx_swiglu_quantize_act",
         "serq_quantize_act_asym", "serq_linear", "serq_mx_linear", "serq_g128_linear"]
# ... and in that of its bind_kv()
_FAST_KV = ["serq_kv_append", "serq_paged_attn"]
# ... and in that of its bind_norm()
_FAST_NORM = ["serq_rmsnorm_quantize_act", "serq_rmsnorm_quantize_act_asym", "serq_mx_rmsnorm_quantize_act", "serq_kv_append_norm",
              "serq_paged_attn_mod"]


class SerqError(RuntimeError):
    def __init__(self, fn: str, code: int):
        msg = lib().serq_strerror(code).decode()
        super().__init__(f"{fn} failed: {msg} ({code})")
        self.code = code


def lib() -> C.CDLL:
    """Load libserq.so (built by paper_2603_08185_amd/build.py).  Raises if it is absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                f"{LIB_PATH} not found: build it with `python -m paper_2603_08185_amd.build` "
                "(the SERQ kernels have no fallback implementation)")
        L = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _load_fastcall(L)
        _lib = L
    return _lib


def _load_fastcall(L: C.CDLL) -> None:
    # (packing and sizes do without it: that it is missing, or built for another torch, is an error where it is used)
    global _fast, _fast_error
    try:
        spec = importlib.util.spec_from_file_location("_fastcall", FASTCALL_PATH)
        mod = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(mod)
    except ImportError as e:
        _fast_error = e
        return
    mod.bind(*(C.cast(getattr(L, name), C.c_void_p).value for name in _FAST))
    mod.bind_kv(*(C.cast(getattr(L, name), C.c_void_p).value for name in _FAST_KV))
    mod.bind_norm(*(C.cast(getattr(L, name), C.c_void_p).value for name in _FAST_NORM))
    _fast = mod


def _native():
    """The extension module; its functions return None for arguments that need the general way."""
    lib()
    if _fast is None:
        raise ImportError(f"{FASTCALL_PATH} cannot be loaded: build it with `python -m paper_2603_08185_amd.build`") from _fast_error
    return _fast


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()          # (ctypes makes the void* from the number)


def _stream_short():
    # torch.cuda.current_stream().cuda_stream without the Stream object built on the way: 0.2 instead of 2.7 us, a
    # third of what a call costs the host
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _stream_public():
    return torch.cuda.current_stream().cuda_stream


def _pick_stream(names):
    """The short way stands on two names of torch's own; where it has them no longer, the public way."""
    return _stream_short if {"_cuda_getCurrentRawStream", "_cuda_getDevice"} <= set(names) else _stream_public


_stream = _pick_stream(dir(torch._C))


def _check(fn: str, rc: int):
    if rc != 0:
        raise SerqError(fn, rc)


def _dev(t: torch.Tensor, name: str):
    if not t.is_cuda:
        raise ValueError(f"{name} must live in device memory")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def flags(path: int = PATH_AUTO, splitk: int = 0, groupm: int = 0, coltiles: int = 0) -> int:
    return (path & 0xff) | ((splitk & 0xff) << 8) | ((groupm & 0xf) << 16) | ((coltiles & 0x7ff) << 20)


def workspace(M: int, N: int, K: int, r: int, abits: int, device) -> torch.Tensor:
    """A zeroed workspace for linear (paged_attention has its own)."""
    n = lib().serq_workspace_bytes(M, N, K, r, abits)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=device)
    _check("serq_workspace_init", lib().serq_workspace_init(_ptr(ws), ws.numel(), _stream()))
    return ws


@dataclass
class PackedLayer:
    """Device-resident artefacts of serq_pack_weights for one layer."""
    N: int
    K: int
    r: int
    Wq: torch.Tensor        # uint8 blob
    wscale: torch.Tensor    # fp32 [N]
    perm: torch.Tensor      # int32 [K]
    s_inv: torch.Tensor     # fp32 [K]
    R: Optional[torch.Tensor]    # [r,N] canonical residual (r_dtype) or None
    Rp: Optional[torch.Tensor]   # packed residual or None


def pack_weights(W: torch.Tensor, s: Optional[torch.Tensor], r: int, perm_in: Optional[torch.Tensor] = None,
                 r_dtype: torch.dtype = torch.bfloat16, want_R: bool = True, want_Rp: bool = True) -> PackedLayer:
    _dev(W, "W")
    N, K = W.shape
    L = lib()
    nbytes = L.serq_packed_weight_bytes(N, K)
    if nbytes == 0:
        raise SerqError("serq_packed_weight_bytes", -3)
    dev = W.device
    Wq = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    wscale = torch.empty(N, dtype=torch.float32, device=dev)
    perm = torch.empty(K, dtype=torch.int32, device=dev)
    s_inv = torch.empty(K, dtype=torch.float32, device=dev)
    R = torch.empty((r, N), dtype=r_dtype, device=dev) if (r > 0 and want_R) else None
    Rp = None
    if r > 0 and want_Rp and r_dtype in (torch.float16, torch.bfloat16):
        Rp = torch.empty(L.serq_packed_lowrank_bytes(N, r), dtype=torch.uint8, device=dev)
    if s is not None:
        _dev(s, "s")
    if perm_in is not None:
        _dev(perm_in, "perm_in")
    rc = L.serq_pack_weights(_ptr(W), _DT[W.dtype], _ptr(s), _ptr(perm_in), N, K, r, _ptr(Wq), _ptr(wscale),
                             _ptr(perm), _ptr(s_inv), _ptr(R), _DT[r_dtype], _ptr(Rp), _stream())
    _check("serq_pack_weights", rc)
    return PackedLayer(N, K, r, Wq, wscale, perm, s_inv, R, Rp)


def pack_lowrank(R: torch.Tensor) -> torch.Tensor:
    _dev(R, "R")
    r, N = R.shape
    L = lib()
    Rp = torch.empty(max(L.serq_packed_lowrank_bytes(N, r), 16), dtype=torch.uint8, device=R.device)
    _check("serq_pack_lowrank", L.serq_pack_lowrank(_ptr(R), _DT[R.dtype], N, r, _ptr(Rp), _stream()))
    return Rp


def unpack_lowrank(Rp: torch.Tensor, N: int, r: int, dtype: torch.dtype) -> torch.Tensor:
    out = torch.empty((r, N), dtype=dtype, device=Rp.device)
    _check("serq_unpack_lowrank", lib().serq_unpack_lowrank(_ptr(Rp), N, r, _ptr(out), _stream()))
    return out


def pack_lowrank_q4(R: torch.Tensor) -> torch.Tensor:
    """serq_pack_lowrank_q4: the compensation matrix [r,N] as 4-bit codes + per-channel scales."""
    _dev(R, "R")
    r, N = R.shape
    L = lib()
    Rq = torch.empty(max(L.serq_packed_lowrank_q4_bytes(N, r), 16), dtype=torch.uint8, device=R.device)
    _check("serq_pack_lowrank_q4", L.serq_pack_lowrank_q4(_ptr(R), _DT[R.dtype], N, r, _ptr(Rq), _stream()))
    return Rq


def unpack_lowrank_q4(Rq: torch.Tensor, N: int, r: int):
    codes = torch.empty((r, N), dtype=torch.int8, device=Rq.device)
    rscale = torch.empty(N, dtype=torch.float32, device=Rq.device)
    _check("serq_unpack_lowrank_q4",
           lib().serq_unpack_lowrank_q4(_ptr(Rq), N, r, _ptr(codes), _ptr(rscale), _stream()))
    return codes, rscale


def unpack_weights(Wq: torch.Tensor, N: int, K: int) -> torch.Tensor:
    out = torch.empty((N, K), dtype=torch.int8, device=Wq.device)
    _check("serq_unpack_weights", lib().serq_unpack_weights(_ptr(Wq), N, K, _ptr(out), _stream()))
    return out


def unpack_act(Xq: torch.Tensor, abits: int, M: int, K: int) -> torch.Tensor:
    out = torch.empty((M, K), dtype=torch.int8, device=Xq.device)
    _check("serq_unpack_act", lib().serq_unpack_act(_ptr(Xq), abits, M, K, _ptr(out), _stream()))
    return out


def quantize_act(X: torch.Tensor, s_inv: Optional[torch.Tensor], abits: int,
                 Xq: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None):
    """serq_quantize_act: returns (Xq packed uint8 blob, scale fp32 [M])."""
    if Xq is not None and scale is not None:
        rc = (_fast or _native()).quantize_act(X, s_inv, abits, Xq, scale)
        if rc == 0:
            return Xq, scale
        if rc is not None:
            raise SerqError("serq_quantize_act", rc)
    if not X.is_cuda:
        raise ValueError("X must live in device memory")
    if X.dim() != 2 or X.stride(1) != 1:
        raise ValueError("X must be [M,K] with unit inner stride")
    M, K = X.shape
    L = lib()
    if Xq is None:
        Xq = torch.empty(max(L.serq_packed_act_bytes(M, K, abits), 16), dtype=torch.uint8, device=X.device)
    if scale is None:
        scale = torch.empty(max(M, 1), dtype=torch.float32, device=X.device)[:M]
    ldx = X.stride(0) if M > 0 else K
    rc = L.serq_quantize_act(_ptr(X), _DT[X.dtype], _ptr(s_inv), M, K, ldx, abits, _ptr(Xq), _ptr(scale), _stream())
    _check("serq_quantize_act", rc)
    return Xq, scale


def _rows(T: torch.Tensor, what: str):
    if not T.is_cuda:
        raise ValueError(f"{what} must live in device memory")
    if T.dim() != 2 or T.stride(1) != 1:
        raise ValueError(f"{what} must be [M,K] with unit inner stride")


def swiglu_quantize_act(G: torch.Tensor, U: torch.Tensor, s_inv: Optional[torch.Tensor], abits: int,
                        Xq: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None):
    """serq_swiglu_quantize_act: quantize_act of silu(G) * U; returns (Xq packed uint8 blob, scale fp32 [M])."""
    if Xq is not None and scale is not None:
        rc = (_fast or _native()).swiglu_quantize_act(G, U, s_inv, abits, Xq, scale)
        if rc == 0:
            return Xq, scale
        if rc is not None:
            raise SerqError("serq_swiglu_quantize_act", rc)
    _rows(G, "G")
    _rows(U, "U")
    if G.shape != U.shape or G.dtype != U.dtype:
        raise ValueError("G and U must agree in shape and dtype")
    M, K = G.shape
    L = lib()
    if Xq is None:
        Xq = torch.empty(max(L.serq_packed_act_bytes(M, K, abits), 16), dtype=torch.uint8, device=G.device)
    if scale is None:
        scale = torch.empty(max(M, 1), dtype=torch.float32, device=G.device)[:M]
    rc = L.serq_swiglu_quantize_act(_ptr(G), _ptr(U), _DT[G.dtype], _ptr(s_inv), M, K, G.stride(0) if M > 0 else K,
                                    U.stride(0) if M > 0 else K, abits, _ptr(Xq), _ptr(scale), _stream())
    _check("serq_swiglu_quantize_act", rc)
    return Xq, scale


def mx_swiglu_quantize_act(G: torch.Tensor, U: torch.Tensor, s_inv: Optional[torch.Tensor],
                           Xq: Optional[torch.Tensor] = None, xsc: Optional[torch.Tensor] = None):
    """serq_mx_swiglu_quantize_act: mx_quantize_act of silu(G) * U; returns (codes blob, block-scale blob)."""
    if Xq is not None and xsc is not None:
        rc = (_fast or _native()).mx_swiglu_quantize_act(G, U, s_inv, Xq, xsc)
        if rc == 0:
            return Xq, xsc
        if rc is not None:
            raise SerqError("serq_mx_swiglu_quantize_act", rc)
    _rows(G, "G")
    _rows(U, "U")
    if G.shape != U.shape or G.dtype != U.dtype:
        raise ValueError("G and U must agree in shape and dtype")
    M, K = G.shape
    L = lib()
    if Xq is None:
        Xq = torch.empty(max(L.serq_packed_act_bytes(M, K, 4), 16), dtype=torch.uint8, device=G.device)
    if xsc is None:
        xsc = torch.empty(max(L.serq_mx_act_scale_bytes(M, K), 16), dtype=torch.uint8, device=G.device)
    rc = L.serq_mx_swiglu_quantize_act(_ptr(G), _ptr(U), _DT[G.dtype], _ptr(s_inv), M, K, G.stride(0) if M > 0 else K,
                                       U.stride(0) if M > 0 else K, _ptr(Xq), _ptr(xsc), _stream())
    _check("serq_mx_swiglu_quantize_act", rc)
    return Xq, xsc


def linear(Xq: torch.Tensor, scale: torch.Tensor, abits: int, Wq: torch.Tensor, wscale: torch.Tensor,
           M: int, N: int, K: int, Rp: Optional[torch.Tensor] = None, r: int = 0,
           r_dtype=torch.bfloat16, s_begin: int = 0,
           out_dtype: torch.dtype = torch.bfloat16, Y: Optional[torch.Tensor] = None,
           ws: Optional[torch.Tensor] = None, flags_: int = 0) -> torch.Tensor:
    """serq_linear: Y = scale * (wscale * (Xq . Wq^T) + Xq[:, S] . R).  r_dtype is the 16-bit dtype of the
    packed R, or the constant I4 when Rp is the blob of pack_lowrank_q4."""
    if Y is None:
        Y = torch.empty((M, N), dtype=out_dtype, device=Xq.device)
    rc = (_fast or _native()).linear(Xq, scale, abits, Wq, wscale, s_begin, r, Rp, _DT.get(r_dtype, r_dtype), M, N, K, Y, ws, flags_)
    if rc == 0:
        return Y
    if rc is not None:
        raise SerqError("serq_linear", rc)
    rc = lib().serq_linear(_ptr(Xq), _ptr(scale), abits, _ptr(Wq), _ptr(wscale), s_begin, r, _ptr(Rp),
                           r_dtype if isinstance(r_dtype, int) else _DT[r_dtype], M, N, K, _ptr(Y), _DT[Y.dtype],
                           Y.stride(0),
                           _ptr(ws), 0 if ws is None else ws.numel(), flags_, _stream())
    _check("serq_linear", rc)
    return Y


def linear_noalloc(Xq: torch.Tensor, scale: torch.Tensor, abits: int, Wq: torch.Tensor, wscale: torch.Tensor,
                   M: int, N: int, K: int, Y: torch.Tensor, Rp: Optional[torch.Tensor] = None, r: int = 0,
                   r_dtype=torch.bfloat16, s_begin: int = 0, flags_: int = 0) -> torch.Tensor:
    """serq_linear_noalloc: serq_linear on the library's built-in scratch buffer; the caller passes Y."""
    rc = lib().serq_linear_noalloc(_ptr(Xq), _ptr(scale), abits, _ptr(Wq), _ptr(wscale), s_begin, r, _ptr(Rp),
                                   r_dtype if isinstance(r_dtype, int) else _DT[r_dtype], M, N, K, _ptr(Y),
                                   _DT[Y.dtype], Y.stride(0), flags_, _stream())
    _check("serq_linear_noalloc", rc)
    return Y


def gemm_i32(Xq: torch.Tensor, abits: int, Wq: torch.Tensor, M: int, N: int, K: int,
             ws: Optional[torch.Tensor] = None, flags_: int = 0) -> torch.Tensor:
    """serq_gemm_i32: the raw INT32 accumulators [M,N]."""
    acc = torch.empty((M, N), dtype=torch.int32, device=Xq.device)
    rc = lib().serq_gemm_i32(_ptr(Xq), abits, _ptr(Wq), M, N, K, _ptr(acc), N,
                             _ptr(ws), 0 if ws is None else ws.numel(), flags_, _stream())
    _check("serq_gemm_i32", rc)
    return acc


# ---- MXFP4 variant ---------------------------------------------------------------------------------
@dataclass
class MxPackedLayer:
    """Device-resident artefacts of serq_mx_pack_weights for one layer."""
    N: int
    K: int
    r: int
    Wq: torch.Tensor        # uint8 blob: E2M1 codes
    wsc: torch.Tensor       # uint8 blob: E8M0 block scales
    perm: torch.Tensor      # int32 [K]
    s_inv: torch.Tensor     # fp32 [K]
    Rq: Optional[torch.Tensor]
    rsc: Optional[torch.Tensor]


def mx_pack_weights(W: torch.Tensor, s: Optional[torch.Tensor], r: int,
                    perm_in: Optional[torch.Tensor] = None) -> MxPackedLayer:
    _dev(W, "W")
    N, K = W.shape
    L = lib()
    nbytes = L.serq_packed_weight_bytes(N, K)
    if nbytes == 0:
        raise SerqError("serq_packed_weight_bytes", -3)
    dev = W.device
    Wq = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    wsc = torch.empty(L.serq_mx_weight_scale_bytes(N, K), dtype=torch.uint8, device=dev)
    perm = torch.empty(K, dtype=torch.int32, device=dev)
    s_inv = torch.empty(K, dtype=torch.float32, device=dev)
    Rq = rsc = None
    if r > 0:
        rk = 64 * ((r + 63) // 64)
        Rq = torch.empty(max(L.serq_packed_weight_bytes(N, rk), 16), dtype=torch.uint8, device=dev)
        rsc = torch.empty(max(L.serq_mx_weight_scale_bytes(N, rk), 16), dtype=torch.uint8, device=dev)
    if s is not None:
        _dev(s, "s")
    if perm_in is not None:
        _dev(perm_in, "perm_in")
    rc = L.serq_mx_pack_weights(_ptr(W), _DT[W.dtype], _ptr(s), _ptr(perm_in), N, K, r, _ptr(Wq), _ptr(wsc),
                                _ptr(perm), _ptr(s_inv), _ptr(Rq), _ptr(rsc), _stream())
    _check("serq_mx_pack_weights", rc)
    return MxPackedLayer(N, K, r, Wq, wsc, perm, s_inv, Rq, rsc)


def mx_unpack_weights(Wq: torch.Tensor, wsc: torch.Tensor, N: int, K: int):
    """Canonical view: (codes uint8 [N,K], exponent bytes uint8 [N,K/32])."""
    codes = torch.empty((N, K), dtype=torch.uint8, device=Wq.device)
    exps = torch.empty((N, K // 32), dtype=torch.uint8, device=Wq.device)
    _check("serq_mx_unpack_weights",
           lib().serq_mx_unpack_weights(_ptr(Wq), _ptr(wsc), N, K, _ptr(codes), _ptr(exps), _stream()))
    return codes, exps


def mx_quantize_act(X: torch.Tensor, s_inv: Optional[torch.Tensor],
                    Xq: Optional[torch.Tensor] = None, xsc: Optional[torch.Tensor] = None):
    """serq_mx_quantize_act: returns (E2M1 codes blob, E8M0 block-scale blob)."""
    if Xq is not None and xsc is not None:
        rc = (_fast or _native()).mx_quantize_act(X, s_inv, Xq, xsc)
        if rc == 0:
            return Xq, xsc
        if rc is not None:
            raise SerqError("serq_mx_quantize_act", rc)
    if not X.is_cuda:
        raise ValueError("X must live in device memory")
    if X.dim() != 2 or X.stride(1) != 1:
        raise ValueError("X must be [M,K] with unit inner stride")
    M, K = X.shape
    L = lib()
    if Xq is None:
        Xq = torch.empty(max(L.serq_packed_act_bytes(M, K, 4), 16), dtype=torch.uint8, device=X.device)
    if xsc is None:
        xsc = torch.empty(max(L.serq_mx_act_scale_bytes(M, K), 16), dtype=torch.uint8, device=X.device)
    ldx = X.stride(0) if M > 0 else K
    rc = L.serq_mx_quantize_act(_ptr(X), _DT[X.dtype], _ptr(s_inv), M, K, ldx, _ptr(Xq), _ptr(xsc), _stream())
    _check("serq_mx_quantize_act", rc)
    return Xq, xsc


def mx_workspace(M: int, N: int, K: int, device) -> torch.Tensor:
    """A zeroed workspace for serq_mx_linear (K slicing of the decode kernel)."""
    n = lib().serq_mx_workspace_bytes(M, N, K)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=device)
    _check("serq_workspace_init", lib().serq_workspace_init(_ptr(ws), ws.numel(), _stream()))
    return ws


def mx_unpack_act(Xq: torch.Tensor, xsc: torch.Tensor, M: int, K: int):
    codes = torch.empty((M, K), dtype=torch.uint8, device=Xq.device)
    exps = torch.empty((M, K // 32), dtype=torch.uint8, device=Xq.device)
    _check("serq_mx_unpack_act",
           lib().serq_mx_unpack_act(_ptr(Xq), _ptr(xsc), M, K, _ptr(codes), _ptr(exps), _stream()))
    return codes, exps


def mx_linear(Xq: torch.Tensor, xsc: torch.Tensor, Wq: torch.Tensor, wsc: torch.Tensor, M: int, N: int, K: int,
              Rq: Optional[torch.Tensor] = None, rsc: Optional[torch.Tensor] = None, r: int = 0, s_begin: int = 0,
              out_dtype: torch.dtype = torch.bfloat16, Y: Optional[torch.Tensor] = None,
              ws: Optional[torch.Tensor] = None, flags_: int = 0) -> torch.Tensor:
    """serq_mx_linear: Y = deq(X) . deq(W)^T + deq(X)[:, S] . deq(R)^T on the block-scaled FP4 units."""
    if Y is None:
        Y = torch.empty((M, N), dtype=out_dtype, device=Xq.device)
    rc = (_fast or _native()).mx_linear(Xq, xsc, Wq, wsc, s_begin, r, Rq, rsc, M, N, K, Y, ws, flags_)
    if rc == 0:
        return Y
    if rc is not None:
        raise SerqError("serq_mx_linear", rc)
    rc = lib().serq_mx_linear(_ptr(Xq), _ptr(xsc), _ptr(Wq), _ptr(wsc), s_begin, r, _ptr(Rq), _ptr(rsc), M, N, K,
                              _ptr(Y), _DT[Y.dtype], Y.stride(0) if M > 0 else N,
                              _ptr(ws), 0 if ws is None else ws.numel(), flags_, _stream())
    _check("serq_mx_linear", rc)
    return Y


def bench_mfma_peak(operands: torch.Tensor, iters: int, workgroups: int, sink: torch.Tensor) -> None:
    """serq_bench_mfma_peak: nothing but int8 MFMAs on the given 32 KiB of operand bytes."""
    assert operands.numel() * operands.element_size() >= 32768
    _check("serq_bench_mfma_peak", lib().serq_bench_mfma_peak(_ptr(operands), iters, workgroups, _ptr(sink), _stream()))


def bench_mfma_fp4_peak(operands: torch.Tensor, iters: int, workgroups: int, sink: torch.Tensor) -> None:
    """serq_bench_mfma_fp4_peak: nothing but block-scaled FP4 MFMAs on the given 32 KiB of operand bytes."""
    assert operands.numel() * operands.element_size() >= 32768
    _check("serq_bench_mfma_fp4_peak",
           lib().serq_bench_mfma_fp4_peak(_ptr(operands), iters, workgroups, _ptr(sink), _stream()))


def bench_read(src: torch.Tensor, nbytes: int, workgroups: int, sink: torch.Tensor) -> None:
    """serq_bench_read: nothing but one read of the first nbytes of src."""
    _check("serq_bench_read", lib().serq_bench_read(_ptr(src), nbytes, workgroups, _ptr(sink), _stream()))


# ---- group-128 weight scales + asymmetric activations -------------------------------------------------
@dataclass
class G128PackedLayer:
    """Device-resident artefacts of serq_g128_pack_weights for one layer."""
    N: int
    K: int
    r: int
    Wq: torch.Tensor        # uint8 blob (the layout of serq_pack_weights)
    gscale: torch.Tensor    # uint8 blob: fp16 group scales
    wsum: torch.Tensor      # fp32 [N]
    perm: torch.Tensor
    s_inv: torch.Tensor
    R: Optional[torch.Tensor]
    Rp: Optional[torch.Tensor]


def g128_pack_weights(W: torch.Tensor, s: Optional[torch.Tensor], r: int, perm_in: Optional[torch.Tensor] = None,
                      r_dtype: torch.dtype = torch.bfloat16) -> G128PackedLayer:
    _dev(W, "W")
    N, K = W.shape
    L = lib()
    nb = L.serq_g128_scale_bytes(N, K)
    if nb == 0:
        raise SerqError("serq_g128_scale_bytes", -3)
    dev = W.device
    Wq = torch.empty(N * K // 2, dtype=torch.uint8, device=dev)
    gsc = torch.empty(nb, dtype=torch.uint8, device=dev)
    wsum = torch.empty(N, dtype=torch.float32, device=dev)
    perm = torch.empty(K, dtype=torch.int32, device=dev)
    s_inv = torch.empty(K, dtype=torch.float32, device=dev)
    R = torch.empty((r, N), dtype=r_dtype, device=dev) if r > 0 else None
    Rp = torch.empty(L.serq_packed_lowrank_bytes(N, r), dtype=torch.uint8, device=dev) \
        if r > 0 and r_dtype in (torch.float16, torch.bfloat16) else None
    rc = L.serq_g128_pack_weights(_ptr(W), _DT[W.dtype], _ptr(s), _ptr(perm_in), N, K, r, _ptr(Wq), _ptr(gsc), _ptr(wsum),
                                  _ptr(perm), _ptr(s_inv), _ptr(R), _DT[r_dtype], _ptr(Rp), _stream())
    _check("serq_g128_pack_weights", rc)
    return G128PackedLayer(N, K, r, Wq, gsc, wsum, perm, s_inv, R, Rp)


def g128_unpack_scales(gscale: torch.Tensor, N: int, K: int) -> torch.Tensor:
    out = torch.empty((N, K // 128), dtype=torch.float32, device=gscale.device)
    _check("serq_g128_unpack_scales", lib().serq_g128_unpack_scales(_ptr(gscale), N, K, _ptr(out), _stream()))
    return out


def quantize_act_asym(X: torch.Tensor, s_inv: Optional[torch.Tensor], abits: int, Xq: Optional[torch.Tensor] = None,
                      scale: Optional[torch.Tensor] = None, zero: Optional[torch.Tensor] = None):
    """serq_quantize_act_asym: returns (Xq packed uint8 blob, scale fp32 [M], zero int32 [M])."""
    if Xq is not None and scale is not None and zero is not None:
        rc = (_fast or _native()).quantize_act_asym(X, s_inv, abits, Xq, scale, zero)
        if rc == 0:
            return Xq, scale, zero
        if rc is not None:
            raise SerqError("serq_quantize_act_asym", rc)
    _rows(X, "X")
    M, K = X.shape
    L = lib()
    if Xq is None:
        Xq = torch.empty(max(L.serq_packed_act_bytes(M, K, abits), 16), dtype=torch.uint8, device=X.device)
    if scale is None:
        scale = torch.empty(max(M, 1), dtype=torch.float32, device=X.device)[:M]
    if zero is None:
        zero = torch.empty(max(M, 1), dtype=torch.int32, device=X.device)[:M]
    rc = L.serq_quantize_act_asym(_ptr(X), _DT[X.dtype], _ptr(s_inv), M, K, X.stride(0) if M > 0 else K, abits,
                                  _ptr(Xq), _ptr(scale), _ptr(zero), _stream())
    _check("serq_quantize_act_asym", rc)
    return Xq, scale, zero


def g128_linear(Xq: torch.Tensor, scale: torch.Tensor, zero: Optional[torch.Tensor], abits: int, Wq: torch.Tensor,
                gscale: torch.Tensor, wsum: torch.Tensor, M: int, N: int, K: int, Rp: Optional[torch.Tensor] = None,
                r: int = 0, r_dtype: torch.dtype = torch.bfloat16, s_begin: int = 0,
                out_dtype: torch.dtype = torch.bfloat16, Y: Optional[torch.Tensor] = None, flags_: int = 0) -> torch.Tensor:
    """serq_g128_linear: the layer with group-128 weight scales and (optionally) per-token zero points."""
    if Y is None:
        Y = torch.empty((M, N), dtype=out_dtype, device=Xq.device)
    rc = (_fast or _native()).g128_linear(Xq, scale, zero, abits, Wq, gscale, wsum, s_begin, r, Rp, _DT.get(r_dtype), M, N, K, Y, flags_)
    if rc == 0:
        return Y
    if rc is not None:
        raise SerqError("serq_g128_linear", rc)
    rc = lib().serq_g128_linear(_ptr(Xq), _ptr(scale), _ptr(zero), abits, _ptr(Wq), _ptr(gscale), _ptr(wsum), s_begin, r,
                                _ptr(Rp), _DT[r_dtype], M, N, K, _ptr(Y), _DT[Y.dtype], Y.stride(0), flags_, _stream())
    _check("serq_g128_linear", rc)
    return Y


# ---- the quantisers fused into the residual sum and the norm ---------------------------------------------------
def _norm_rows(X, gain, residual, h):
    """Checks of rmsnorm_quantize_act and its forms; returns the arguments that describe the rows, and h."""
    _rows(X, "X")
    if X.dtype not in _DT:
        raise ValueError("X must be float32, float16 or bfloat16")
    M, K = X.shape
    if gain is not None and (not gain.is_cuda or gain.dtype != torch.float32 or gain.shape != (K,) or not gain.is_contiguous()):
        raise ValueError("gain must be fp32 [K] in device memory")
    if residual is None:
        if h is not None:
            raise ValueError("without a residual the sum is X itself: no h")
        return (M, K, X.stride(0) if M > 0 else K, 0), None
    if h is None:
        h = torch.empty((M, K), dtype=X.dtype, device=X.device)
    for t, what in ((residual, "residual"), (h, "h")):
        _rows(t, what)
        if t.shape != X.shape or t.dtype != X.dtype:
            raise ValueError(f"{what} must agree with X in shape and dtype")
    return (M, K, X.stride(0) if M > 0 else K, residual.stride(0) if M > 0 else K), h


def _buffer(t: Optional[torch.Tensor], n: int, what: str, dtype: torch.dtype, device) -> torch.Tensor:
    """A caller's output buffer of at least n elements, or a new one."""
    if t is None:
        return torch.empty(max(n, 16), dtype=dtype, device=device)
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous() or t.numel() < n:
        raise ValueError(f"{what} must be a contiguous {dtype} buffer of at least {n} elements in device memory")
    return t


def rmsnorm_quantize_act(X: torch.Tensor, gain: Optional[torch.Tensor], eps: float, abits: int, residual: Optional[torch.Tensor] = None,
                         h: Optional[torch.Tensor] = None, Xq: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None):
    """serq_rmsnorm_quantize_act: quantize_act of the normalised sum X + residual times gain; returns (Xq packed uint8 blob, scale fp32 [M],
    the sum: h, or X where there is no residual)."""
    if Xq is not None and scale is not None and (residual is None or h is not None):
        rc = (_fast or _native()).rmsnorm_quantize_act(X, gain, eps, abits, residual, h, Xq, scale)
        if rc == 0:
            return Xq, scale, X if h is None else h
        if rc is not None:
            raise SerqError("serq_rmsnorm_quantize_act", rc)
    (M, K, ldx, ldr), h = _norm_rows(X, gain, residual, h)
    L = lib()
    Xq = _buffer(Xq, L.serq_packed_act_bytes(M, K, abits), "Xq", torch.uint8, X.device)
    scale = _buffer(scale, M, "scale", torch.float32, X.device)[:M]
    rc = L.serq_rmsnorm_quantize_act(_ptr(X), _ptr(residual), _DT[X.dtype], _ptr(gain), eps, M, K, ldx, ldr, _ptr(h),
                                     h.stride(0) if h is not None and M > 0 else K, abits, _ptr(Xq), _ptr(scale), _stream())
    _check("serq_rmsnorm_quantize_act", rc)
    return Xq, scale, X if h is None else h


def rmsnorm_quantize_act_asym(X: torch.Tensor, gain: Optional[torch.Tensor], eps: float, abits: int, residual: Optional[torch.Tensor] = None,
                              h: Optional[torch.Tensor] = None, Xq: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                              zero: Optional[torch.Tensor] = None):
    """serq_rmsnorm_quantize_act_asym: quantize_act_asym of the normalised sum; returns (Xq packed uint8 blob, scale fp32 [M], zero int32
    [M], the sum)."""
    if Xq is not None and scale is not None and zero is not None and (residual is None or h is not None):
        rc = (_fast or _native()).rmsnorm_quantize_act_asym(X, gain, eps, abits, residual, h, Xq, scale, zero)
        if rc == 0:
            return Xq, scale, zero, X if h is None else h
        if rc is not None:
            raise SerqError("serq_rmsnorm_quantize_act_asym", rc)
    (M, K, ldx, ldr), h = _norm_rows(X, gain, residual, h)
    L = lib()
    Xq = _buffer(Xq, L.serq_packed_act_bytes(M, K, abits), "Xq", torch.uint8, X.device)
    scale = _buffer(scale, M, "scale", torch.float32, X.device)[:M]
    zero = _buffer(zero, M, "zero", torch.int32, X.device)[:M]
    rc = L.serq_rmsnorm_quantize_act_asym(_ptr(X), _ptr(residual), _DT[X.dtype], _ptr(gain), eps, M, K, ldx, ldr, _ptr(h),
                                          h.stride(0) if h is not None and M > 0 else K, abits, _ptr(Xq), _ptr(scale), _ptr(zero), _stream())
    _check("serq_rmsnorm_quantize_act_asym", rc)
    return Xq, scale, zero, X if h is None else h


def mx_rmsnorm_quantize_act(X: torch.Tensor, gain: Optional[torch.Tensor], eps: float, residual: Optional[torch.Tensor] = None,
                            h: Optional[torch.Tensor] = None, Xq: Optional[torch.Tensor] = None, xsc: Optional[torch.Tensor] = None):
    """serq_mx_rmsnorm_quantize_act: mx_quantize_act of the normalised sum; returns (codes blob, block-scale blob, the sum)."""
    if Xq is not None and xsc is not None and (residual is None or h is not None):
        rc = (_fast or _native()).mx_rmsnorm_quantize_act(X, gain, eps, residual, h, Xq, xsc)
        if rc == 0:
            return Xq, xsc, X if h is None else h
        if rc is not None:
            raise SerqError("serq_mx_rmsnorm_quantize_act", rc)
    (M, K, ldx, ldr), h = _norm_rows(X, gain, residual, h)
    L = lib()
    Xq = _buffer(Xq, L.serq_packed_act_bytes(M, K, 4), "Xq", torch.uint8, X.device)
    xsc = _buffer(xsc, L.serq_mx_act_scale_bytes(M, K), "xsc", torch.uint8, X.device)
    rc = L.serq_mx_rmsnorm_quantize_act(_ptr(X), _ptr(residual), _DT[X.dtype], _ptr(gain), eps, M, K, ldx, ldr, _ptr(h),
                                        h.stride(0) if h is not None and M > 0 else K, _ptr(Xq), _ptr(xsc), _stream())
    _check("serq_mx_rmsnorm_quantize_act", rc)
    return Xq, xsc, X if h is None else h


# ---- experiment: W4A4 integer sums on the FP6 form of the scaled matrix instruction -----------------------
def fp6_pack_weights(codes: torch.Tensor) -> torch.Tensor:
    """serq_fp6_pack_weights: canonical int8 codes [N,K] -> FP6 weight fragments."""
    _dev(codes, "codes")
    N, K = codes.shape
    out = torch.empty(max(lib().serq_fp6_weight_bytes(N, K), 16), dtype=torch.uint8, device=codes.device)
    _check("serq_fp6_pack_weights", lib().serq_fp6_pack_weights(_ptr(codes), N, K, _ptr(out), _stream()))
    return out


def fp6_pack_act(codes: torch.Tensor) -> torch.Tensor:
    """serq_fp6_pack_act: canonical int8 codes [M,K] -> FP6 rows."""
    _dev(codes, "codes")
    M, K = codes.shape
    out = torch.empty(max(lib().serq_fp6_act_bytes(M, K), 16), dtype=torch.uint8, device=codes.device)
    _check("serq_fp6_pack_act", lib().serq_fp6_pack_act(_ptr(codes), M, K, _ptr(out), _stream()))
    return out


def proto_gemm_i32(X: torch.Tensor, W: torch.Tensor, fp6: bool, M: int, N: int, K: int,
                   acc: Optional[torch.Tensor] = None) -> torch.Tensor:
    """serq_proto_gemm_i32: the INT32 sums from the plain tiled kernel, int8 route (fp6 = False) or FP6 route."""
    if acc is None:
        acc = torch.empty((M, N), dtype=torch.int32, device=X.device)
    _check("serq_proto_gemm_i32", lib().serq_proto_gemm_i32(_ptr(X), _ptr(W), 1 if fp6 else 0, M, N, K, _ptr(acc),
                                                            acc.stride(0) if M > 0 else N, _stream()))
    return acc


# ---- the paged cache of keys and values, and attention over it ----------------------------------------------------
class _KvCache(C.Structure):
    """serq_kv_cache (include/serq_kv.h)."""
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp),
                ("k_page", _i64), ("k_token", _i64), ("k_head", _i64), ("v_page", _i64), ("v_token", _i64), ("v_head", _i64),
                ("pages", _i64), ("page_size", C.c_int32), ("heads", C.c_int32), ("dim", C.c_int32), ("dtype", C.c_int32)]


class _KvBatch(C.Structure):
    """serq_kv_batch (include/serq_kv.h)."""
    _fields_ = [("cu_q", _vp), ("kv_len", _vp), ("table", _vp), ("table_ld", _i64), ("tokens", _i64),
                ("table_width", C.c_int32), ("seqs", C.c_int32)]


class _AttnMod(C.Structure):
    """serq_attn_mod (include/serq_kv.h)."""
    _fields_ = [("slopes", _vp), ("see_from", _vp), ("see_to", _vp), ("cap", C.c_float)]


def _heads(T: torch.Tensor, what: str, dim: Optional[int] = None):
    if not T.is_cuda:
        raise ValueError(f"{what} must live in device memory")
    if T.dim() != 3 or (T.stride(2) != 1 and T.numel() > 0) or (dim is not None and T.shape[2] != dim):
        raise ValueError(f"{what} must be [tokens, heads, dim] with unit inner stride")


def _kv_structs(K, V, table, cu_q, kv_len, tokens, dtype, k_scale, v_scale):
    for t, what in ((K, "K"), (V, "V")):
        if not t.is_cuda:
            raise ValueError(f"{what} must live in device memory")
        if t.dim() != 4 or (t.stride(3) != 1 and t.numel() > 0):
            raise ValueError(f"{what} must be [pages, page_size, heads, dim] with unit inner stride")
    if K.shape != V.shape or K.dtype != V.dtype:
        raise ValueError("K and V must agree in shape and dtype")
    for t, what, nd in ((table, "table", 2), (cu_q, "cu_q", 1), (kv_len, "kv_len", 1)):
        if not t.is_cuda or t.dtype != torch.int32 or t.dim() != nd or (t.numel() > 0 and t.stride(-1) != 1):
            raise ValueError(f"{what} must be int32 in device memory, {nd}-dimensional, with unit inner stride")
    B = kv_len.shape[0]
    if cu_q.shape[0] != B + 1 or table.shape[0] != B:
        raise ValueError("cu_q has one entry more than there are sequences, table one row a sequence")
    fp8 = K.dtype == torch.float8_e4m3fn
    if not fp8 and K.dtype != dtype:
        raise ValueError("the cache has the dtype of q, or float8_e4m3fn")
    for t, what in ((k_scale, "k_scale"), (v_scale, "v_scale")):
        if t is not None and (not t.is_cuda or t.dtype != torch.float32 or t.dim() != 1 or t.shape[0] != K.shape[2] or not t.is_contiguous()):
            raise ValueError(f"{what} must be fp32 [heads] in device memory")
    c = _KvCache(_ptr(K), _ptr(V), _ptr(k_scale), _ptr(v_scale), K.stride(0), K.stride(1), K.stride(2), V.stride(0), V.stride(1),
                 V.stride(2), K.shape[0], K.shape[1], K.shape[2], K.shape[3], F8 if fp8 else _DT[dtype])
    b = _KvBatch(_ptr(cu_q), _ptr(kv_len), _ptr(table), max(table.stride(0), table.shape[1]) if B <= 1 else table.stride(0), tokens,
                 table.shape[1], B)
    return c, b


def kv_append(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, K: torch.Tensor, V: torch.Tensor, table: torch.Tensor,
              cu_q: torch.Tensor, kv_len: torch.Tensor, cos: Optional[torch.Tensor] = None, sin: Optional[torch.Tensor] = None,
              interleaved: bool = False, positions: Optional[torch.Tensor] = None, k_scale: Optional[torch.Tensor] = None,
              v_scale: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None, q_norm: Optional[torch.Tensor] = None,
              k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6) -> Optional[torch.Tensor]:
    """serq_kv_append: rotates q and k (tables cos, sin [positions, rotated channels / 2] fp32; None: no rotation), puts k and v into
    the paged cache K, V [pages, page_size, heads, dim]; returns the rotated q (q None: keys and values only).  With q_norm, k_norm [dim] fp32
    (either may be None) serq_kv_append_norm: every head of q, of k is normalised by its root mean square first."""
    if q is not None and q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    normed = q_norm is not None or k_norm is not None
    if normed:
        rc = (_fast or _native()).kv_append_norm(q, k, v, K, V, table, cu_q, kv_len, cos, sin, 1 if interleaved else 0, positions, k_scale,
                                                 v_scale, q_out, q_norm, k_norm, eps)
    else:
        rc = (_fast or _native()).kv_append(q, k, v, K, V, table, cu_q, kv_len, cos, sin, 1 if interleaved else 0, positions, k_scale, v_scale,
                                            q_out)
    if rc == 0:
        return q_out
    if rc is not None:
        raise SerqError("serq_kv_append_norm" if normed else "serq_kv_append", rc)
    D = K.shape[-1]
    for t, what in ((k, "k"), (v, "v"), (q, "q"), (q_out, "q_out")):
        if t is not None:
            _heads(t, what, D)
            if t.shape[0] != k.shape[0] or t.dtype != k.dtype:
                raise ValueError("q, k, v and q_out must agree in tokens and dtype")
    if k.shape[1] != K.shape[2] or v.shape[1] != K.shape[2] or (q is not None and q_out.shape != q.shape):
        raise ValueError("k and v must have the cache's heads, q_out q's")
    rot = rows = 0
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin come together")
    if cos is not None:
        for t, what in ((cos, "cos"), (sin, "sin")):
            if not t.is_cuda or t.dtype != torch.float32 or t.dim() != 2 or not t.is_contiguous() or t.shape != cos.shape:
                raise ValueError(f"{what} must be fp32 [positions, rotated channels / 2] in device memory")
        rows, rot = cos.shape[0], 2 * cos.shape[1]
    if positions is not None and (not positions.is_cuda or positions.dtype != torch.int32 or positions.dim() != 1
                                  or positions.shape[0] < k.shape[0] or (positions.numel() > 1 and positions.stride(0) != 1)):
        raise ValueError("positions must be int32 [tokens] in device memory")
    c, b = _kv_structs(K, V, table, cu_q, kv_len, k.shape[0], k.dtype, k_scale, v_scale)
    for t, what in ((q_norm, "q_norm"), (k_norm, "k_norm")):
        if t is not None and (not t.is_cuda or t.dtype != torch.float32 or t.shape != (D,) or not t.is_contiguous()):
            raise ValueError(f"{what} must be fp32 [dim] in device memory")
    head = (_ptr(q), q.stride(0) if q is not None else 0, q.stride(1) if q is not None else 0, q.shape[1] if q is not None else 0,
            _ptr(k), k.stride(0), k.stride(1), _ptr(v), v.stride(0), v.stride(1), _DT[k.dtype])
    tail = (_ptr(cos), _ptr(sin), rows, rot, 1 if interleaved else 0, _ptr(positions), C.addressof(c), C.addressof(b), _ptr(q_out),
            q_out.stride(0) if q is not None else 0, q_out.stride(1) if q is not None else 0, _stream())
    if normed:
        _check("serq_kv_append_norm", lib().serq_kv_append_norm(*head, _ptr(q_norm), _ptr(k_norm), eps, *tail))
    else:
        _check("serq_kv_append", lib().serq_kv_append(*head, *tail))
    return q_out


def paged_attention_workspace(tokens: int, seqs: int, max_q: int, max_kv: int, q_heads: int, kv_heads: int, dim: int, device) -> torch.Tensor:
    """A zeroed workspace for paged_attention (slices of a long cache): for every call of up to these tokens, sequences and bounds.
    Not for the layers: theirs is workspace()'s, and neither serves the other."""
    n = lib().serq_paged_attn_workspace_bytes(tokens, seqs, max_q, max_kv, q_heads, kv_heads, dim)
    if n == 0:
        raise SerqError("serq_paged_attn_workspace_bytes", -3)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=device)
    _check("serq_workspace_init", lib().serq_workspace_init(_ptr(ws), ws.numel(), _stream()))
    return ws


def paged_attention(q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, table: torch.Tensor, cu_q: torch.Tensor, kv_len: torch.Tensor,
                    max_q: int, max_kv: int, scale: Optional[float] = None, window: int = 0, k_scale: Optional[torch.Tensor] = None,
                    v_scale: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                    ws: Optional[torch.Tensor] = None, cap: float = 0.0, slopes: Optional[torch.Tensor] = None,
                    see_from: Optional[torch.Tensor] = None, see_to: Optional[torch.Tensor] = None) -> torch.Tensor:
    """serq_paged_attn: softmax(scale q K^T) V over the cached positions up to each new token's own (scale: 1 / sqrt(dim) by default;
    window > 0: the last `window` of them); lse [tokens, q_heads] fp32 takes the logarithm of the softmax' sum.  serq_paged_attn_mod where one of these
    is given: cap > 0: scores become cap tanh(score / cap); slopes [q_heads] fp32: a head's slope times the distance is taken off; see_from, see_to
    [tokens] int32: token t sees the positions see_from[t] .. see_to[t]-1 (packed documents, prefixes seen both ways, padding)."""
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if scale is None:
        scale = q.shape[-1] ** -0.5
    modified = cap != 0 or slopes is not None or see_from is not None or see_to is not None
    if modified:
        rc = (_fast or _native()).paged_attention_mod(q, K, V, table, cu_q, kv_len, max_q, max_kv, scale, window, k_scale, v_scale, out, lse, ws,
                                                      cap, slopes, see_from, see_to)
    else:
        rc = (_fast or _native()).paged_attention(q, K, V, table, cu_q, kv_len, max_q, max_kv, scale, window, k_scale, v_scale, out, lse, ws)
    if rc == 0:
        return out
    if rc is not None:
        raise SerqError("serq_paged_attn_mod" if modified else "serq_paged_attn", rc)
    D = K.shape[-1]
    for t, what in ((q, "q"), (out, "out")):
        _heads(t, what, D)
    if out.shape != q.shape or out.dtype != q.dtype:
        raise ValueError("out must agree with q in shape and dtype")
    if lse is not None and (not lse.is_cuda or lse.dtype != torch.float32 or lse.shape != q.shape[:2] or not lse.is_contiguous()):
        raise ValueError("lse must be fp32 [tokens, q_heads] in device memory")
    if ws is not None and (not ws.is_cuda or ws.dtype != torch.uint8 or not ws.is_contiguous()):
        raise ValueError("ws must be a uint8 buffer in device memory")
    if cap != 0 and C.c_float(cap).value == 0:
        raise ValueError("cap must be a positive fp32 number, or 0 for none")
    for t, what, dt, n in ((slopes, "slopes", torch.float32, q.shape[1]), (see_from, "see_from", torch.int32, q.shape[0]),
                           (see_to, "see_to", torch.int32, q.shape[0])):
        if t is not None and (not t.is_cuda or t.dtype != dt or t.shape != (n,) or not t.is_contiguous()):
            raise ValueError(f"{what} must be {'fp32 [q_heads]' if what == 'slopes' else 'int32 [tokens]'} in device memory")
    c, b = _kv_structs(K, V, table, cu_q, kv_len, q.shape[0], q.dtype, k_scale, v_scale)
    head = (_ptr(q), q.stride(0), q.stride(1), q.shape[1], _DT[q.dtype], C.addressof(c), C.addressof(b), max_q, max_kv, scale, window)
    tail = (_ptr(out), out.stride(0), out.stride(1), _ptr(lse), _ptr(ws), 0 if ws is None else ws.numel(), _stream())
    if modified:
        m = _AttnMod(_ptr(slopes), _ptr(see_from), _ptr(see_to), cap)
        _check("serq_paged_attn_mod", lib().serq_paged_attn_mod(*head, C.addressof(m), *tail))
    else:
        _check("serq_paged_attn", lib().serq_paged_attn(*head, *tail))
    return out
