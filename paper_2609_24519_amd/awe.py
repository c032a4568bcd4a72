"""Thin ctypes binding of ``libawe.so`` (declared in include/awe.h).

Names follow the C ABI.  This module only marshals arguments: device buffers
are torch tensors (or raw integer device pointers), the stream defaults to
torch's current stream, and every step of the computation runs in the HIP
library.  If the library has not been built, ``lib()`` raises; nothing here
falls back to another implementation.
"""
import ctypes
import os
import re
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libawe.so")
HEADER = os.path.join(os.path.dirname(_HERE), "include", "awe.h")

# awe_status
OK, ERR_INVALID_VALUE, ERR_UNSUPPORTED, ERR_OVERFLOW, ERR_WORKSPACE, ERR_HIP, ERR_TABLE = range(7)
_FORMATS = ("e2m1", "e4m3", "e2m3")  # element format codes of awe_encoding_info
# awe_encoding
ENC_B13, ENC_AWE6, ENC_AWE6ALT, ENC_AWE4, ENC_MOD, ENC_TERNARY, ENC_FP16, ENC_FP8FP4, ENC_FP6K3, \
    ENC_FP6P4 = 1, 2, 3, 4, 5, 6, 7, 8, 9, 10
ENCODINGS = {"b13": ENC_B13, "awe6": ENC_AWE6, "awe6_alt": ENC_AWE6ALT, "awe4": ENC_AWE4, "mod": ENC_MOD,
             "ternary": ENC_TERNARY, "fp16_12": ENC_FP16, "fp8fp4": ENC_FP8FP4,
             "fp6k3": ENC_FP6K3, "fp6p4": ENC_FP6P4}
# awe_side, awe_dtype
SIDE_A, SIDE_B = 0, 1
I32, I64 = 0, 1
I8, F32, BF16, F16 = 2, 3, 4, 5  # element types of the operators of quantised inference

MAX_LIMBS, MAX_PLANES, MAX_PRODUCTS = 4, 8, 16
K_PAD = 256  # AWE_K_PAD: stored planes pad the reduction length to a multiple of this
NOALLOC_MAX_BYTES = 64 << 20  # AWE_NOALLOC_MAX_BYTES: the planes array of gemm_exact_noalloc


class EncodingInfo(ctypes.Structure):
    _fields_ = [
        ("r", ctypes.c_int32),
        ("limbs_a", ctypes.c_int32), ("limbs_b", ctypes.c_int32),
        ("planes_a", ctypes.c_int32), ("planes_b", ctypes.c_int32),
        ("log2_D", ctypes.c_int32),
        ("c_a", ctypes.c_int32), ("c_b", ctypes.c_int32),
        ("n_g", ctypes.c_int32),
        ("modulus", ctypes.c_int32),
        ("xmin_a", ctypes.c_int32), ("xmax_a", ctypes.c_int32),
        ("xmin_b", ctypes.c_int32), ("xmax_b", ctypes.c_int32),
        ("coverage_a", ctypes.c_int32), ("coverage_b", ctypes.c_int32),
        ("w", ctypes.c_int32 * MAX_LIMBS), ("v", ctypes.c_int32 * MAX_LIMBS),
        ("alpha", (ctypes.c_int32 * MAX_LIMBS) * MAX_PLANES),
        ("beta", (ctypes.c_int32 * MAX_LIMBS) * MAX_PLANES),
        ("pair_a", ctypes.c_int32 * MAX_PRODUCTS), ("pair_b", ctypes.c_int32 * MAX_PRODUCTS),
        ("ell", ctypes.c_int64 * MAX_PRODUCTS),
        ("group", ctypes.c_int32 * MAX_PRODUCTS),
        ("k_star", ctypes.c_int64), ("k_seg", ctypes.c_int64),
        ("format_a", ctypes.c_int32 * MAX_PLANES), ("format_b", ctypes.c_int32 * MAX_PLANES),
    ]


class CacheStruct(ctypes.Structure):  # awe_cache
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p),
                ("num_blocks", ctypes.c_int64),
                ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("block", ctypes.c_int32)]


class BatchStruct(ctypes.Structure):  # awe_batch
    _fields_ = [("sequences", ctypes.c_int32),
                ("starts", ctypes.c_void_p), ("lengths", ctypes.c_void_p), ("blocks", ctypes.c_void_p),
                ("ld_blocks", ctypes.c_int64),
                ("rows", ctypes.c_int64), ("max_rows", ctypes.c_int64), ("max_length", ctypes.c_int64)]


class AweError(RuntimeError):
    def __init__(self, status, where, detail):
        self.status = status
        super().__init__("%s: %s (%d)%s" % (where, _status_string(status), status,
                                            (": " + detail) if detail else ""))


_lib = None
_I32, _I64, _SZ, _P = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p


def lib():
    """The loaded library; raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libawe.so is not built: run `python -m paper_2609_24519_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        L.awe_get_encoding_info.argtypes = [_I32, _I32, ctypes.POINTER(EncodingInfo)]
        L.awe_get_plane_table.argtypes = [_I32, _I32, _I32, _P, _I64]
        L.awe_plane_bytes.argtypes = [_I32, _I32, _I32, _I64, _I64, ctypes.POINTER(_SZ)]
        L.awe_encode.argtypes = [_I32, _I32, _I32, _P, _I64, _I64, _I64, _P, _P, _P]
        L.awe_gemm_planes.argtypes = [_I32, _I32, _I64, _I64, _I64, _P, _P, _P, _I64, _I32, _I64, _P]
        L.awe_workspace_bytes.argtypes = [_I32, _I32, _I64, _I64, _I64, ctypes.POINTER(_SZ)]
        L.awe_gemm_exact.argtypes = [_I32, _I64, _I64, _I64, _P, _I64, _P, _I64, _P, _I64, _I32,
                                     _P, _SZ, _P, _P]
        L.awe_gemm_mod.argtypes = [_I32, _I64, _I64, _I64, _P, _I64, _P, _I64, _P, _I64,
                                   _P, _SZ, _P, _P]
        L.awe_gemm_exact_noalloc.argtypes = [_I32, _I64, _I64, _I64, _P, _I64, _P, _I64, _P, _I64, _I32,
                                             _P, _P]
        L.awe_residues.argtypes = [_P, _I64, _I64, _I64, _I64, _P, _I32, _P, _I64, _P, _P]
        L.awe_crt.argtypes = [_P, _I64, _I64, _I64, _I64, _P, _I32, _P, _P, _I64, _P]
        L.awe_crt_workspace_bytes.argtypes = [_P, _I32, _I64, _I64, _I64, ctypes.POINTER(_SZ)]
        L.awe_gemm_crt.argtypes = [_I64, _I64, _I64, _P, _I64, _P, _I64, _I64, _I64, _P, _I32,
                                   _P, _P, _I64, _P, _SZ, _P, _P]
        L.awe_gemm_w4.argtypes = [_I64, _I64, _I64, _P, _I64, _I32, _P, _P, _I64, _P, _I64, _I32, _P, _I64,
                                  _I64, _P, _I64, _I32, _P]
        L.awe_cache_store.argtypes = [_P, _P, _P, _I64, _I64, _P, _I64, _I64, _I32, _P, _P]
        L.awe_cache_load.argtypes = [_P, _P, _P, _I64, _I64, _P, _I64, _I64, _I32, _P, _P]
        L.awe_cache_attend_workspace_bytes.argtypes = [_P, _P, _I32, ctypes.POINTER(_SZ)]
        L.awe_cache_attend.argtypes = [_P, _P, _P, _I64, _I64, _I32, _I32, ctypes.c_float, _I32, _P, _I64, _I64,
                                       _P, _SZ, _P, _P]
        L.awe_status_string.argtypes = [_I32]
        L.awe_status_string.restype = ctypes.c_char_p
        L.awe_last_error.argtypes = []
        L.awe_last_error.restype = ctypes.c_char_p
        for name in ("awe_get_encoding_info", "awe_get_plane_table", "awe_plane_bytes", "awe_encode",
                     "awe_gemm_planes", "awe_workspace_bytes", "awe_gemm_exact", "awe_gemm_exact_noalloc",
                     "awe_gemm_mod",
                     "awe_residues", "awe_crt", "awe_crt_workspace_bytes", "awe_gemm_crt",
                     "awe_gemm_w4", "awe_cache_store", "awe_cache_load", "awe_cache_attend",
                     "awe_cache_attend_workspace_bytes"):
            getattr(L, name).restype = _I32
        _lib = L
    return _lib


def header_symbols():
    """Names of the functions include/awe.h declares."""
    with open(HEADER) as f:
        text = f.read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(awe_[a-z_0-9]+)\s*\(", text)))


def _status_string(st):
    try:
        return lib().awe_status_string(st).decode()
    except Exception:  # noqa: BLE001 - message only
        return "status"


def _check(st, where):
    if st != OK:
        raise AweError(st, where, lib().awe_last_error().decode())


def _ptr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


_torch_c = None  # torch._C once CUDA is initialised


def _current_stream():
    """Handle of torch's current stream on the current device.  Without the Stream object that
    torch.cuda.current_stream() builds on every call (2.8 us, a quarter of a small product's host time)."""
    global _torch_c
    if _torch_c is None:
        import torch
        handle = torch.cuda.current_stream().cuda_stream  # initialises CUDA
        if hasattr(torch._C, "_cuda_getCurrentRawStream") and hasattr(torch._C, "_cuda_getDevice"):
            _torch_c = torch._C
        return handle
    return _torch_c._cuda_getCurrentRawStream(_torch_c._cuda_getDevice())


def _stream(stream):
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


# ---- host queries -----------------------------------------------------------
def get_encoding_info(enc, modulus=0):
    info = EncodingInfo()
    _check(lib().awe_get_encoding_info(enc, modulus, ctypes.byref(info)), "awe_get_encoding_info")
    r = info.r
    return {
        "r": r, "limbs_a": info.limbs_a, "limbs_b": info.limbs_b,
        "planes_a": info.planes_a, "planes_b": info.planes_b, "log2_D": info.log2_D,
        "c_a": info.c_a, "c_b": info.c_b, "n_g": info.n_g, "modulus": info.modulus,
        "range_a": (info.xmin_a, info.xmax_a), "range_b": (info.xmin_b, info.xmax_b),
        "coverage_a": info.coverage_a, "coverage_b": info.coverage_b,
        "w": tuple(info.w[:info.limbs_a]), "v": tuple(info.v[:info.limbs_b]),
        "alpha": [tuple(info.alpha[k][:info.limbs_a]) for k in range(info.planes_a)],
        "beta": [tuple(info.beta[k][:info.limbs_b]) for k in range(info.planes_b)],
        "pair_a": list(info.pair_a[:r]), "pair_b": list(info.pair_b[:r]),
        "ell": list(info.ell[:r]), "group": list(info.group[:r]),
        "k_star": info.k_star, "k_seg": info.k_seg,
        "formats_a": [_FORMATS[f] for f in info.format_a[:info.planes_a]],
        "formats_b": [_FORMATS[f] for f in info.format_b[:info.planes_b]],
    }


def get_plane_table(enc, modulus, side):
    """(xmin, T) with T[x - xmin, k] the stored value of plane k for input x."""
    info = get_encoding_info(enc, modulus)
    lo, hi = info["range_a"] if side == SIDE_A else info["range_b"]
    npl = info["planes_a"] if side == SIDE_A else info["planes_b"]
    T = np.zeros((hi - lo + 1, npl), dtype=np.int32)
    _check(lib().awe_get_plane_table(enc, modulus, side, T.ctypes.data, T.size), "awe_get_plane_table")
    return lo, T


def plane_bytes(enc, modulus, side, rows, K):
    n = _SZ()
    _check(lib().awe_plane_bytes(enc, modulus, side, rows, K, ctypes.byref(n)), "awe_plane_bytes")
    return n.value


def workspace_bytes(enc, modulus, M, N, K):
    n = _SZ()
    _check(lib().awe_workspace_bytes(enc, modulus, M, N, K, ctypes.byref(n)), "awe_workspace_bytes")
    return n.value


# ---- device calls (same argument order as the C ABI) ----------------------------
def encode(enc, modulus, side, x, rows, K, ld, planes, d_range_flag=None, stream=None):
    _check(lib().awe_encode(enc, modulus, side, _ptr(x), rows, K, ld, _ptr(planes),
                            _ptr(d_range_flag), _stream(stream)), "awe_encode")


def gemm_planes(enc, modulus, M, N, K, planes_a, planes_b, C, ldc, c_type, k_seg=0, stream=None):
    _check(lib().awe_gemm_planes(enc, modulus, M, N, K, _ptr(planes_a), _ptr(planes_b), _ptr(C),
                                 ldc, c_type, k_seg, _stream(stream)), "awe_gemm_planes")


def gemm_exact(enc, M, N, K, A, lda, B, ldb, C, ldc, c_type, workspace, ws_bytes,
               d_range_flag=None, stream=None):
    _check(lib().awe_gemm_exact(enc, M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, c_type,
                                _ptr(workspace), ws_bytes, _ptr(d_range_flag), _stream(stream)),
           "awe_gemm_exact")


def gemm_exact_noalloc(enc, M, N, K, A, lda, B, ldb, C, ldc, c_type, d_range_flag=None, stream=None):
    _check(lib().awe_gemm_exact_noalloc(enc, M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, c_type,
                                        _ptr(d_range_flag), _stream(stream)), "awe_gemm_exact_noalloc")


def gemm_mod(m, M, N, K, A, lda, B, ldb, C, ldc, workspace, ws_bytes, d_range_flag=None, stream=None):
    _check(lib().awe_gemm_mod(m, M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, _ptr(workspace),
                              ws_bytes, _ptr(d_range_flag), _stream(stream)), "awe_gemm_mod")


# ---- residue number system (moduli: a sequence of ints, passed as a host int32 array) ----
def _moduli(moduli):
    arr = (ctypes.c_int32 * len(moduli))(*[int(m) for m in moduli])
    return arr, len(moduli)


def residues(x, rows, cols, ld, bound, moduli, out, out_stride, d_range_flag=None, stream=None):
    arr, n = _moduli(moduli)
    _check(lib().awe_residues(_ptr(x), rows, cols, ld, bound, arr, n, _ptr(out), out_stride,
                              _ptr(d_range_flag), _stream(stream)), "awe_residues")


def crt(res, res_stride, rows, cols, ld_res, moduli, c128=None, c64=None, ldc=None, stream=None):
    arr, n = _moduli(moduli)
    _check(lib().awe_crt(_ptr(res), res_stride, rows, cols, ld_res, arr, n, _ptr(c128), _ptr(c64),
                         cols if ldc is None else ldc, _stream(stream)), "awe_crt")


def crt_workspace_bytes(moduli, M, N, K):
    arr, n = _moduli(moduli)
    out = _SZ(0)
    _check(lib().awe_crt_workspace_bytes(arr, n, M, N, K, ctypes.byref(out)), "awe_crt_workspace_bytes")
    return out.value


def gemm_crt(M, N, K, A, lda, B, ldb, bound_a, bound_b, moduli, c128, c64, ldc, workspace, ws_bytes,
             d_range_flag=None, stream=None):
    arr, n = _moduli(moduli)
    _check(lib().awe_gemm_crt(M, N, K, _ptr(A), lda, _ptr(B), ldb, bound_a, bound_b, arr, n,
                              _ptr(c128), _ptr(c64), ldc, _ptr(workspace), ws_bytes,
                              _ptr(d_range_flag), _stream(stream)), "awe_gemm_crt")


# ---- quantised inference (cache and batch: Cache and Batch below, or their structures) ----------
def _struct(x):  # (bytes are passed as the address of their contents)
    if isinstance(x, ctypes.Structure):
        return ctypes.addressof(x)
    return x.packed if x is not None else None


def gemm_w4(M, N, K, X, ldx, x_type, x_scales, W, ldw, w_scales, lds, s_type, zeros, ldz, group, Y, ldy, y_type,
            stream=None):
    _check(lib().awe_gemm_w4(M, N, K, _ptr(X), ldx, x_type, _ptr(x_scales), _ptr(W), ldw, _ptr(w_scales), lds,
                             s_type, _ptr(zeros), ldz, group, _ptr(Y), ldy, y_type, _stream(stream)), "awe_gemm_w4")


def cache_store(cache, batch, k, k_row, k_head, v, v_row, v_head, dtype, d_range_flag=None, stream=None):
    _check(lib().awe_cache_store(_struct(cache), _struct(batch), _ptr(k), k_row, k_head, _ptr(v), v_row, v_head,
                                 dtype, _ptr(d_range_flag), _stream(stream)), "awe_cache_store")


def cache_load(cache, batch, k, k_row, k_head, v, v_row, v_head, dtype, d_range_flag=None, stream=None):
    _check(lib().awe_cache_load(_struct(cache), _struct(batch), _ptr(k), k_row, k_head, _ptr(v), v_row, v_head,
                                dtype, _ptr(d_range_flag), _stream(stream)), "awe_cache_load")


def cache_attend_workspace_bytes(cache, batch, q_heads):
    n = _SZ()
    _check(lib().awe_cache_attend_workspace_bytes(_struct(cache), _struct(batch), q_heads, ctypes.byref(n)),
           "awe_cache_attend_workspace_bytes")
    return n.value


def cache_attend(cache, batch, q, q_row, q_head, q_heads, dtype, scale, causal, out, out_row, out_head, workspace,
                 ws_bytes, d_range_flag=None, stream=None):
    _check(lib().awe_cache_attend(_struct(cache), _struct(batch), _ptr(q), q_row, q_head, q_heads, dtype, scale,
                                  causal, _ptr(out), out_row, out_head, _ptr(workspace), ws_bytes,
                                  _ptr(d_range_flag), _stream(stream)), "awe_cache_attend")


# ---- torch conveniences (allocation with torch, then the calls above) -------------
def matmul_exact(A, B, enc=ENC_AWE6, out_dtype=None, d_range_flag=None):
    """C = A B exactly for int8 CUDA tensors A (M x K) and B (K x N)."""
    import torch
    M, K = A.shape
    K2, N = B.shape
    if K != K2:
        raise ValueError("inner dimensions differ")
    out_dtype = out_dtype or torch.int32
    c_type = I64 if out_dtype == torch.int64 else I32
    C = torch.empty((M, N), dtype=out_dtype, device=A.device)
    ws_n = workspace_bytes(enc, 0, M, N, K)
    ws = torch.empty(max(ws_n, 1), dtype=torch.uint8, device=A.device)
    gemm_exact(enc, M, N, K, A, A.stride(0), B, B.stride(0), C, C.stride(0), c_type, ws, ws_n,
               d_range_flag)
    return C


def matmul_mod(m, A, B, d_range_flag=None):
    """(A B) mod m for uint8 residue CUDA tensors."""
    import torch
    M, K = A.shape
    _, N = B.shape
    C = torch.empty((M, N), dtype=torch.int32, device=A.device)
    ws_n = workspace_bytes(ENC_MOD, m, M, N, K)
    ws = torch.empty(max(ws_n, 1), dtype=torch.uint8, device=A.device)
    gemm_mod(m, M, N, K, A, A.stride(0), B, B.stride(0), C, C.stride(0), ws, ws_n, d_range_flag)
    return C


def matmul_crt(A, B, moduli, bound_a, bound_b, d_range_flag=None):
    """Exact A B for int64 CUDA tensors through residues; returns (c128, c64): the integer as
    an int64 tensor of shape (M, N, 2) holding (low, high) words, and its nearest double."""
    import torch
    M, K = A.shape
    _, N = B.shape
    c128 = torch.empty((M, N, 2), dtype=torch.int64, device=A.device)
    c64 = torch.empty((M, N), dtype=torch.float64, device=A.device)
    ws_n = crt_workspace_bytes(moduli, M, N, K)
    ws = torch.empty(max(ws_n, 1), dtype=torch.uint8, device=A.device)
    gemm_crt(M, N, K, A, A.stride(0), B, B.stride(0), bound_a, bound_b, moduli, c128, c64, N, ws, ws_n,
             d_range_flag)
    return c128, c64


# ---- quantised inference on torch tensors (for inference: no gradients, tensors that ask for one are refused) ---
_types = {}  # torch dtype -> awe_dtype
_REAL, _REAL16, _REAL16_OR_INT8, _INT32 = (F32, BF16, F16), (BF16, F16), (BF16, F16, I8), (I32,)
_torch = None  # both set when torch is first needed


def _load_torch():
    global _torch
    if _torch is None:
        import torch
        _types.update({torch.int8: I8, torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16,
                       torch.int32: I32})
        _torch = torch


def _dtype(t, allowed):
    if _torch is None:
        _load_torch()
    code = _types.get(t)
    if code not in allowed:
        raise ValueError("element type %s is not supported here" % t)
    return code


def _launch_stream(*tensors):
    """Handle of the current stream; the library launches on the current device, so the tensors must be there, and
    records nothing for a backward pass, so none may ask for a gradient."""
    if _torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError("no gradient is computed here: detach the tensor, or call under torch.no_grad()")
    if _torch_c is None:
        if any(t is not None and t.get_device() < 0 for t in tensors):
            raise ValueError("a tensor is not on the current device")
        _current_stream()  # initialises CUDA the first time
    here = _torch.cuda.current_device() if _torch_c is None else _torch_c._cuda_getDevice()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError("a tensor is not on the current device")
    return _current_stream()


def _rows_2d(t, what):
    """Leading dimension of a matrix with adjacent elements in its rows (a single row may have any stride)."""
    if t.dim() != 2:
        raise ValueError("%s must be a matrix" % what)
    (rows, cols), (ld, one) = t.shape, t.stride()
    if (one != 1 and cols > 1) or (ld < cols and rows > 1):
        raise ValueError("%s must have adjacent elements in its rows, and rows that share no memory" % what)
    return ld if ld > cols and rows > 1 else cols


def matmul_w4(x, w, scales, group, zeros=None, x_scales=None, out_dtype=None):
    """Y = X W^T for CUDA tensors: x (M x K, bfloat16, float16 or int8), w (N x ceil(K / 2), uint8, two
    codes per byte, the low nibble first), scales and zeros (N x ceil(K / group); zeros uint8 or None
    for 8), x_scales (M float32, int8 x only).  out_dtype: x's type, bfloat16 for int8, if not given.
    Computes no gradients."""
    try:
        ((M, K), (ldx, one)), ((N, packed), (ldw, w_one)), (lds, s_one) = \
            (x.shape, x.stride()), (w.shape, w.stride()), scales.stride()
    except ValueError:
        raise ValueError("x, w and scales must be matrices") from None
    if group <= 0:
        raise ValueError("group must be positive")
    groups = -(-K // group)
    x_type = _dtype(x.dtype, _REAL16_OR_INT8)
    s_type = _dtype(scales.dtype, _REAL)
    if out_dtype is None:
        out_dtype = _torch.bfloat16 if x_type == I8 else x.dtype
    y_type = _dtype(out_dtype, _REAL)
    if w.dtype is not _torch.uint8 or packed != (K + 1) // 2:
        raise ValueError("w must be uint8 of N x ceil(K / 2)")
    if scales.shape != (N, groups):
        raise ValueError("scales must be N x ceil(K / group)")
    # (anything but adjacent rows takes a closer look)
    if one != 1 or ldx != K:
        ldx = _rows_2d(x, "x")
    if w_one != 1 or ldw != packed:
        ldw = _rows_2d(w, "w")
    if s_one != 1 or lds != groups:
        lds = _rows_2d(scales, "scales")
    ldz = 0
    if zeros is not None:
        ldz = _rows_2d(zeros, "zeros")
        if zeros.dtype is not _torch.uint8 or zeros.shape != (N, groups):
            raise ValueError("zeros must be uint8 of N x ceil(K / group)")
    if x_scales is not None and (x_scales.dtype != _torch.float32 or x_scales.shape != (M,)
                                 or not x_scales.is_contiguous()):
        raise ValueError("x_scales must be M float32 values")
    stream = _launch_stream(x, w, scales, zeros, x_scales)
    y = x.new_empty((M, N), dtype=out_dtype)
    _check(lib().awe_gemm_w4(M, N, K, x.data_ptr(), ldx, x_type, _ptr(x_scales), w.data_ptr(), ldw, scales.data_ptr(),
                             lds, s_type, _ptr(zeros), ldz, group, y.data_ptr(), N, y_type, stream), "awe_gemm_w4")
    return y


class Cache:
    """An int8 cache of keys and values on CUDA tensors: k (blocks x heads x block x dim) and v (blocks x
    heads x dim x block) int8, k_scales and v_scales (blocks x heads) float32, all contiguous.  Keeps
    the tensors alive; ``Cache.empty`` allocates them."""

    _layout = struct.Struct("@PPPPqiii0q")  # awe_cache

    def __init__(self, k, v, k_scales, v_scales):
        try:
            blocks, heads, block, dim = k.shape
        except ValueError:
            raise ValueError("k must be int8 of blocks x heads x block x dim") from None
        _load_torch()
        if k.dtype is not _torch.int8 or v.dtype is not _torch.int8 or v.shape != (blocks, heads, dim, block):
            raise ValueError("k must be int8 of blocks x heads x block x dim, v of blocks x heads x dim x block")
        at, per_head = k.device, (blocks, heads)
        for s in (k_scales, v_scales):
            if s.dtype is not _torch.float32 or s.shape != per_head:
                raise ValueError("scales must be float32 of blocks x heads")
            if s.requires_grad:
                raise ValueError("scales are written in place and take no gradient")
        for t in (k, v, k_scales, v_scales):
            if not t.is_contiguous() or t.device != at:
                raise ValueError("the cache's tensors must be contiguous, and on one device")
        self.k, self.v, self.k_scales, self.v_scales = k, v, k_scales, v_scales
        self.heads, self.head_dim, self.block = heads, dim, block
        self.packed = self._layout.pack(k.data_ptr(), v.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(),
                                        blocks, heads, dim, block)

    @classmethod
    def empty(cls, num_blocks, heads, head_dim, block, device="cuda"):
        import torch
        return cls(torch.empty((num_blocks, heads, block, head_dim), dtype=torch.int8, device=device),
                   torch.empty((num_blocks, heads, head_dim, block), dtype=torch.int8, device=device),
                   torch.empty((num_blocks, heads), dtype=torch.float32, device=device),
                   torch.empty((num_blocks, heads), dtype=torch.float32, device=device))


class Batch:
    """The sequences of a call on CUDA int32 tensors: starts (sequences + 1), lengths (sequences) and blocks
    (sequences x entries, rows with adjacent entries); rows, max_rows and max_length are plain numbers
    (the rows of the row tensors, and bounds).  Keeps the tensors alive."""

    _layout = struct.Struct("@iPPPqqqq")  # awe_batch

    def __init__(self, starts, lengths, blocks, rows, max_rows, max_length):
        try:
            (offsets,), (n,), (rows_of, entries), (ld, one) = starts.shape, lengths.shape, blocks.shape, blocks.stride()
        except ValueError:
            raise ValueError("starts and lengths must be vectors, blocks a matrix") from None
        if offsets != n + 1 or rows_of != n:
            raise ValueError("starts, lengths and blocks must have sequences + 1, sequences and sequences rows")
        _load_torch()
        at, i32 = starts.device, _torch.int32
        if (starts.dtype is not i32 or lengths.dtype is not i32 or blocks.dtype is not i32 or lengths.device != at
                or blocks.device != at):
            raise ValueError("starts, lengths and blocks must be int32, and on one device")
        if not starts.is_contiguous() or not lengths.is_contiguous():
            raise ValueError("starts and lengths must be contiguous")
        if (one != 1 and entries > 1) or (ld < entries and n > 1):
            ld = _rows_2d(blocks, "blocks")  # (refuses it)
        self.starts, self.lengths, self.blocks, self.rows = starts, lengths, blocks, rows
        # the last row holds `entries` entries, so no position may lie past them
        self.entries, self.max_length = entries, max_length
        try:
            self.packed = self._layout.pack(n, starts.data_ptr(), lengths.data_ptr(), blocks.data_ptr(),
                                            ld if n > 1 else entries, rows, max_rows, max_length)
        except struct.error:
            raise ValueError("rows, max_rows and max_length must be whole numbers of 64 bits") from None


def _row_tensor(t, cache, batch, heads, what):
    stride = t.stride()
    if t.shape != (batch.rows, heads, cache.head_dim) or stride[2] != 1:
        raise ValueError("%s must be rows x %d x %d with adjacent elements in the last dimension"
                         % (what, heads, cache.head_dim))
    return stride[0], stride[1]


def _fits(cache, batch):
    if batch.max_length > batch.entries * cache.block:
        raise ValueError("max_length lies past the block table's entries")


def _flag(t):
    if t is None:
        return None
    _dtype(t.dtype, _INT32)
    return t.data_ptr()


def store_tokens(cache, batch, k, v, d_range_flag=None):
    """Stores k and v (rows x heads x dim) as the newest tokens of the batch's sequences, without gradients."""
    _fits(cache, batch)
    k_row, k_head = _row_tensor(k, cache, batch, cache.heads, "k")
    v_row, v_head = _row_tensor(v, cache, batch, cache.heads, "v")
    if k.dtype is not v.dtype:
        raise ValueError("k and v have different types")
    flag, stream = _flag(d_range_flag), _launch_stream(cache.k, batch.starts, k, v, d_range_flag)
    _check(lib().awe_cache_store(cache.packed, batch.packed, k.data_ptr(), k_row, k_head, v.data_ptr(), v_row, v_head,
                                 _dtype(k.dtype, _REAL), flag, stream), "awe_cache_store")


def load_tokens(cache, batch, dtype, d_range_flag=None):
    """(k, v), rows x heads x dim of dtype: what the newest tokens of the batch's sequences stand for.
    Rows that belong to no sequence are not written."""
    _fits(cache, batch)
    code = _dtype(dtype, _REAL)
    flag, stream = _flag(d_range_flag), _launch_stream(cache.k, batch.starts, d_range_flag)
    heads, dim = cache.heads, cache.head_dim
    k = cache.k.new_empty((batch.rows, heads, dim), dtype=dtype)
    v = _torch.empty_like(k)
    _check(lib().awe_cache_load(cache.packed, batch.packed, k.data_ptr(), heads * dim, dim, v.data_ptr(), heads * dim,
                                dim, code, flag, stream), "awe_cache_load")
    return k, v


def attend(cache, batch, q, scale, causal=True, out=None, d_range_flag=None):
    """Attention of q (rows x query heads x dim) over the cached tokens of the batch's sequences.  Rows that
    belong to no sequence are not written.  out shares no memory with q.  Prompts, and sequences of few rows
    over many tokens, are best two calls.  Computes no gradients."""
    _fits(cache, batch)
    heads = q.shape[1] if q.dim() == 3 else 0
    q_row, q_head = _row_tensor(q, cache, batch, heads, "q")
    dtype = _dtype(q.dtype, _REAL16)
    if out is not None:
        if out.dtype is not q.dtype:
            raise ValueError("out and q have different types")
        out_row, out_head = _row_tensor(out, cache, batch, heads, "out")
    flag, stream = _flag(d_range_flag), _launch_stream(cache.k, batch.starts, q, out, d_range_flag)
    if out is None:
        out = _torch.empty_like(q) if q.is_contiguous() else q.new_empty(q.shape)
        out_row, out_head = heads * cache.head_dim, cache.head_dim

    def call(ws, n):
        return lib().awe_cache_attend(cache.packed, batch.packed, q.data_ptr(), q_row, q_head, heads, dtype, scale,
                                      1 if causal else 0, out.data_ptr(), out_row, out_head, ws, n, flag, stream)
    # most calls need no workspace; those that do are refused, before anything is enqueued
    st = call(None, 0)
    if st == ERR_WORKSPACE:
        n = cache_attend_workspace_bytes(cache, batch, heads)
        ws = q.new_empty(n, dtype=_torch.uint8)
        st = call(ws.data_ptr(), n)
    _check(st, "awe_cache_attend")
    return out
