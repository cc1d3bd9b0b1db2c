"""ctypes binding of libaf1_head.so (include/af1_head.h): the 8-bit
block-scaled linear, the log probabilities of given tokens and the KL
divergence to a teacher.  Argument marshalling only; every step runs in the
library.  Loading raises when the library has not been built: there is no
fallback path."""
import ctypes
import os

from .af1 import AF1_OK, Af1Error, _addr, _stream

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libaf1_head.so")
AF1_FP8_E4M3, AF1_FP8_E5M2 = 0, 1
AF1_HEAD_MAX_TOKENS = 1 << 20
AF1_HEAD_MAX_VOCAB = 1 << 24
AF1_HEAD_MAX_TOP = 32
_lib = None


class af1_fp8_matrix(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("format", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("codes", ctypes.c_void_p),
                ("scales", ctypes.c_void_p)]


def lib():
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build() "
                           "(there is no fallback path)")
    L = ctypes.CDLL(LIB_PATH)
    P, I64, I32, SZ, F = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t,
                          ctypes.c_float)
    M = ctypes.POINTER(af1_fp8_matrix)
    sizes = {"af1_fp8_code_bytes": [I64, I64], "af1_fp8_scale_bytes": [I64, I64],
             "af1_fp8_linear_workspace_bytes": [I64, I64, I64],
             "af1_token_logprobs_workspace_bytes": [I64, I64, I32],
             "af1_distill_kl_workspace_bytes": [I64, I64]}
    calls = {"af1_fp8_quantize": [P, I32, I64, I64, I32, P, P, P],
             "af1_fp8_dequantize": [M, P, I32, P],
             "af1_fp8_transpose": [M, P, P, P],
             "af1_fp8_linear": [M, P, I32, I32, I64, P, I32, P, SZ, P],
             "af1_token_logprobs": [P, I32, I64, I64, I64, F, P, P, P, P, I32, P, P, P, P, SZ, P],
             "af1_token_logprobs_backward": [P, I32, I64, I64, I64, F, P, P, P, P, P, I64, P],
             "af1_distill_kl": [P, P, I32, I64, I64, I64, I64, F, P, P, P, I64, P, SZ, P]}
    for names, restype in ((sizes, SZ), (calls, I32)):
        for name, args in names.items():
            getattr(L, name).argtypes = args
            getattr(L, name).restype = restype
    _lib = L
    return L


def _ret(st, name, check):
    if check and st != AF1_OK:
        raise Af1Error(st, name)
    return st


def _ref(W):
    return ctypes.byref(W) if W is not None else None


def make_matrix(rows, cols, fmt, codes, scales) -> af1_fp8_matrix:
    """The C descriptor of one 8-bit matrix (device arrays)."""
    return af1_fp8_matrix(rows, cols, fmt, 0, _addr(codes), _addr(scales))


def af1_fp8_code_bytes(rows, cols) -> int:
    return int(lib().af1_fp8_code_bytes(rows, cols))


def af1_fp8_scale_bytes(rows, cols) -> int:
    return int(lib().af1_fp8_scale_bytes(rows, cols))


def af1_fp8_quantize(src, src_dtype, rows, cols, fmt, codes, scales, stream=None, check=True):
    return _ret(lib().af1_fp8_quantize(_addr(src), src_dtype, rows, cols, fmt, _addr(codes),
                                       _addr(scales), _stream(stream)), "af1_fp8_quantize", check)


def af1_fp8_dequantize(W, dst, dst_dtype, stream=None, check=True):
    return _ret(lib().af1_fp8_dequantize(_ref(W), _addr(dst), dst_dtype, _stream(stream)),
                "af1_fp8_dequantize", check)


def af1_fp8_transpose(W, codes, scales, stream=None, check=True):
    return _ret(lib().af1_fp8_transpose(_ref(W), _addr(codes), _addr(scales), _stream(stream)),
                "af1_fp8_transpose", check)


def af1_fp8_linear_workspace_bytes(m, n, T) -> int:
    return int(lib().af1_fp8_linear_workspace_bytes(m, n, T))


def af1_fp8_linear(W, x, x_dtype, x_format, T, y, y_dtype, ws, ws_bytes, stream=None, check=True):
    return _ret(lib().af1_fp8_linear(_ref(W), _addr(x), x_dtype, x_format, T, _addr(y), y_dtype,
                                     _addr(ws), ws_bytes, _stream(stream)), "af1_fp8_linear",
                check)


def af1_token_logprobs_workspace_bytes(T, V, k) -> int:
    return int(lib().af1_token_logprobs_workspace_bytes(T, V, k))


def af1_token_logprobs(logits, dtype, T, V, ld, scale, targets, logprob, entropy, lse, k,
                       top_logprob, top_index, saved, ws, ws_bytes, stream=None, check=True):
    return _ret(lib().af1_token_logprobs(_addr(logits), dtype, T, V, ld, scale, _addr(targets),
                                         _addr(logprob), _addr(entropy), _addr(lse), k,
                                         _addr(top_logprob), _addr(top_index), _addr(saved),
                                         _addr(ws), ws_bytes, _stream(stream)),
                "af1_token_logprobs", check)


def af1_token_logprobs_backward(logits, dtype, T, V, ld, scale, targets, saved, g_logprob,
                                g_entropy, dlogits, ldd, stream=None, check=True):
    return _ret(lib().af1_token_logprobs_backward(_addr(logits), dtype, T, V, ld, scale,
                                                  _addr(targets), _addr(saved), _addr(g_logprob),
                                                  _addr(g_entropy), _addr(dlogits), ldd,
                                                  _stream(stream)),
                "af1_token_logprobs_backward", check)


def af1_distill_kl_workspace_bytes(T, V) -> int:
    return int(lib().af1_distill_kl_workspace_bytes(T, V))


def af1_distill_kl(student, teacher, dtype, T, V, ld_s, ld_t, scale, weight, kl, dstudent, ldd,
                   ws, ws_bytes, stream=None, check=True):
    return _ret(lib().af1_distill_kl(_addr(student), _addr(teacher), dtype, T, V, ld_s, ld_t,
                                     scale, _addr(weight), _addr(kl), _addr(dstudent), ldd,
                                     _addr(ws), ws_bytes, _stream(stream)), "af1_distill_kl",
                check)
