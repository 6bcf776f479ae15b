"""Thin ctypes binding of ``libmipgemm.so``: same names as ``include/mipgemm.h``.

Argument marshalling only -- every step of the method runs in the CUDA kernels
behind the C ABI.  Tensors are ``torch`` CUDA tensors (or raw device addresses as
``int``); PyTorch is used for device memory and streams, nothing else.  There is
no CPU fallback: if the shared library has not been built, importing this module
raises.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmipgemm.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        "libmipgemm.so is missing (%s). Build it with `python -m paper_2506_11728_b200.build` "
        "or `__graft_entry__.build()`; there is no fallback path." % LIB_PATH)

_lib = ctypes.CDLL(LIB_PATH)

_i64, _int, _vp, _sz = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
_f32, _u64 = ctypes.c_float, ctypes.c_uint64

OK, ERR_INVALID_ARG, ERR_K_TOO_LARGE, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = range(7)
ERR_STATIC_SCRATCH_LIMIT = 7
STATIC_SCRATCH_BYTES = 8 << 20
PATH_NONE, PATH_DENSE, PATH_DENSE_PAIR, PATH_SKINNY, PATH_TRIVIAL = range(5)
PATH_MASK = 0xFF
PATH_REPACK, PATH_SPLITK, PATH_IM2COL_TMA, PATH_IM2COL_EXPLICIT = 0x100, 0x200, 0x400, 0x800
PATH_BATCHED = 0x1000
PATH_IM2COL_GATHER = 0x2000

#: every symbol include/mipgemm.h declares, with (restype, argtypes)
SIGNATURES = {
    "mipgemm_s8s8s32": (_int, [_i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _int, _vp]),
    "mipgemm_u8s8s32": (_int, [_i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _int, _vp]),
    "mipgemm_conv_u8s8s32": (_int, [_i64] * 5 + [_int] * 8 + [_vp, _vp, _vp, _int, _vp]),
    "mipgemm_gemm_ex": (_int, [_int] * 5 + [_i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _int, _vp]),
    "mipgemm_batched_s8s8s32": (_int, [_i64] * 4 + [_vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _int, _vp]),
    "mipgemm_batched_u8s8s32": (_int, [_i64] * 4 + [_vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _int, _vp]),
    "mipgemm_s8s8f32_dequant": (_int, [_i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, ctypes.c_float, _vp]),
    "mipgemm_u8s8f32_dequant": (_int, [_i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, ctypes.c_float, _vp]),
    "mipgemm_conv_u8s8f32_dequant": (_int, [_i64] * 5 + [_int] * 8 + [_vp, _vp, _vp, ctypes.c_float, _vp]),
    "mipgemm_s8s8s8_requant": (_int, [_i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, ctypes.c_float, _int, _vp]),
    "mipgemm_u8s8u8_requant": (_int, [_i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, ctypes.c_float, _vp]),
    "mipgemm_conv_u8s8u8_requant": (_int, [_i64] * 5 + [_int] * 8 + [_vp, _vp, _vp, ctypes.c_float, _vp]),
    "mipgemm_s8s8f32_dequant_bias": (_int, [_i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, ctypes.c_float, _vp, _vp]),
    "mipgemm_u8s8f32_dequant_bias": (_int, [_i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, ctypes.c_float, _vp, _vp]),
    "mipgemm_conv_u8s8f32_dequant_bias": (_int, [_i64] * 5 + [_int] * 8 + [_vp, _vp, _vp, ctypes.c_float, _vp, _vp]),
    "mipgemm_s8s8s8_requant_bias": (_int, [_i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, ctypes.c_float, _int, _vp, _vp]),
    "mipgemm_u8s8u8_requant_bias": (_int, [_i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, ctypes.c_float, _vp, _vp]),
    "mipgemm_conv_u8s8u8_requant_bias": (_int, [_i64] * 5 + [_int] * 8 + [_vp, _vp, _vp, ctypes.c_float, _vp, _vp]),
    "mipgemm_quantize_rows": (_int, [_int, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _vp]),
    "mipgemm_dequantize_rows": (_int, [_int, _i64, _i64, _vp, _i64, _vp, _vp, _i64, _vp]),
    "mipgemm_s8s8_linear": (_int, [_int] * 2 + [_i64] * 3 + [_vp, _i64, _vp] * 2 + [_vp, _vp, _i64, _vp, _i64, _vp]),
    "mipgemm_u8s8_linear": (_int, [_int] * 2 + [_i64] * 3 + [_vp, _i64, _vp] * 2 + [_vp, _vp, _i64, _vp, _i64, _vp]),
    "mipgemm_s8s8_gated": (_int, [_int] * 2 + [_i64] * 3 + [_vp, _i64, _vp] * 3 + [_vp, _i64, _vp]),
    "mipgemm_s8s8_gated_grad": (_int, [_int] * 2 + [_i64] * 3 + [_vp, _i64, _vp] * 3 + [_vp, _i64] * 3 + [_vp]),
    "mipgemm_bf16s8_product": (_int, [_int] * 2 + [_i64] * 3 + [_vp, _i64] * 2 + [_vp, _vp, _i64, _int, _vp]),
    "mipgemm_f8_quantize": (_int, [_int] * 2 + [_i64] * 2 + [_vp, _i64] * 5 + [_vp]),
    "mipgemm_f8_quantize_squares": (_int, [_int] * 2 + [_i64] * 2 + [_vp, _i64] * 3 + [_vp]),
    "mipgemm_f8_dequantize": (_int, [_int] * 3 + [_i64] * 2 + [_vp, _i64] * 3 + [_vp]),
    "mipgemm_f8f8_product": (_int, [_int] * 6 + [_i64] * 3 + [_vp, _i64] * 4 + [_vp] + [_vp, _i64] * 2 + [_vp]),
    "mipgemm_norm_step": (_int, [_int] * 3 + [_i64] * 2 + [_f32, _vp, _i64, _f32, _vp, _i64, _vp, _vp, _vp, _i64, _i64, _f32, _u64, _vp,
                                                           _vp, _vp, _vp, _i64, _vp, _i64, _int, _vp, _i64, _vp, _i64, _vp, _vp]),
    "mipgemm_norm_step_grad": (_int, [_int] * 3 + [_i64] * 2 + [_vp, _i64] * 3 + [_vp, _f32, _vp, _i64, _vp, _vp, _vp, _i64, _i64, _f32, _u64,
                                                                _vp, _vp] + [_vp, _i64] * 3 + [_vp] * 5),
    "mipgemm_host_s8s8s32": (_int, [_i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _int, _vp]),
    "mipgemm_host_u8s8s32": (_int, [_i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _int, _vp]),
    "mipgemm_s8s8s32_static_scratch": (_int, [_i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _int, _vp]),
    "mipgemm_launch_count": (ctypes.c_uint64, []),
    "mipgemm_device_status": (_int, [_vp]),
    "mipgemm_set_workspace": (_int, [_vp, _sz]),
    "mipgemm_workspace_query_gemm": (_sz, [_i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _int]),
    "mipgemm_workspace_query_conv": (_sz, [_i64] * 5 + [_int] * 8),
    "mipgemm_last_path": (_int, []),
    "mipgemm_last_cuda_error": (_int, []),
    "mipgemm_status_string": (ctypes.c_char_p, [_int]),
    "mipgemm_version": (_int, []),
    "mipgemm_probe_i8_peak": (_int, [_int, ctypes.POINTER(_int), ctypes.POINTER(ctypes.c_double), _vp, _vp]),
    "mipgemm_set_tuning": (_int, [_int, _int, _int, _int]),
    "mipgemm_set_weights_constant": (_int, [_int]),
    "mipgemm_register_constant_weights": (_int, [_vp, _sz]),
    "mipgemm_unregister_constant_weights": (_int, [_vp]),
    "mipgemm_static_scratch_status": (_int, [_vp]),
    "mipgemm_release_staging": (_int, []),
    "mipgemm_debug_set": (_int, [_int, ctypes.c_ulonglong]),
    "mipgemm_plan_cache_stats": (_int, [ctypes.POINTER(ctypes.c_uint64), ctypes.POINTER(ctypes.c_uint64)]),
}
for _name, (_res, _args) in SIGNATURES.items():
    _fn = getattr(_lib, _name)
    _fn.restype = _res
    _fn.argtypes = _args


class MipGemmError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__("libmipgemm: %s (status %d, cuda error %d)" % (
            mipgemm_status_string(status), status, mipgemm_last_cuda_error()))


def _ptr(x) -> int:
    if x is None:
        return 0
    if isinstance(x, int):
        return x
    return x.data_ptr()


_current_device = _current_stream = None


def _stream(stream) -> int:
    if stream is None:
        # the current stream's handle without a Stream object around it (0.3 us a call instead of 3); the two functions
        # are looked up once CUDA is initialised
        global _current_device, _current_stream
        if _current_stream is None:
            import torch
            if not torch.cuda.is_initialized():
                return torch.cuda.current_stream().cuda_stream
            _current_device, _current_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
        return _current_stream(_current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(status: int, check: bool) -> int:
    if check and status != OK:
        raise MipGemmError(status)
    return status


def mipgemm_s8s8s32(M, N, K, A, lda, B, ldb, C, ldc, accumulate=0, stream=None, check=True) -> int:
    """C[int32, MxN, pitch ldc] (+)= A[int8, MxK row-major, pitch lda] * B[int8, KxN column-major, pitch ldb]."""
    return _check(_lib.mipgemm_s8s8s32(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                       int(bool(accumulate)), _stream(stream)), check)


def mipgemm_u8s8s32(M, N, K, A, lda, B, ldb, C, ldc, accumulate=0, stream=None, check=True) -> int:
    """Same with unsigned 8-bit A."""
    return _check(_lib.mipgemm_u8s8s32(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                       int(bool(accumulate)), _stream(stream)), check)


def mipgemm_conv_u8s8s32(Nb, H, W, Cin, Cout, R, S, stride_h, stride_w, pad_h, pad_w, dil_h, dil_w,
                         X, Wt, Y, accumulate=0, stream=None, check=True) -> int:
    """Y[int32 NHWC] (+)= Conv(Wt[int8 KRSC], X[uint8 NHWC])."""
    return _check(_lib.mipgemm_conv_u8s8s32(Nb, H, W, Cin, Cout, R, S, stride_h, stride_w, pad_h, pad_w,
                                            dil_h, dil_w, _ptr(X), _ptr(Wt), _ptr(Y),
                                            int(bool(accumulate)), _stream(stream)), check)


K_CONTIGUOUS, MN_CONTIGUOUS = 0, 1


def mipgemm_gemm_ex(a_unsigned, b_unsigned, a_order, b_order, c_col_major, M, N, K, A, lda, B, ldb, C, ldc,
                    accumulate=0, stream=None, check=True) -> int:
    """General GEMM: any signedness pair, either storage order for A and B, row- or column-major C."""
    return _check(_lib.mipgemm_gemm_ex(int(a_unsigned), int(b_unsigned), int(a_order), int(b_order),
                                       int(c_col_major), M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                       int(bool(accumulate)), _stream(stream)), check)


def mipgemm_batched_s8s8s32(batch, M, N, K, A, lda, stride_a, B, ldb, stride_b, C, ldc, stride_c,
                            accumulate=0, stream=None, check=True) -> int:
    """C_b (+)= A_b * B_b for b < batch; member b of X starts stride_x elements after member b-1."""
    return _check(_lib.mipgemm_batched_s8s8s32(batch, M, N, K, _ptr(A), lda, stride_a, _ptr(B), ldb, stride_b,
                                               _ptr(C), ldc, stride_c, int(bool(accumulate)), _stream(stream)), check)


def mipgemm_batched_u8s8s32(batch, M, N, K, A, lda, stride_a, B, ldb, stride_b, C, ldc, stride_c,
                            accumulate=0, stream=None, check=True) -> int:
    return _check(_lib.mipgemm_batched_u8s8s32(batch, M, N, K, _ptr(A), lda, stride_a, _ptr(B), ldb, stride_b,
                                               _ptr(C), ldc, stride_c, int(bool(accumulate)), _stream(stream)), check)


def mipgemm_s8s8s8_requant(M, N, K, A, lda, B, ldb, C, ldc, scale, relu=0, stream=None, check=True) -> int:
    """C[int8] = sat(rne(scale * (A * B))) (clamped at 0 from below with relu)."""
    return _check(_lib.mipgemm_s8s8s8_requant(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                              float(scale), int(bool(relu)), _stream(stream)), check)


def mipgemm_u8s8u8_requant(M, N, K, A, lda, B, ldb, C, ldc, scale, stream=None, check=True) -> int:
    """C[uint8] = sat(rne(scale * (A * B))), A unsigned."""
    return _check(_lib.mipgemm_u8s8u8_requant(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                              float(scale), _stream(stream)), check)


def mipgemm_conv_u8s8u8_requant(Nb, H, W, Cin, Cout, R, S, stride_h, stride_w, pad_h, pad_w, dil_h, dil_w,
                                X, Wt, Y, scale, stream=None, check=True) -> int:
    """Y[uint8 NHWC] = sat(rne(scale * Conv(Wt, X)))."""
    return _check(_lib.mipgemm_conv_u8s8u8_requant(Nb, H, W, Cin, Cout, R, S, stride_h, stride_w, pad_h, pad_w,
                                                   dil_h, dil_w, _ptr(X), _ptr(Wt), _ptr(Y), float(scale),
                                                   _stream(stream)), check)


def mipgemm_s8s8f32_dequant_bias(M, N, K, A, lda, B, ldb, C, ldc, scale, bias, stream=None, check=True) -> int:
    """C[float32] = scale * (A * B + bias[column])."""
    return _check(_lib.mipgemm_s8s8f32_dequant_bias(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                                    float(scale), _ptr(bias), _stream(stream)), check)


def mipgemm_u8s8f32_dequant_bias(M, N, K, A, lda, B, ldb, C, ldc, scale, bias, stream=None, check=True) -> int:
    """C[float32] = scale * (A * B + bias[column]), A unsigned."""
    return _check(_lib.mipgemm_u8s8f32_dequant_bias(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                                    float(scale), _ptr(bias), _stream(stream)), check)


def mipgemm_conv_u8s8f32_dequant_bias(Nb, H, W, Cin, Cout, R, S, stride_h, stride_w, pad_h, pad_w, dil_h, dil_w,
                                      X, Wt, Y, scale, bias, stream=None, check=True) -> int:
    """Y[float32 NHWC] = scale * (Conv(Wt, X) + bias[channel])."""
    return _check(_lib.mipgemm_conv_u8s8f32_dequant_bias(Nb, H, W, Cin, Cout, R, S, stride_h, stride_w, pad_h, pad_w,
                                                         dil_h, dil_w, _ptr(X), _ptr(Wt), _ptr(Y), float(scale),
                                                         _ptr(bias), _stream(stream)), check)


def mipgemm_s8s8s8_requant_bias(M, N, K, A, lda, B, ldb, C, ldc, scale, bias, relu=0, stream=None, check=True) -> int:
    """C[int8] = sat(rne(scale * (A * B + bias[column]))) (clamped at 0 from below with relu)."""
    return _check(_lib.mipgemm_s8s8s8_requant_bias(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                                   float(scale), int(bool(relu)), _ptr(bias), _stream(stream)), check)


def mipgemm_u8s8u8_requant_bias(M, N, K, A, lda, B, ldb, C, ldc, scale, bias, stream=None, check=True) -> int:
    """C[uint8] = sat(rne(scale * (A * B + bias[column]))), A unsigned."""
    return _check(_lib.mipgemm_u8s8u8_requant_bias(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                                   float(scale), _ptr(bias), _stream(stream)), check)


def mipgemm_conv_u8s8u8_requant_bias(Nb, H, W, Cin, Cout, R, S, stride_h, stride_w, pad_h, pad_w, dil_h, dil_w,
                                     X, Wt, Y, scale, bias, stream=None, check=True) -> int:
    """Y[uint8 NHWC] = sat(rne(scale * (Conv(Wt, X) + bias[channel])))."""
    return _check(_lib.mipgemm_conv_u8s8u8_requant_bias(Nb, H, W, Cin, Cout, R, S, stride_h, stride_w, pad_h, pad_w,
                                                        dil_h, dil_w, _ptr(X), _ptr(Wt), _ptr(Y), float(scale),
                                                        _ptr(bias), _stream(stream)), check)


def mipgemm_s8s8f32_dequant(M, N, K, A, lda, B, ldb, C, ldc, scale, stream=None, check=True) -> int:
    """C[float32] = scale * (A * B): the exact int32 sum, converted and scaled in the epilogue."""
    return _check(_lib.mipgemm_s8s8f32_dequant(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                               float(scale), _stream(stream)), check)


def mipgemm_u8s8f32_dequant(M, N, K, A, lda, B, ldb, C, ldc, scale, stream=None, check=True) -> int:
    return _check(_lib.mipgemm_u8s8f32_dequant(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                               float(scale), _stream(stream)), check)


def mipgemm_conv_u8s8f32_dequant(Nb, H, W, Cin, Cout, R, S, stride_h, stride_w, pad_h, pad_w, dil_h, dil_w,
                                 X, Wt, Y, scale, stream=None, check=True) -> int:
    return _check(_lib.mipgemm_conv_u8s8f32_dequant(Nb, H, W, Cin, Cout, R, S, stride_h, stride_w, pad_h, pad_w,
                                                    dil_h, dil_w, _ptr(X), _ptr(Wt), _ptr(Y), float(scale),
                                                    _stream(stream)), check)


#: mipgemm_type_t and mipgemm_activation_t by name
TYPES = {"f32": 0, "f16": 1, "bf16": 2}
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}


def mipgemm_quantize_rows(type, M, N, X, ldx, Q, ldq, scale, stream=None, check=True) -> int:
    """Q[int8] = rne(X * 127 / rowmax), scale[row] = rowmax / 127."""
    return _check(_lib.mipgemm_quantize_rows(type, M, N, _ptr(X), ldx, _ptr(Q), ldq, _ptr(scale), _stream(stream)), check)


def mipgemm_dequantize_rows(type, M, N, Q, ldq, scale, X, ldx, stream=None, check=True) -> int:
    """X = diag(scale) Q."""
    return _check(_lib.mipgemm_dequantize_rows(type, M, N, _ptr(Q), ldq, _ptr(scale), _ptr(X), ldx, _stream(stream)),
                  check)


def mipgemm_s8s8_linear(type, act, M, N, K, A, lda, a_scale, B, ldb, b_scale, bias, residual, ldr, C, ldc, stream=None,
                        check=True) -> int:
    """C = act(a_scale[row] * b_scale[column] * (A * B) + bias[column]) + residual; scales, bias and residual may be None."""
    return _check(_lib.mipgemm_s8s8_linear(type, act, M, N, K, _ptr(A), lda, _ptr(a_scale), _ptr(B), ldb, _ptr(b_scale),
                                           _ptr(bias), _ptr(residual), ldr, _ptr(C), ldc, _stream(stream)), check)


def mipgemm_u8s8_linear(type, act, M, N, K, A, lda, a_scale, B, ldb, b_scale, bias, residual, ldr, C, ldc, stream=None,
                        check=True) -> int:
    """Same with unsigned 8-bit A."""
    return _check(_lib.mipgemm_u8s8_linear(type, act, M, N, K, _ptr(A), lda, _ptr(a_scale), _ptr(B), ldb, _ptr(b_scale),
                                           _ptr(bias), _ptr(residual), ldr, _ptr(C), ldc, _stream(stream)), check)


def mipgemm_s8s8_gated(type, act, M, F, K, X, ldx, x_scale, Wg, ldg, g_scale, Wu, ldu, u_scale, H, ldh, stream=None,
                       check=True) -> int:
    """H = act(x_scale[row] * g_scale[column] * (X * Wg)) * (x_scale[row] * u_scale[column] * (X * Wu))."""
    return _check(_lib.mipgemm_s8s8_gated(type, act, M, F, K, _ptr(X), ldx, _ptr(x_scale), _ptr(Wg), ldg, _ptr(g_scale),
                                          _ptr(Wu), ldu, _ptr(u_scale), _ptr(H), ldh, _stream(stream)), check)


def mipgemm_s8s8_gated_grad(type, act, M, F, K, X, ldx, x_scale, Wg, ldg, g_scale, Wu, ldu, u_scale, dH, lddh, dG, lddg,
                            dU, lddu, stream=None, check=True) -> int:
    """dG = dH * U * act'(G), dU = dH * act(G), with G and U recomputed from the codes."""
    return _check(_lib.mipgemm_s8s8_gated_grad(type, act, M, F, K, _ptr(X), ldx, _ptr(x_scale), _ptr(Wg), ldg,
                                               _ptr(g_scale), _ptr(Wu), ldu, _ptr(u_scale), _ptr(dH), lddh, _ptr(dG), lddg,
                                               _ptr(dU), lddu, _stream(stream)), check)


def mipgemm_bf16s8_product(type, a_order, M, N, K, A, lda, B, ldb, b_scale, C, ldc, accumulate=0, stream=None,
                           check=True) -> int:
    """C (+)= A[bf16] * diag(b_scale) * B[int8, K x N row-major]; a_order K_CONTIGUOUS or MN_CONTIGUOUS."""
    return _check(_lib.mipgemm_bf16s8_product(type, a_order, M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(b_scale), _ptr(C),
                                              ldc, int(bool(accumulate)), _stream(stream)), check)


#: mipgemm_f8_format_t, mipgemm_f8_blocks_t, mipgemm_norm_t and mipgemm_codes_t by name
F8_FORMATS = {"e4m3": 0, "e5m2": 1}
F8_BLOCKS = {"rows": 0, "columns": 1, "squares": 2}
NORMS = {"none": 0, "rms": 1, "layer": 2}
CODES = {"none": 0, "s8": 1, "e4m3": 2, "e5m2": 3}


def mipgemm_f8_quantize(type, format, M, N, X, ldx, Qr, ldqr, r_scale, ldrs, Qc, ldqc, c_scale, ldcs, stream=None, check=True) -> int:
    """8-bit floating-point codes with a scale for each block of 128 along the rows (Qr), along the columns (Qc), or both."""
    return _check(_lib.mipgemm_f8_quantize(type, format, M, N, _ptr(X), ldx, _ptr(Qr), ldqr, _ptr(r_scale), ldrs, _ptr(Qc), ldqc,
                                           _ptr(c_scale), ldcs, _stream(stream)), check)


def mipgemm_f8_quantize_squares(type, format, M, N, X, ldx, Q, ldq, scale, lds, stream=None, check=True) -> int:
    """8-bit floating-point codes with a scale for each square of 128 x 128."""
    return _check(_lib.mipgemm_f8_quantize_squares(type, format, M, N, _ptr(X), ldx, _ptr(Q), ldq, _ptr(scale), lds, _stream(stream)),
                  check)


def mipgemm_f8_dequantize(type, format, blocks, M, N, Q, ldq, scale, lds, X, ldx, stream=None, check=True) -> int:
    """X = codes times their blocks' scales."""
    return _check(_lib.mipgemm_f8_dequantize(type, format, blocks, M, N, _ptr(Q), ldq, _ptr(scale), lds, _ptr(X), ldx, _stream(stream)),
                  check)


def mipgemm_f8f8_product(type, a_format, b_format, a_order, b_order, b_blocks, M, N, K, A, lda, a_scale, ldas, B, ldb, b_scale, ldbs, bias,
                         residual, ldr, C, ldc, stream=None, check=True) -> int:
    """C = sum over blocks of 128 k of a_scale * b_scale * (A * B) + bias[column] + residual; scales, bias and residual may be None."""
    return _check(_lib.mipgemm_f8f8_product(type, a_format, b_format, a_order, b_order, b_blocks, M, N, K, _ptr(A), lda, _ptr(a_scale), ldas,
                                            _ptr(B), ldb, _ptr(b_scale), ldbs, _ptr(bias), _ptr(residual), ldr, _ptr(C), ldc,
                                            _stream(stream)), check)


def mipgemm_norm_step(type, post, pre, M, N, eps=1e-5, X=None, ldx=0, x_scale=1.0, Z=None, ldz=0, post_weight=None, post_bias=None,
                      gate=None, ldgate=0, gate_rows=1, drop=0.0, seed=0, counter=None, pre_weight=None, pre_bias=None, Y=None, ldy=0,
                      H=None, ldh=0, codes=0, Q=None, ldq=0, q_scale=None, ldqs=0, stats=None, stream=None, check=True) -> int:
    """Y = x_scale * X + dropout(gate * post(Z)), H = pre(Y), as values and / or codes."""
    # (None is passed on as it is: most of the pointers usually are)
    return _check(_lib.mipgemm_norm_step(type, post, pre, M, N, eps, X if X is None else _ptr(X), ldx, x_scale, Z if Z is None else _ptr(Z), ldz,
                                         post_weight if post_weight is None else _ptr(post_weight), post_bias if post_bias is None else _ptr(post_bias),
                                         gate if gate is None else _ptr(gate), ldgate, gate_rows, drop, seed, counter if counter is None else _ptr(counter),
                                         pre_weight if pre_weight is None else _ptr(pre_weight), pre_bias if pre_bias is None else _ptr(pre_bias),
                                         Y if Y is None else _ptr(Y), ldy, H if H is None else _ptr(H), ldh, codes, Q if Q is None else _ptr(Q), ldq,
                                         q_scale if q_scale is None else _ptr(q_scale), ldqs, stats if stats is None else _ptr(stats),
                                         _stream(stream)), check)


def mipgemm_norm_step_grad(type, post, pre, M, N, dY=None, lddy=0, dH=None, lddh=0, Y=None, ldy=0, pre_weight=None, x_scale=1.0, Z=None,
                           ldz=0, post_weight=None, post_bias=None, gate=None, ldgate=0, gate_rows=1, drop=0.0, seed=0, counter=None,
                           stats=None, dX=None, lddx=0, dZ=None, lddz=0, dgate=None, lddgate=0, dpost_weight=None, dpost_bias=None,
                           dpre_weight=None, dpre_bias=None, stream=None, check=True) -> int:
    """Gradients of that step's X, Z, gate, weights and biases from those of Y and H."""
    return _check(_lib.mipgemm_norm_step_grad(type, post, pre, M, N, _ptr(dY), lddy, _ptr(dH), lddh, _ptr(Y), ldy, _ptr(pre_weight), x_scale,
                                              _ptr(Z), ldz, _ptr(post_weight), _ptr(post_bias), _ptr(gate), ldgate, gate_rows, drop, seed,
                                              _ptr(counter), _ptr(stats), _ptr(dX), lddx, _ptr(dZ), lddz, _ptr(dgate), lddgate,
                                              _ptr(dpost_weight), _ptr(dpost_bias), _ptr(dpre_weight), _ptr(dpre_bias),
                                              _stream(stream)), check)


def mipgemm_host_s8s8s32(M, N, K, A, lda, B, ldb, C, ldc, accumulate=0, stream=None, check=True) -> int:
    """Host-buffer variant: A, B, C are host tensors/arrays (``data_ptr()``) or raw host addresses;
    copies in, computes on the device, copies C back and synchronises."""
    return _check(_lib.mipgemm_host_s8s8s32(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                            int(bool(accumulate)), _stream(stream)), check)


def mipgemm_host_u8s8s32(M, N, K, A, lda, B, ldb, C, ldc, accumulate=0, stream=None, check=True) -> int:
    return _check(_lib.mipgemm_host_u8s8s32(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                            int(bool(accumulate)), _stream(stream)), check)


def mipgemm_s8s8s32_static_scratch(M, N, K, A, lda, B, ldb, C, ldc, accumulate=0, stream=None, check=True) -> int:
    """mipgemm_s8s8s32 for callers that may not allocate device memory: re-pitching scratch comes from
    a fixed STATIC_SCRATCH_BYTES array inside the library (one per GPU, shared by all calls -- calls
    that can overlap on the GPU race on it).  Returns ERR_STATIC_SCRATCH_LIMIT, having launched
    nothing, when the operands need more than that.  Make the first call on a device outside any
    stream capture."""
    return _check(_lib.mipgemm_s8s8s32_static_scratch(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                                      int(bool(accumulate)), _stream(stream)), check)


def mipgemm_launch_count() -> int:
    return int(_lib.mipgemm_launch_count())


def mipgemm_device_status(stream=None) -> int:
    return _lib.mipgemm_device_status(_stream(stream))


def mipgemm_set_workspace(buf, nbytes: int = 0) -> int:
    return _lib.mipgemm_set_workspace(_ptr(buf), nbytes)


def mipgemm_workspace_query_gemm(M, N, K, A, lda, B, ldb, C, ldc, accumulate=0) -> int:
    return _lib.mipgemm_workspace_query_gemm(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                             int(bool(accumulate)))


def mipgemm_workspace_query_conv(Nb, H, W, Cin, Cout, R, S, stride_h, stride_w, pad_h, pad_w,
                                 dil_h, dil_w) -> int:
    return _lib.mipgemm_workspace_query_conv(Nb, H, W, Cin, Cout, R, S, stride_h, stride_w, pad_h, pad_w,
                                             dil_h, dil_w)


def mipgemm_last_path() -> int:
    return _lib.mipgemm_last_path()


def mipgemm_last_cuda_error() -> int:
    return _lib.mipgemm_last_cuda_error()


def mipgemm_status_string(status: int) -> str:
    return _lib.mipgemm_status_string(status).decode()


def mipgemm_version() -> int:
    return _lib.mipgemm_version()


def mipgemm_probe_i8_peak(iters: int, sink, stream=None):
    """Launches the tensor-pipe probe; returns (grid, ops_per_launch)."""
    grid = _int(0)
    ops = ctypes.c_double(0.0)
    st = _lib.mipgemm_probe_i8_peak(iters, ctypes.byref(grid), ctypes.byref(ops), _ptr(sink), _stream(stream))
    _check(st, True)
    return grid.value, ops.value


def mipgemm_set_weights_constant(on) -> int:
    """Promise that B of later M <= 16 calls is never written by work still pending on the stream."""
    return _check(_lib.mipgemm_set_weights_constant(int(bool(on))), True)


def mipgemm_register_constant_weights(buf, nbytes: int = 0, check=True) -> int:
    """Declares [buf, buf + nbytes) constant: M <= 16 calls whose B lies inside it may fetch it early.
    ``nbytes`` defaults to the tensor's size."""
    if not nbytes and hasattr(buf, "numel"):
        nbytes = buf.numel() * buf.element_size()
    return _check(_lib.mipgemm_register_constant_weights(_ptr(buf), nbytes), check)


def mipgemm_unregister_constant_weights(buf, check=True) -> int:
    return _check(_lib.mipgemm_unregister_constant_weights(_ptr(buf)), check)


def mipgemm_release_staging() -> int:
    """Frees the device staging buffer the host-buffer entry points keep between calls."""
    return _check(_lib.mipgemm_release_staging(), True)


def mipgemm_debug_set(flags=0, wait_budget_ns=0) -> int:
    """Test hook: withhold a device-side signal (bit 0) and set the limit of device-side waits (0 = 4 s)."""
    return _check(_lib.mipgemm_debug_set(int(flags), int(wait_budget_ns)), True)


def mipgemm_plan_cache_stats():
    """(enabled, hits, misses) of the plan / tensor-map cache."""
    hits, misses = ctypes.c_uint64(0), ctypes.c_uint64(0)
    on = _lib.mipgemm_plan_cache_stats(ctypes.byref(hits), ctypes.byref(misses))
    return bool(on), hits.value, misses.value


def mipgemm_static_scratch_status(stream=None) -> int:
    """Allocation-free status query of mipgemm_s8s8s32_static_scratch (synchronises the stream)."""
    return _lib.mipgemm_static_scratch_status(_stream(stream))


def mipgemm_set_tuning(block_n=0, stages=0, split_k=0, force_path=0) -> int:
    return _check(_lib.mipgemm_set_tuning(block_n, stages, split_k, force_path), True)
