"""MI355X-native load-compute-pipelined GEMM / BMM / implicit-GEMM conv2d (ALCOP, arXiv 2210.16691), and the linear
layers, norms, 8-bit rows, experts' products and loss of a transformer around them.

Thin binding over ``libalcop.so`` (C ABI declared in ``include/alcop.h``).  Argument marshalling
only (the hot entry points' in C++, the rest with ctypes): every step of the hot path runs in the
HIP kernels.  PyTorch is used for device
memory and streams.  There is no CPU fallback: if the shared library is missing, importing the
binding's functions raises.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libalcop.so")

F16, BF16, F32, E4M3 = 0, 1, 2, 3
FP32_SUMS = 16           # added to alcop_linear_tail's act
OP_GEMM, OP_BMM, OP_CONV2D = 0, 1, 2

OK = 0
ERR_NULL, ERR_DTYPE, ERR_ALIGN, ERR_SHAPE, ERR_SCHED, ERR_LAUNCH, ERR_UNSUPPORTED, ERR_SIZE, ERR_IO = (
    -1, -2, -3, -4, -5, -6, -7, -8, -9)

EXPORTS = [
    "alcop_gemm", "alcop_bmm", "alcop_gemm_fused", "alcop_bmm_fused", "alcop_conv2d_igemm", "alcop_sched_supported", "alcop_sched_space",
    "alcop_model_predict", "alcop_tune", "alcop_time", "alcop_strerror", "alcop_version",
    "alcop_sched_auto", "alcop_cache_save", "alcop_cache_load",
    "alcop_corrector_features", "alcop_corrector_fit", "alcop_splitk_workspace_bytes", "alcop_gemm_splitk", "alcop_gemm_splitk_static", "alcop_conv2d_igemm_splitk", "alcop_splitk_auto", "alcop_splitk_space", "alcop_tune_splitk", "alcop_conv2d_igemm_krsc", "alcop_conv2d_igemm_fused", "alcop_conv2d_igemm_dilated", "alcop_sched_variants", "alcop_sched_ranked",
    "alcop_unaligned_workspace_bytes", "alcop_bmm_unaligned", "alcop_conv2d_unaligned_workspace_bytes",
    "alcop_conv2d_igemm_unaligned", "alcop_init",
    "alcop_linear", "alcop_linear_backward", "alcop_linear_backward_workspace_bytes", "alcop_rmsnorm",
    "alcop_rmsnorm_backward", "alcop_rmsnorm_backward_workspace_bytes", "alcop_quantize_rows",
    "alcop_layernorm", "alcop_layernorm_backward", "alcop_layernorm_backward_workspace_bytes", "alcop_grouped_linear",
    "alcop_grouped_linear_backward", "alcop_grouped_linear_backward_workspace_bytes", "alcop_linear_cross_entropy",
    "alcop_linear_cross_entropy_workspace_bytes", "alcop_linear_cross_entropy_backward",
    "alcop_linear_cross_entropy_backward_workspace_bytes",
]


class AlcopError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__("%s failed: %s (%d)" % (what, strerror(code), code))
        self.code = code


class Sched(ctypes.Structure):
    """Mirror of ``alcop_sched``."""
    _fields_ = [(n, ctypes.c_int) for n in
                ("bm", "bn", "bk", "wm", "wn", "stages", "reg_stages", "fuse_inner", "raster",
                 "l2_prefetch", "variant")]

    def key(self):
        return tuple(getattr(self, n) for n, _ in self._fields_)

    def __repr__(self):
        return "Sched(%dx%dx%d w%dx%d S%d R%d F%d r%d pf%d)" % self.key()[:10] + (
            "" if self.variant == 0 else "[v%d]" % self.variant)


def sched(bm, bn, bk, wm, wn, stages=1, reg_stages=1, fuse_inner=0, raster=1, l2_prefetch=0,
          variant=0) -> Sched:
    return Sched(bm, bn, bk, wm, wn, stages, reg_stages, fuse_inner, raster, l2_prefetch, variant)


class Epilogue(ctypes.Structure):
    """Mirror of ``alcop_epilogue``: C = act(alpha * A.B + bias[j])."""
    _fields_ = [("alpha", ctypes.c_float), ("bias", ctypes.c_void_p), ("act", ctypes.c_int)]


class LinearTail(ctypes.Structure):
    """Mirror of ``alcop_linear_tail``."""
    _fields_ = [("alpha", ctypes.c_float), ("bias", ctypes.c_void_p), ("act", ctypes.c_int), ("residual", ctypes.c_void_p),
                ("ldr", ctypes.c_long), ("pre", ctypes.c_void_p), ("ldp", ctypes.c_long), ("scale_a", ctypes.c_void_p),
                ("scale_w", ctypes.c_void_p)]


class Problem(ctypes.Structure):
    """Mirror of ``alcop_problem``."""
    _fields_ = [("op", ctypes.c_int), ("batch", ctypes.c_int), ("M", ctypes.c_int),
                ("N", ctypes.c_int), ("K", ctypes.c_int), ("transB", ctypes.c_int),
                ("in_", ctypes.c_int), ("out", ctypes.c_int), ("conv_C", ctypes.c_int),
                ("transA", ctypes.c_int)]


_lib = None
_marshal = None          # C++ marshalling of the hot entry points (csrc/py_binding.cpp) ...
_marshal_lib = None      # ... and the library its calls go to


def _declare(L: ctypes.CDLL) -> ctypes.CDLL:
    """Sets the argument and result types of every entry point of include/alcop.h on L."""
    vp, i, l = ctypes.c_void_p, ctypes.c_int, ctypes.c_long
    dp = ctypes.POINTER(ctypes.c_double)
    ip = ctypes.POINTER(ctypes.c_int)
    sp = ctypes.POINTER(Sched)
    pp = ctypes.POINTER(Problem)
    ep = ctypes.POINTER(Epilogue)
    L.alcop_gemm.restype = i
    L.alcop_gemm.argtypes = [vp, vp, vp, i, i, i, l, l, l, i, i, i, i, sp, vp]
    L.alcop_bmm.restype = i
    L.alcop_bmm.argtypes = [vp, vp, vp, i, i, i, i, l, l, l, l, l, l, i, i, i, i, sp, vp]
    L.alcop_gemm_fused.restype = i
    L.alcop_gemm_fused.argtypes = [vp, vp, vp, i, i, i, l, l, l, i, i, i, i, ep, sp, vp]
    L.alcop_bmm_fused.restype = i
    L.alcop_bmm_fused.argtypes = [vp, vp, vp, i, i, i, i, l, l, l, l, l, l, i, i, i, i, ep, sp, vp]
    L.alcop_conv2d_igemm.restype = i
    L.alcop_conv2d_igemm.argtypes = [vp, vp, vp] + [i] * 11 + [i, i, sp, vp]
    L.alcop_conv2d_igemm_krsc.restype = i
    L.alcop_conv2d_igemm_krsc.argtypes = [vp, vp, vp] + [i] * 11 + [i, i, sp, vp]
    L.alcop_conv2d_igemm_fused.restype = i
    L.alcop_conv2d_igemm_fused.argtypes = [vp, vp, vp] + [i] * 11 + [i, i, ep, i, sp, vp]
    L.alcop_sched_supported.restype = i
    L.alcop_sched_supported.argtypes = [pp, sp]
    L.alcop_sched_space.restype = i
    L.alcop_sched_space.argtypes = [pp, sp, i]
    L.alcop_model_predict.restype = i
    L.alcop_model_predict.argtypes = [pp, sp, i, dp, dp]
    L.alcop_tune.restype = i
    L.alcop_tune.argtypes = [pp, vp, vp, vp, l, l, l, l, l, l, ip, i, i, i, i, sp, dp, ip, ip,
                             sp, dp, dp, i, vp]
    L.alcop_sched_ranked.restype = i
    L.alcop_sched_ranked.argtypes = [pp, i, i, i, sp, i]
    L.alcop_sched_variants.restype = i
    L.alcop_sched_variants.argtypes = [pp, sp, i]
    L.alcop_time.restype = i
    L.alcop_time.argtypes = [pp, vp, vp, vp, l, l, l, l, l, l, ip, sp, i, i, dp, vp]
    L.alcop_sched_auto.restype = i
    L.alcop_sched_auto.argtypes = [pp, sp]
    L.alcop_cache_save.restype = i
    L.alcop_cache_save.argtypes = [ctypes.c_char_p]
    L.alcop_cache_load.restype = i
    L.alcop_cache_load.argtypes = [ctypes.c_char_p]
    L.alcop_corrector_features.restype = i
    L.alcop_corrector_features.argtypes = [pp, sp, dp]
    L.alcop_corrector_fit.restype = i
    L.alcop_corrector_fit.argtypes = [dp, dp, i, dp]
    sz = ctypes.c_size_t
    L.alcop_splitk_workspace_bytes.restype = sz
    L.alcop_splitk_workspace_bytes.argtypes = [i, i, i, i]
    L.alcop_gemm_splitk.restype = i
    L.alcop_gemm_splitk.argtypes = [vp, vp, vp, i, i, i, i, l, l, l, l, l, l, i, i, i, i, ep, sp, i,
                                    vp, sz, vp]
    L.alcop_gemm_splitk_static.restype = i
    L.alcop_gemm_splitk_static.argtypes = [vp, vp, vp, i, i, i, i, l, l, l, l, l, l, i, i, i, i, ep, sp, i, vp]
    L.alcop_conv2d_igemm_dilated.restype = i
    L.alcop_conv2d_igemm_dilated.argtypes = [vp, vp, vp] + [i] * 14 + [i, i, ep, sp, vp]
    L.alcop_unaligned_workspace_bytes.restype = sz
    L.alcop_unaligned_workspace_bytes.argtypes = [i, i, i, i, i]
    L.alcop_bmm_unaligned.restype = i
    L.alcop_bmm_unaligned.argtypes = [vp, vp, vp, i, i, i, i, l, l, l, l, l, l, i, i, i, i, ep, sp, vp, sz, vp]
    L.alcop_conv2d_unaligned_workspace_bytes.restype = sz
    L.alcop_conv2d_unaligned_workspace_bytes.argtypes = [i] * 14
    L.alcop_conv2d_igemm_unaligned.restype = i
    L.alcop_conv2d_igemm_unaligned.argtypes = [vp, vp, vp] + [i] * 13 + [i, i, ep, sp, vp, sz, vp]
    L.alcop_conv2d_igemm_splitk.restype = i
    L.alcop_conv2d_igemm_splitk.argtypes = [vp, vp, vp] + [i] * 11 + [i, i, sp, i, vp, sz, vp]
    L.alcop_tune_splitk.restype = i
    L.alcop_tune_splitk.argtypes = [pp, vp, vp, vp, l, l, l, l, l, l, ip, vp, sz, i, i, sp, ip, dp, ip, ip,
                                    sp, ip, dp, dp, i, vp]
    L.alcop_splitk_space.restype = i
    L.alcop_splitk_space.argtypes = [pp, sp, i]
    L.alcop_splitk_auto.restype = i
    L.alcop_splitk_auto.argtypes = [pp, i, sp, ip, dp]
    tp, f = ctypes.POINTER(LinearTail), ctypes.c_float
    L.alcop_linear.restype = i
    L.alcop_linear.argtypes = [vp, vp, vp, i, i, i, l, l, l, i, i, i, tp, vp]
    L.alcop_linear_backward_workspace_bytes.restype = sz
    L.alcop_linear_backward_workspace_bytes.argtypes = [i, i, i]
    L.alcop_linear_backward.restype = i
    L.alcop_linear_backward.argtypes = [vp] * 7 + [i] * 3 + [l] * 6 + [i, i, i, f, i, vp, sz, vp]
    L.alcop_rmsnorm.restype = i
    L.alcop_rmsnorm.argtypes = [vp] * 7 + [i, i] + [l] * 4 + [f, i, i, vp]
    L.alcop_rmsnorm_backward_workspace_bytes.restype = sz
    L.alcop_rmsnorm_backward_workspace_bytes.argtypes = [i, i]
    L.alcop_rmsnorm_backward.restype = i
    L.alcop_rmsnorm_backward.argtypes = [vp] * 7 + [i, i] + [l] * 4 + [i, vp, sz, vp]
    L.alcop_quantize_rows.restype = i
    L.alcop_quantize_rows.argtypes = [vp, vp, vp, i, i, l, l, i, vp]
    L.alcop_layernorm.restype = i
    L.alcop_layernorm.argtypes = [vp] * 9 + [i, i] + [l] * 4 + [f, i, i, vp]
    L.alcop_layernorm_backward_workspace_bytes.restype = sz
    L.alcop_layernorm_backward_workspace_bytes.argtypes = [i, i]
    L.alcop_layernorm_backward.restype = i
    L.alcop_layernorm_backward.argtypes = [vp] * 9 + [i, i] + [l] * 4 + [i, vp, sz, vp]
    L.alcop_grouped_linear.restype = i
    L.alcop_grouped_linear.argtypes = [vp] * 4 + [i] * 4 + [l] * 4 + [i, i, i, tp, vp]
    L.alcop_grouped_linear_backward_workspace_bytes.restype = sz
    L.alcop_grouped_linear_backward_workspace_bytes.argtypes = [i] * 4
    L.alcop_grouped_linear_backward.restype = i
    L.alcop_grouped_linear_backward.argtypes = [vp] * 8 + [i] * 4 + [l] * 8 + [i, i, i, f, i, vp, sz, vp]
    L.alcop_linear_cross_entropy_workspace_bytes.restype = sz
    L.alcop_linear_cross_entropy_workspace_bytes.argtypes = [i] * 3
    L.alcop_linear_cross_entropy.restype = i
    L.alcop_linear_cross_entropy.argtypes = [vp] * 5 + [i] * 3 + [l, l, f, i, vp, sz, vp]
    L.alcop_linear_cross_entropy_backward_workspace_bytes.restype = sz
    L.alcop_linear_cross_entropy_backward_workspace_bytes.argtypes = [i] * 3
    L.alcop_linear_cross_entropy_backward.restype = i
    L.alcop_linear_cross_entropy_backward.argtypes = [vp] * 7 + [i] * 3 + [l] * 4 + [f, i, i, vp, sz, vp]
    L.alcop_init.restype = i
    L.alcop_init.argtypes = []
    L.alcop_strerror.restype = ctypes.c_char_p
    L.alcop_strerror.argtypes = [i]
    L.alcop_version.restype = ctypes.c_char_p
    L.alcop_version.argtypes = []
    return L


def lib() -> ctypes.CDLL:
    """Loads libalcop.so (built by ``python -m paper_2210_16691_amd.build``); fails loudly if absent."""
    global _lib, _marshal, _marshal_lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libalcop.so is not built: run `python -m paper_2210_16691_amd.build`")
        L = _declare(ctypes.CDLL(LIB_PATH))
        import torch  # noqa: F401  (the module below links against it)

        from . import _binding as m
        m.init(Sched, *[ctypes.cast(f, ctypes.c_void_p).value for f in
                        (L.alcop_gemm_fused, L.alcop_bmm_fused, L.alcop_bmm_unaligned, L.alcop_conv2d_igemm_dilated,
                         L.alcop_conv2d_igemm_unaligned)])
        m.init_layers(*[ctypes.cast(f, ctypes.c_void_p).value for f in
                        (L.alcop_linear, L.alcop_linear_backward, L.alcop_rmsnorm, L.alcop_rmsnorm_backward,
                         L.alcop_quantize_rows)])
        m.init_more(*[ctypes.cast(f, ctypes.c_void_p).value for f in
                        (L.alcop_layernorm, L.alcop_layernorm_backward, L.alcop_grouped_linear,
                         L.alcop_grouped_linear_backward, L.alcop_linear_cross_entropy, L.alcop_linear_cross_entropy_backward)])
        _lib, _marshal, _marshal_lib = L, m, L
    return _lib


def alcop_init() -> None:
    """Does ahead of time what the first call of each entry point would do besides launching."""
    _check(lib().alcop_init(), "alcop_init")


def strerror(code: int) -> str:
    return lib().alcop_strerror(int(code)).decode()


def version() -> str:
    return lib().alcop_version().decode()


# ---- marshalling helpers ---------------------------------------------------------------------
def _dtype_code(t) -> int:
    import torch
    return {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32}[t.dtype]


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def _stream(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _sp(s):
    return ctypes.byref(s) if s is not None else None


def _check(rc, what):
    if rc != OK:
        raise AlcopError(rc, what)


def _same_place(*ts):
    dev = ts[0].device
    for t in ts:
        if t is not None and t.device != dev:
            raise ValueError("operands live on different devices: %s and %s" % (dev, t.device))


def _mm_shapes(A, B, C, transA, transB, bias=None):
    """Operand checks of the matrix entry points, before anything reaches the C call: the library
    sizes its buffer descriptors from (M, N, K) and the leading dimensions it is told, so a tensor
    that does not have that shape would be read or written past its end on the GPU.  Returns
    (batch, M, N, K)."""
    if A.dim() != B.dim() or A.dim() != C.dim() or A.dim() not in (2, 3):
        raise ValueError("A, B, C must all be 2-D (GEMM) or all 3-D (batched)")
    if A.dtype != B.dtype:
        raise ValueError("A and B differ in dtype: %s and %s" % (A.dtype, B.dtype))
    _dtype_code(C)
    _same_place(A, B, C, bias)
    for name, t in (("A", A), ("B", B), ("C", C)):
        if t.stride(-1) != 1:
            raise ValueError("%s: the last dimension must be contiguous" % name)
    b = A.shape[0] if A.dim() == 3 else 1
    if A.dim() == 3 and (B.shape[0] != b or C.shape[0] != b):
        raise ValueError("batch sizes differ: %d, %d, %d" % (b, B.shape[0], C.shape[0]))
    K, M = tuple(A.shape[-2:]) if transA else tuple(A.shape[-2:])[::-1]
    Kb, N = tuple(B.shape[-2:])[::-1] if transB else tuple(B.shape[-2:])
    if Kb != K:
        raise ValueError("reduction extents differ: A has K = %d, B has K = %d" % (K, Kb))
    if tuple(C.shape[-2:]) != (M, N):
        raise ValueError("C is %s, expected %s" % (tuple(C.shape[-2:]), (M, N)))
    if bias is not None and (bias.dim() != 1 or bias.shape[0] != N or not bias.is_contiguous()
                             or bias.element_size() != 4 or not bias.is_floating_point()):
        raise ValueError("bias must be a contiguous fp32 vector of N = %d values" % N)
    return b, M, N, K


def _conv_shapes(x, w, y, stride, pad, krsc=False, bias=None, dilation=(1, 1)):
    """Operand checks of the convolution entry points.  Returns (N, H, W, C, K, R, S)."""
    if x.dim() != 4 or w.dim() != 4 or y.dim() != 4:
        raise ValueError("x, w, y must be 4-D (NHWC, RSCK or KRSC, NPQK)")
    if x.dtype != w.dtype:
        raise ValueError("x and w differ in dtype: %s and %s" % (x.dtype, w.dtype))
    _dtype_code(y)
    _same_place(x, w, y, bias)
    for name, t in (("x", x), ("w", w), ("y", y)):
        if not t.is_contiguous():
            raise ValueError("%s must be contiguous" % name)
    N, H, W, Cc = x.shape
    if krsc:
        K, R, S, Cw = w.shape
    else:
        R, S, Cw, K = w.shape
    if Cw != Cc:
        raise ValueError("channel counts differ: x has %d, w has %d" % (Cc, Cw))
    if stride[0] <= 0 or stride[1] <= 0 or pad[0] < 0 or pad[1] < 0 or dilation[0] <= 0 or dilation[1] <= 0:
        raise ValueError("stride and dilation must be positive and padding non-negative")
    P = (H + 2 * pad[0] - dilation[0] * (R - 1) - 1) // stride[0] + 1
    Q = (W + 2 * pad[1] - dilation[1] * (S - 1) - 1) // stride[1] + 1
    if tuple(y.shape) != (N, P, Q, K):
        raise ValueError("y is %s, expected %s" % (tuple(y.shape), (N, P, Q, K)))
    if bias is not None and (bias.dim() != 1 or bias.shape[0] != K or not bias.is_contiguous()
                             or bias.element_size() != 4 or not bias.is_floating_point()):
        raise ValueError("bias must be a contiguous fp32 vector of K = %d values" % K)
    return N, H, W, Cc, K, R, S


# ---- the entry points (same names as the C ABI) ----------------------------------------------
def alcop_gemm(A, B, C, sched=None, transB=False, stream=None, transA=False):
    """C[M,N] = A . B  (A is [M,K], or [K,M] if transA; B is [K,N], or [N,K] if transB).  Tensors
    are 2-D CUDA tensors whose last dimension is contiguous; C's dtype selects the output type."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.mm(A, B, C, transA, transB, sched, stream) if A.dim() == 2 else None
        if rc is not None:
            if rc:
                raise AlcopError(rc, "alcop_gemm")
            return C
    if A.dim() != 2:
        raise ValueError("alcop_gemm takes 2-D tensors")
    _, M, N, K = _mm_shapes(A, B, C, transA, transB)
    rc = lib().alcop_gemm(_ptr(A), _ptr(B), _ptr(C), M, N, K, A.stride(0), B.stride(0), C.stride(0),
                          int(transA), int(transB), _dtype_code(A), _dtype_code(C), _sp(sched),
                          _stream(stream))
    _check(rc, "alcop_gemm")
    return C


def alcop_bmm(A, B, C, sched=None, transB=False, stream=None, transA=False):
    """Batched: A [b,M,K] (or [b,K,M] if transA), B [b,K,N] (or [b,N,K] if transB), C [b,M,N]."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.mm(A, B, C, transA, transB, sched, stream) if A.dim() == 3 else None
        if rc is not None:
            if rc:
                raise AlcopError(rc, "alcop_bmm")
            return C
    if A.dim() != 3:
        raise ValueError("alcop_bmm takes 3-D tensors")
    b, M, N, K = _mm_shapes(A, B, C, transA, transB)
    rc = lib().alcop_bmm(_ptr(A), _ptr(B), _ptr(C), b, M, N, K, A.stride(1), B.stride(1), C.stride(1),
                         A.stride(0), B.stride(0), C.stride(0), int(transA), int(transB),
                         _dtype_code(A), _dtype_code(C), _sp(sched), _stream(stream))
    _check(rc, "alcop_bmm")
    return C


def _epilogue(alpha, bias, act):
    return Epilogue(float(alpha), bias.data_ptr() if bias is not None else None, int(act))


def alcop_gemm_fused(A, B, C, alpha=1.0, bias=None, act=0, sched=None, transB=False, stream=None):
    """C = act(alpha * A.B + bias[j]); bias is an fp32 CUDA vector of N values or None; act 1 = ReLU."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.mm(A, B, C, False, transB, sched, stream, alpha, bias, act) if A.dim() == 2 else None
        if rc is not None:
            if rc:
                raise AlcopError(rc, "alcop_gemm_fused")
            return C
    if A.dim() != 2:
        raise ValueError("alcop_gemm_fused takes 2-D tensors")
    _, M, N, K = _mm_shapes(A, B, C, False, transB, bias)
    e = _epilogue(alpha, bias, act)
    rc = lib().alcop_gemm_fused(_ptr(A), _ptr(B), _ptr(C), M, N, K, A.stride(0), B.stride(0),
                                C.stride(0), 0, int(transB), _dtype_code(A), _dtype_code(C),
                                ctypes.byref(e), _sp(sched), _stream(stream))
    _check(rc, "alcop_gemm_fused")
    return C


def alcop_bmm_fused(A, B, C, alpha=1.0, bias=None, act=0, sched=None, transB=False, stream=None):
    if _marshal_lib is _lib is not None:
        rc = _marshal.mm(A, B, C, False, transB, sched, stream, alpha, bias, act) if A.dim() == 3 else None
        if rc is not None:
            if rc:
                raise AlcopError(rc, "alcop_bmm_fused")
            return C
    if A.dim() != 3:
        raise ValueError("alcop_bmm_fused takes 3-D tensors")
    b, M, N, K = _mm_shapes(A, B, C, False, transB, bias)
    e = _epilogue(alpha, bias, act)
    rc = lib().alcop_bmm_fused(_ptr(A), _ptr(B), _ptr(C), b, M, N, K, A.stride(1), B.stride(1),
                               C.stride(1), A.stride(0), B.stride(0), C.stride(0), 0, int(transB),
                               _dtype_code(A), _dtype_code(C), ctypes.byref(e), _sp(sched),
                               _stream(stream))
    _check(rc, "alcop_bmm_fused")
    return C


def alcop_conv2d_igemm(x, w, y, stride=(1, 1), pad=(0, 0), sched=None, stream=None):
    """x NHWC [N,H,W,C], w RSCK [R,S,C,K], y NPQK [N,P,Q,K]; all contiguous."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.conv(x, w, y, stride, pad, (1, 1), False, sched, stream, 1.0, None, 0)
        if rc is not None:
            if rc:
                raise AlcopError(rc, "alcop_conv2d_igemm")
            return y
    N, H, W, Cc, K, R, S = _conv_shapes(x, w, y, stride, pad)
    rc = lib().alcop_conv2d_igemm(_ptr(x), _ptr(w), _ptr(y), N, H, W, Cc, K, R, S,
                                  stride[0], stride[1], pad[0], pad[1],
                                  _dtype_code(x), _dtype_code(y), _sp(sched), _stream(stream))
    _check(rc, "alcop_conv2d_igemm")
    return y


# ---- linear layers, norms, 8-bit rows --------------------------------------------------------
def _kind(t) -> int:
    import torch
    if t.dtype == torch.float8_e4m3fn:
        return E4M3
    return _dtype_code(t)


def _rows(name, t, rows=None, cols=None, like=None):
    """Checks a matrix of rows and returns (rows, cols, pitch).  A single row has no pitch of its own."""
    if t.dim() != 2 or t.numel() == 0:
        raise ValueError("%s must be a 2-D tensor with at least one element" % name)
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError("%s: the last dimension must be contiguous" % name)
    if rows is not None and tuple(t.shape) != (rows, cols):
        raise ValueError("%s is %s, expected %s" % (name, tuple(t.shape), (rows, cols)))
    if like is not None and t.dtype != like.dtype:
        raise ValueError("%s is %s, expected %s" % (name, t.dtype, like.dtype))
    return t.shape[0], t.shape[1], t.shape[1] if t.shape[0] == 1 else t.stride(0)


def _vector(name, t, n):
    import torch
    if t is not None and (t.dtype != torch.float32 or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous()):
        raise ValueError("%s must be a contiguous fp32 vector of %d values" % (name, n))


def _workspace(t):
    if t is not None and not t.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return _ptr(t), 0 if t is None else t.numel() * t.element_size()


def _pitch(t):
    return 0 if t is None else (t.shape[1] if t.shape[0] == 1 else t.stride(0))


def _call_on(t, what, fn, *args, stream=None):
    """Calls fn(*args, stream) on t's device; without a stream on that device's current one."""
    if not t.is_cuda and lib() is _marshal_lib:
        raise ValueError("%s takes tensors on a GPU" % what)
    if t.is_cuda:
        import torch
        with torch.cuda.device(t.device):
            rc = fn(*args, _stream(stream))
    else:
        rc = fn(*args, _stream(stream))
    _check(rc, what)


def alcop_linear(A, W, C, transB=False, alpha=1.0, bias=None, act=0, residual=None, pre=None, scale_a=None, scale_w=None,
                 stream=None, fp32_sums=False):
    """C = act(Z) + residual with Z = alpha * scale_a[i] * scale_w[j] * A.W + bias[j]; `pre` receives Z.

    A is [M,K], W [K,N] or, with transB, [N,K] (a layer's weights); both fp16, bf16 or, with transB, e4m3
    (torch.float8_e4m3fn).  C, residual and pre are [M,N] of one type: fp16, bf16 or fp32; residual may be C.  bias,
    scale_w (N) and scale_a (M) are fp32 vectors.  act: 0 none, 1 ReLU, 2 GELU (erf), 3 GELU (tanh), 4 SiLU.

    Sums are fp32, but for e4m3 operands, a 16-bit C and a layer that is not small: the 8-bit matrix instruction cuts off, of
    every eight products (k = 8g .. 8g+7), what lies below 2^-13 of the largest.  Z is then off by up to 2^-10 of the sum of its terms'
    magnitudes (numbers below 2^-6 counting as 2^-6), of normally distributed numbers by 2^-16 of its standard deviation.  fp32_sums=True has fp32 sums there too."""
    if fp32_sums:
        act = int(act) | FP32_SUMS
    if _marshal_lib is _lib is not None:
        rc = _marshal.linear(A, W, C, transB, alpha, bias, act, residual, pre, scale_a, scale_w, stream)
        if rc is not None:
            _check(rc, "alcop_linear")
            return C
    M, K, lda = _rows("A", A)
    N, Kw, ldw = _rows("W", W, like=A)
    if not transB:
        N, Kw = Kw, N
    if Kw != K:
        raise ValueError("reduction extents differ: A has K = %d, W has K = %d" % (K, Kw))
    _, _, ldc = _rows("C", C, M, N)
    _dtype_code(C)
    for name, t in (("residual", residual), ("pre", pre)):
        if t is not None:
            _rows(name, t, M, N, like=C)
    _vector("bias", bias, N)
    _vector("scale_a", scale_a, M)
    _vector("scale_w", scale_w, N)
    _same_place(A, W, C, bias, residual, pre, scale_a, scale_w)
    p = lambda t: None if t is None else t.data_ptr()
    tail = LinearTail(float(alpha), p(bias), int(act), p(residual), _pitch(residual), p(pre), _pitch(pre), p(scale_a),
                      p(scale_w))
    _call_on(A, "alcop_linear", lib().alcop_linear, _ptr(A), _ptr(W), _ptr(C), M, N, K, lda, ldw, ldc, int(transB), _kind(A),
             _kind(C), ctypes.byref(tail), stream=stream)
    return C


def alcop_linear_backward_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(lib().alcop_linear_backward_workspace_bytes(M, N, K))


def alcop_linear_backward(dC, A, W, dA=None, dW=None, dbias=None, pre=None, act=0, alpha=1.0, transB=False, workspace=None,
                          stream=None):
    """Gradients of alcop_linear: with dZ = dC * act'(pre), dA = alpha * dZ.W^T, dW = alpha * A^T.dZ (stored as W is) and
    dbias = the column sums of dZ; what is None is left out.  dC, A, W, pre have one type, fp16 or bf16; dA and
    dW are both of it or both fp32; dbias fp32.  workspace: at least alcop_linear_backward_workspace_bytes(M, N, K) bytes, for
    an activation or dbias."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.linear_backward(dC, A, W, dA, dW, dbias, pre, act, alpha, transB, workspace, stream)
        if rc is not None:
            _check(rc, "alcop_linear_backward")
            return
    M, N, lddc = _rows("dC", dC)
    _, K, lda = _rows("A", A, like=dC)
    _rows("A", A, M, K)
    _, _, ldw = _rows("W", W, *((N, K) if transB else (K, N)), like=dC)
    if dA is not None:
        _rows("dA", dA, M, K, like=dW)
    if dW is not None:
        _rows("dW", dW, *W.shape)
    if pre is not None:
        _rows("pre", pre, M, N, like=dC)
    _vector("dbias", dbias, N)
    _same_place(dC, A, W, dA, dW, dbias, pre, workspace)
    ws, ws_bytes = _workspace(workspace)
    out = dA if dA is not None else dW
    _call_on(dC, "alcop_linear_backward", lib().alcop_linear_backward, _ptr(dC), _ptr(A), _ptr(W), _ptr(pre), _ptr(dA),
             _ptr(dW), _ptr(dbias), M, N, K, lddc, lda, ldw, _pitch(pre), _pitch(dA), _pitch(dW), int(transB), _kind(dC),
             _kind(dC if out is None else out), float(alpha), int(act), ws, ws_bytes, stream=stream)


def alcop_rmsnorm(x, gain, y, residual=None, total=None, scale=None, rstd=None, eps=1e-6, stream=None):
    """y = h * rstd * gain with h = x + residual and rstd = 1 / sqrt(mean(h^2) + eps) per row; total receives h.

    x, residual and total are [rows, cols] of one type (fp16, bf16, fp32); gain, rstd and scale are fp32 vectors of
    cols, rows and rows values; residual, total, gain and rstd may be None.  y is fp16, bf16, fp32 or e4m3, which needs
    scale: max(max |y| / 448, 2^-126) of the row, y then holding y / scale."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.rmsnorm(x, gain, y, residual, total, scale, rstd, eps, stream)
        if rc is not None:
            _check(rc, "alcop_rmsnorm")
            return y
    rows, cols, ldx = _rows("x", x)
    _, _, ldy = _rows("y", y, rows, cols)
    for name, t in (("residual", residual), ("total", total)):
        if t is not None:
            _rows(name, t, rows, cols, like=x)
    _vector("gain", gain, cols)
    _vector("scale", scale, rows)
    _vector("rstd", rstd, rows)
    _same_place(x, y, gain, residual, total, scale, rstd)
    _call_on(x, "alcop_rmsnorm", lib().alcop_rmsnorm, _ptr(x), _ptr(residual), _ptr(gain), _ptr(total), _ptr(y), _ptr(scale),
             _ptr(rstd), rows, cols, ldx, _pitch(residual), _pitch(total), ldy, float(eps), _kind(x), _kind(y), stream=stream)
    return y


def alcop_rmsnorm_backward_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().alcop_rmsnorm_backward_workspace_bytes(rows, cols))


def alcop_rmsnorm_backward(dy, total, gain, rstd, dx, dgain=None, dtotal=None, workspace=None, stream=None):
    """Gradients of alcop_rmsnorm: dx (of x and of the residual), to which the gradient dtotal that arrives at total
    is added, and dgain.  dy, total, dtotal and dx have one type; dx may be dy or dtotal.  workspace: at least
    alcop_rmsnorm_backward_workspace_bytes(rows, cols) bytes, for dgain."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.rmsnorm_backward(dy, total, gain, rstd, dx, dgain, dtotal, workspace, stream)
        if rc is not None:
            _check(rc, "alcop_rmsnorm_backward")
            return dx
    rows, cols, lddy = _rows("dy", dy)
    _, _, ldt = _rows("total", total, rows, cols, like=dy)
    _, _, lddx = _rows("dx", dx, rows, cols, like=dy)
    if dtotal is not None:
        _rows("dtotal", dtotal, rows, cols, like=dy)
    _vector("gain", gain, cols)
    _vector("dgain", dgain, cols)
    _vector("rstd", rstd, rows)
    _same_place(dy, total, dx, dtotal, gain, dgain, rstd, workspace)
    ws, ws_bytes = _workspace(workspace)
    _call_on(dy, "alcop_rmsnorm_backward", lib().alcop_rmsnorm_backward, _ptr(dy), _ptr(total), _ptr(gain), _ptr(rstd),
             _ptr(dtotal), _ptr(dx), _ptr(dgain), rows, cols, lddy, ldt, _pitch(dtotal), lddx, _kind(dy), ws, ws_bytes,
             stream=stream)
    return dx


def alcop_layernorm(x, gain, shift, y, residual=None, total=None, scale=None, mean=None, rstd=None, eps=1e-5, stream=None):
    """y = (h - mean) * rstd * gain + shift with h = x + residual, mean and 1 / rstd^2 = variance + eps per row; total receives h.

    x, residual and total are [rows, cols] of one type (fp16, bf16, fp32); gain and shift (cols), mean, rstd and scale
    (rows) are fp32 vectors; residual, total, gain, shift, mean and rstd may be None.  y is fp16, bf16, fp32 or e4m3, which
    needs scale: max(max |y| / 448, 2^-126) of the row, y then holding y / scale."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.layernorm(x, gain, shift, y, residual, total, scale, mean, rstd, eps, stream)
        if rc is not None:
            _check(rc, "alcop_layernorm")
            return y
    rows, cols, ldx = _rows("x", x)
    _, _, ldy = _rows("y", y, rows, cols)
    for name, t in (("residual", residual), ("total", total)):
        if t is not None:
            _rows(name, t, rows, cols, like=x)
    for name, t, n in (("gain", gain, cols), ("shift", shift, cols), ("scale", scale, rows), ("mean", mean, rows),
                       ("rstd", rstd, rows)):
        _vector(name, t, n)
    _same_place(x, y, gain, shift, residual, total, scale, mean, rstd)
    _call_on(x, "alcop_layernorm", lib().alcop_layernorm, _ptr(x), _ptr(residual), _ptr(gain), _ptr(shift), _ptr(total), _ptr(y),
             _ptr(scale), _ptr(mean), _ptr(rstd), rows, cols, ldx, _pitch(residual), _pitch(total), ldy, float(eps), _kind(x),
             _kind(y), stream=stream)
    return y


def alcop_layernorm_backward_workspace_bytes(rows: int, cols: int) -> int:
    return int(lib().alcop_layernorm_backward_workspace_bytes(rows, cols))


def alcop_layernorm_backward(dy, total, gain, mean, rstd, dx, dgain=None, dshift=None, dtotal=None, workspace=None, stream=None):
    """Gradients of alcop_layernorm: dx (of x and of the residual), to which the gradient dtotal that arrives at total
    is added, dgain and dshift.  dy, total, dtotal and dx have one type; dx may be dy or dtotal.  workspace: at least
    alcop_layernorm_backward_workspace_bytes(rows, cols) bytes, for dgain or dshift."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.layernorm_backward(dy, total, gain, mean, rstd, dx, dgain, dshift, dtotal, workspace, stream)
        if rc is not None:
            _check(rc, "alcop_layernorm_backward")
            return dx
    rows, cols, lddy = _rows("dy", dy)
    _, _, ldt = _rows("total", total, rows, cols, like=dy)
    _, _, lddx = _rows("dx", dx, rows, cols, like=dy)
    if dtotal is not None:
        _rows("dtotal", dtotal, rows, cols, like=dy)
    for name, t, n in (("gain", gain, cols), ("dgain", dgain, cols), ("dshift", dshift, cols), ("mean", mean, rows),
                       ("rstd", rstd, rows)):
        _vector(name, t, n)
    _same_place(dy, total, dx, dtotal, gain, mean, rstd, dgain, dshift, workspace)
    ws, ws_bytes = _workspace(workspace)
    _call_on(dy, "alcop_layernorm_backward", lib().alcop_layernorm_backward, _ptr(dy), _ptr(total), _ptr(gain), _ptr(mean),
             _ptr(rstd), _ptr(dtotal), _ptr(dx), _ptr(dgain), _ptr(dshift), rows, cols, lddy, ldt, _pitch(dtotal), lddx, _kind(dy),
             ws, ws_bytes, stream=stream)
    return dx


def _group_shapes(A, W, offsets, transB):
    """Checks rows, groups of weights and their offsets; returns (rows, groups, N, K, lda, ldw, strideW)."""
    import torch
    rows, K, lda = _rows("A", A)
    ldw, stride = _group_pitches("W", W)
    if W.dtype != A.dtype:
        raise ValueError("W is %s, expected %s" % (W.dtype, A.dtype))
    N, Kw = (W.shape[1], W.shape[2]) if transB else (W.shape[2], W.shape[1])
    if Kw != K:
        raise ValueError("reduction extents differ: A has K = %d, W has K = %d" % (K, Kw))
    if offsets.dtype != torch.int32 or offsets.dim() != 1 or offsets.shape[0] != W.shape[0] + 1 or not offsets.is_contiguous():
        raise ValueError("offsets must be a contiguous int32 vector of groups + 1 = %d numbers" % (W.shape[0] + 1))
    return rows, W.shape[0], N, K, lda, ldw, stride


def _group_pitches(name, t):
    if t.dim() != 3 or t.numel() == 0:
        raise ValueError("%s must be a 3-D tensor with at least one element" % name)
    if t.shape[2] > 1 and t.stride(2) != 1:
        raise ValueError("%s: the last dimension must be contiguous" % name)
    ld = t.shape[2] if t.shape[1] == 1 else t.stride(1)
    return ld, t.shape[1] * ld if t.shape[0] == 1 else t.stride(0)


def _per_group(name, t, groups, n):
    import torch
    if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != (groups, n) or not t.is_contiguous()):
        raise ValueError("%s must be a contiguous fp32 matrix of %d x %d values" % (name, groups, n))


def alcop_grouped_linear(A, W, offsets, C, transB=False, alpha=1.0, bias=None, act=0, pre=None, scale_a=None, scale_w=None,
                         stream=None, fp32_sums=False):
    """Rows offsets[g] .. offsets[g+1]-1 of C = act(Z) with Z = alpha * scale_a[i] * scale_w[g,j] * A.W[g] + bias[g,j]; `pre`
    receives Z.  Rows of no group are left as they are.

    A is [rows,K], sorted by group, W [groups,K,N] or, with transB, [groups,N,K]; both fp16, bf16 or, with transB, e4m3.
    offsets: groups + 1 rising int32 numbers on the GPU, from 0 or more to `rows` or less.  C and pre are [rows,N] of one type:
    fp16, bf16 or fp32.  bias and scale_w are fp32 [groups,N], scale_a an fp32 vector of rows values.  act and the sums of
    e4m3 operands (fp32_sums): as for alcop_linear."""
    if fp32_sums:
        act = int(act) | FP32_SUMS
    if _marshal_lib is _lib is not None:
        rc = _marshal.grouped_linear(A, W, offsets, C, transB, alpha, bias, act, pre, scale_a, scale_w, stream)
        if rc is not None:
            _check(rc, "alcop_grouped_linear")
            return C
    rows, groups, N, K, lda, ldw, stride = _group_shapes(A, W, offsets, transB)
    _, _, ldc = _rows("C", C, rows, N)
    _dtype_code(C)
    if pre is not None:
        _rows("pre", pre, rows, N, like=C)
    _per_group("bias", bias, groups, N)
    _per_group("scale_w", scale_w, groups, N)
    _vector("scale_a", scale_a, rows)
    _same_place(A, W, offsets, C, bias, pre, scale_a, scale_w)
    p = lambda t: None if t is None else t.data_ptr()
    tail = LinearTail(float(alpha), p(bias), int(act), None, 0, p(pre), _pitch(pre), p(scale_a), p(scale_w))
    _call_on(A, "alcop_grouped_linear", lib().alcop_grouped_linear, _ptr(A), _ptr(W), _ptr(offsets), _ptr(C), rows, groups, N, K,
             lda, ldw, stride, ldc, int(transB), _kind(A), _kind(C), ctypes.byref(tail), stream=stream)
    return C


def alcop_grouped_linear_backward_workspace_bytes(rows: int, groups: int, N: int, K: int) -> int:
    return int(lib().alcop_grouped_linear_backward_workspace_bytes(rows, groups, N, K))


def alcop_grouped_linear_backward(dC, A, W, offsets, dA=None, dW=None, dbias=None, pre=None, act=0, alpha=1.0, transB=False,
                                  workspace=None, stream=None):
    """Gradients of alcop_grouped_linear: with dZ = dC * act'(pre), dA = alpha * dZ.W[g]^T, dW[g] = alpha * A_g^T.dZ_g (stored as
    W[g] is) and dbias[g] the column sums of dZ over the group's rows (0 for a group without); what is None is left
    out.  dC, A, W, pre have one type, fp16 or bf16; dA and dW are both of it or both fp32; dbias fp32 [groups,N].  workspace: at
    least alcop_grouped_linear_backward_workspace_bytes(rows, groups, N, K) bytes, for an activation or dbias."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.grouped_linear_backward(dC, A, W, offsets, dA, dW, dbias, pre, act, alpha, transB, workspace, stream)
        if rc is not None:
            _check(rc, "alcop_grouped_linear_backward")
            return
    rows, groups, N, K, lda, ldw, stride = _group_shapes(A, W, offsets, transB)
    _, _, lddc = _rows("dC", dC, rows, N, like=A)
    if dA is not None:
        _rows("dA", dA, rows, K, like=dW)
    lddw = stride_dw = 0
    if dW is not None:
        if tuple(dW.shape) != tuple(W.shape):
            raise ValueError("dW is %s, expected %s" % (tuple(dW.shape), tuple(W.shape)))
        lddw, stride_dw = _group_pitches("dW", dW)
    if pre is not None:
        _rows("pre", pre, rows, N, like=A)
    _per_group("dbias", dbias, groups, N)
    _same_place(dC, A, W, offsets, dA, dW, dbias, pre, workspace)
    ws, ws_bytes = _workspace(workspace)
    out = dA if dA is not None else dW
    _call_on(dC, "alcop_grouped_linear_backward", lib().alcop_grouped_linear_backward, _ptr(dC), _ptr(A), _ptr(W), _ptr(pre),
             _ptr(offsets), _ptr(dA), _ptr(dW), _ptr(dbias), rows, groups, N, K, lddc, lda, ldw, stride, _pitch(pre), _pitch(dA),
             lddw, stride_dw, int(transB), _kind(dC), _kind(dC if out is None else out), float(alpha), int(act), ws, ws_bytes,
             stream=stream)


def _loss_shapes(X, W, labels):
    """Checks rows, a vocabulary's vectors and labels; returns (rows, vocab, K, ldx, ldw)."""
    import torch
    rows, K, ldx = _rows("X", X)
    vocab, Kw, ldw = _rows("W", W, like=X)
    if Kw != K:
        raise ValueError("reduction extents differ: X has K = %d, W has K = %d" % (K, Kw))
    if labels.dtype != torch.int64 or labels.dim() != 1 or labels.shape[0] != rows or not labels.is_contiguous():
        raise ValueError("labels must be a contiguous int64 vector of %d numbers" % rows)
    return rows, vocab, K, ldx, ldw


def alcop_linear_cross_entropy_workspace_bytes(rows: int, vocab: int, K: int) -> int:
    return int(lib().alcop_linear_cross_entropy_workspace_bytes(rows, vocab, K))


def alcop_linear_cross_entropy(X, W, labels, loss, lse=None, workspace=None, alpha=1.0, stream=None):
    """loss = lse - z[label] with z = alpha * X.W^T and lse = log(sum(exp(z))) per row, without keeping z.

    X is [rows,K], W [vocab,K] (a layer's weights), both fp16 or bf16; labels int64; loss and lse fp32 vectors of rows values,
    lse may be None.  A row whose label is no column of the vocabulary does not count: its loss is 0.  workspace: at least
    alcop_linear_cross_entropy_workspace_bytes(rows, vocab, K) bytes.  0 < alpha <= 2e38."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.cross_entropy(X, W, labels, loss, lse, workspace, alpha, stream)
        if rc is not None:
            _check(rc, "alcop_linear_cross_entropy")
            return loss
    rows, vocab, K, ldx, ldw = _loss_shapes(X, W, labels)
    _vector("loss", loss, rows)
    _vector("lse", lse, rows)
    _same_place(X, W, labels, loss, lse, workspace)
    ws, ws_bytes = _workspace(workspace)
    _call_on(X, "alcop_linear_cross_entropy", lib().alcop_linear_cross_entropy, _ptr(X), _ptr(W), _ptr(labels), _ptr(loss), _ptr(lse),
             rows, vocab, K, ldx, ldw, float(alpha), _kind(X), ws, ws_bytes, stream=stream)
    return loss


def alcop_linear_cross_entropy_backward_workspace_bytes(rows: int, vocab: int, K: int) -> int:
    return int(lib().alcop_linear_cross_entropy_backward_workspace_bytes(rows, vocab, K))


def alcop_linear_cross_entropy_backward(X, W, labels, lse, workspace, dX=None, dW=None, dloss=None, alpha=1.0, stream=None):
    """Gradients of alcop_linear_cross_entropy: with G = dloss * (exp(z - lse) - one(label)), 0 in rows that do not count,
    dX = alpha * G.W and dW = alpha * G^T.X; what is None is left out.  lse as the forward call left it; dloss: an fp32 vector of rows
    values, None = 1.  dX and dW both have X's type, or both are fp32.  workspace: at least
    alcop_linear_cross_entropy_backward_workspace_bytes(rows, vocab, K) bytes."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.cross_entropy_backward(X, W, labels, lse, workspace, dX, dW, dloss, alpha, stream)
        if rc is not None:
            _check(rc, "alcop_linear_cross_entropy_backward")
            return
    rows, vocab, K, ldx, ldw = _loss_shapes(X, W, labels)
    if dX is not None:
        _rows("dX", dX, rows, K, like=dW)
    if dW is not None:
        _rows("dW", dW, vocab, K)
    _vector("lse", lse, rows)
    _vector("dloss", dloss, rows)
    _same_place(X, W, labels, lse, dloss, dX, dW, workspace)
    ws, ws_bytes = _workspace(workspace)
    out = dX if dX is not None else dW
    _call_on(X, "alcop_linear_cross_entropy_backward", lib().alcop_linear_cross_entropy_backward, _ptr(X), _ptr(W), _ptr(labels),
             _ptr(lse), _ptr(dloss), _ptr(dX), _ptr(dW), rows, vocab, K, ldx, ldw, _pitch(dX), _pitch(dW), float(alpha), _kind(X),
             _kind(X if out is None else out), ws, ws_bytes, stream=stream)


def alcop_quantize_rows(x, y, scale, stream=None):
    """Rows to e4m3 with a scale each: scale = max(max |x| / 448, 2^-126), y = x / scale."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.quantize_rows(x, y, scale, stream)
        if rc is not None:
            _check(rc, "alcop_quantize_rows")
            return y
    rows, cols, ldx = _rows("x", x)
    _, _, ldy = _rows("y", y, rows, cols)
    if _kind(y) != E4M3:
        raise ValueError("y must be torch.float8_e4m3fn")
    _vector("scale", scale, rows)
    _same_place(x, y, scale)
    _call_on(x, "alcop_quantize_rows", lib().alcop_quantize_rows, _ptr(x), _ptr(y), _ptr(scale), rows, cols, ldx, ldy, _kind(x),
             stream=stream)
    return y


def alcop_splitk_workspace_bytes(batch: int, M: int, N: int, split: int) -> int:
    return int(lib().alcop_splitk_workspace_bytes(batch, M, N, split))


def alcop_gemm_splitk(A, B, C, split, workspace, sched=None, alpha=1.0, bias=None, act=0,
                      transB=False, stream=None, transA=False):
    """C = act(alpha * A.B + bias) with the reduction axis cut into `split` slices (0 = the model's
    choice).  A, B, C are 2-D (GEMM) or 3-D (batched) tensors; `workspace` is a tensor of at least
    alcop_splitk_workspace_bytes(batch, M, N, split) bytes that the call overwrites."""
    b, M, N, K = _mm_shapes(A, B, C, transA, transB, bias)
    if A.dim() == 2:
        sA, sB, sC = 0, 0, 0
        lda, ldb, ldc = A.stride(0), B.stride(0), C.stride(0)
    else:
        lda, ldb, ldc = A.stride(1), B.stride(1), C.stride(1)
        sA, sB, sC = A.stride(0), B.stride(0), C.stride(0)
    e = _epilogue(alpha, bias, act)
    rc = lib().alcop_gemm_splitk(_ptr(A), _ptr(B), _ptr(C), b, M, N, K, lda, ldb, ldc, sA, sB, sC,
                                 int(transA), int(transB), _dtype_code(A), _dtype_code(C),
                                 ctypes.byref(e), _sp(sched), int(split), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream))
    _check(rc, "alcop_gemm_splitk")
    return C


SPLITK_STATIC_BYTES = 32 << 20


def alcop_gemm_splitk_static(A, B, C, split, sched=None, alpha=1.0, bias=None, act=0,
                             transB=False, stream=None, transA=False):
    """alcop_gemm_splitk without a workspace argument: the partial tiles go to the library's own
    device array (at most SPLITK_STATIC_BYTES); the call allocates nothing."""
    b, M, N, K = _mm_shapes(A, B, C, transA, transB, bias)
    if A.dim() == 2:
        sA, sB, sC = 0, 0, 0
        lda, ldb, ldc = A.stride(0), B.stride(0), C.stride(0)
    else:
        lda, ldb, ldc = A.stride(1), B.stride(1), C.stride(1)
        sA, sB, sC = A.stride(0), B.stride(0), C.stride(0)
    e = _epilogue(alpha, bias, act)
    rc = lib().alcop_gemm_splitk_static(_ptr(A), _ptr(B), _ptr(C), b, M, N, K, lda, ldb, ldc, sA, sB,
                                        sC, int(transA), int(transB), _dtype_code(A), _dtype_code(C),
                                        ctypes.byref(e), _sp(sched), int(split), _stream(stream))
    _check(rc, "alcop_gemm_splitk_static")
    return C


def alcop_conv2d_igemm_splitk(x, w, y, split, workspace, stride=(1, 1), pad=(0, 0), sched=None,
                              stream=None):
    """alcop_conv2d_igemm with the reduction axis R*S*C cut into `split` slices."""
    N, H, W, Cc, K, R, S = _conv_shapes(x, w, y, stride, pad)
    _same_place(x, workspace)
    rc = lib().alcop_conv2d_igemm_splitk(_ptr(x), _ptr(w), _ptr(y), N, H, W, Cc, K, R, S,
                                         stride[0], stride[1], pad[0], pad[1],
                                         _dtype_code(x), _dtype_code(y), _sp(sched), int(split),
                                         _ptr(workspace), workspace.numel() * workspace.element_size(),
                                         _stream(stream))
    _check(rc, "alcop_conv2d_igemm_splitk")
    return y


def alcop_splitk_space(prob: "Problem"):
    n = lib().alcop_splitk_space(ctypes.byref(prob), None, 0)
    if n < 0:
        raise AlcopError(n, "alcop_splitk_space")
    arr = (Sched * max(n, 1))()
    lib().alcop_splitk_space(ctypes.byref(prob), arr, n)
    return [Sched(*arr[i].key()) for i in range(n)]


def alcop_splitk_auto(prob: "Problem", split: int = 0):
    """Returns (schedule, split, predicted_us): the model's pick among the split-K variants."""
    s, n, us = Sched(), ctypes.c_int(), ctypes.c_double()
    _check(lib().alcop_splitk_auto(ctypes.byref(prob), int(split), ctypes.byref(s), ctypes.byref(n),
                                   ctypes.byref(us)), "alcop_splitk_auto")
    return s, n.value, us.value


def alcop_conv2d_igemm_fused(x, w, y, stride=(1, 1), pad=(0, 0), alpha=1.0, bias=None, act=0,
                             krsc=False, sched=None, stream=None):
    """y = act(alpha * conv(x, w) + bias[k]); w is RSCK [R,S,C,K], or KRSC [K,R,S,C] if krsc."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.conv(x, w, y, stride, pad, (1, 1), krsc, sched, stream, alpha, bias, act)
        if rc is not None:
            if rc:
                raise AlcopError(rc, "alcop_conv2d_igemm_fused")
            return y
    N, H, W, Cc, K, R, S = _conv_shapes(x, w, y, stride, pad, krsc, bias)
    e = _epilogue(alpha, bias, act)
    rc = lib().alcop_conv2d_igemm_fused(_ptr(x), _ptr(w), _ptr(y), N, H, W, Cc, K, R, S,
                                        stride[0], stride[1], pad[0], pad[1], _dtype_code(x),
                                        _dtype_code(y), ctypes.byref(e), int(krsc), _sp(sched),
                                        _stream(stream))
    _check(rc, "alcop_conv2d_igemm_fused")
    return y


def alcop_conv2d_igemm_dilated(x, w, y, stride=(1, 1), pad=(0, 0), dilation=(1, 1), alpha=1.0, bias=None,
                               act=0, krsc=False, sched=None, stream=None):
    """y = act(alpha * conv(x, w) + bias[k]) with filter taps dilation[0] rows / dilation[1] columns
    apart; w is RSCK [R,S,C,K], or KRSC [K,R,S,C] if krsc."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.conv(x, w, y, stride, pad, dilation, krsc, sched, stream, alpha, bias, act)
        if rc is not None:
            if rc:
                raise AlcopError(rc, "alcop_conv2d_igemm_dilated")
            return y
    N, H, W, Cc, K, R, S = _conv_shapes(x, w, y, stride, pad, krsc, bias, dilation)
    e = _epilogue(alpha, bias, act)
    rc = lib().alcop_conv2d_igemm_dilated(_ptr(x), _ptr(w), _ptr(y), N, H, W, Cc, K, R, S,
                                          stride[0], stride[1], pad[0], pad[1], dilation[0], dilation[1],
                                          int(krsc), _dtype_code(x), _dtype_code(y), ctypes.byref(e),
                                          _sp(sched), _stream(stream))
    _check(rc, "alcop_conv2d_igemm_dilated")
    return y


def alcop_unaligned_workspace_bytes(batch, M, N, K, out_dtype) -> int:
    return lib().alcop_unaligned_workspace_bytes(batch, M, N, K, out_dtype)


def alcop_bmm_unaligned(A, B, C, workspace, alpha=1.0, bias=None, act=0, sched=None, transA=False,
                        transB=False, stream=None):
    """C = act(alpha * A.B + bias[j]) for operands of any extent and element-aligned placement
    (2-D: a GEMM; 3-D: batched); they are padded into `workspace` (a CUDA byte tensor of at least
    alcop_unaligned_workspace_bytes(...) bytes) and multiplied there, or, single products of moderate
    size without a schedule, multiplied where they lie."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.mm_any(A, B, C, workspace, alpha, bias, act, sched, transA, transB, stream)
        if rc is not None:
            if rc:
                raise AlcopError(rc, "alcop_bmm_unaligned")
            return C
    b, M, N, K = _mm_shapes(A, B, C, transA, transB, bias)
    _same_place(A, workspace)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    e = _epilogue(alpha, bias, act)
    if A.dim() == 3:
        ld = (A.stride(1), B.stride(1), C.stride(1), A.stride(0), B.stride(0), C.stride(0))
    else:
        ld = (A.stride(0), B.stride(0), C.stride(0), 0, 0, 0)
    rc = lib().alcop_bmm_unaligned(_ptr(A), _ptr(B), _ptr(C), b, M, N, K, *ld, int(transA), int(transB),
                                   _dtype_code(A), _dtype_code(C), ctypes.byref(e), _sp(sched),
                                   _ptr(workspace), workspace.numel() * workspace.element_size(),
                                   _stream(stream))
    _check(rc, "alcop_bmm_unaligned")
    return C


def alcop_conv2d_unaligned_workspace_bytes(N, H, W, C, K, R, S, stride, pad, dilation, out_dtype) -> int:
    return lib().alcop_conv2d_unaligned_workspace_bytes(N, H, W, C, K, R, S, stride[0], stride[1], pad[0],
                                                        pad[1], dilation[0], dilation[1], out_dtype)


def alcop_conv2d_igemm_unaligned(x, w, y, workspace, stride=(1, 1), pad=(0, 0), dilation=(1, 1), alpha=1.0,
                                 bias=None, act=0, sched=None, stream=None):
    """y = act(alpha * conv(x, w) + bias[k]) for any channel counts (x NHWC, w RSCK, y NPQK); the
    tensors are padded to 8 channels in `workspace` and convolved there."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.conv_any(x, w, y, workspace, stride, pad, dilation, alpha, bias, act, sched, stream)
        if rc is not None:
            if rc:
                raise AlcopError(rc, "alcop_conv2d_igemm_unaligned")
            return y
    N, H, W, Cc, K, R, S = _conv_shapes(x, w, y, stride, pad, False, bias, dilation)
    _same_place(x, workspace)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    e = _epilogue(alpha, bias, act)
    rc = lib().alcop_conv2d_igemm_unaligned(_ptr(x), _ptr(w), _ptr(y), N, H, W, Cc, K, R, S, stride[0],
                                            stride[1], pad[0], pad[1], dilation[0], dilation[1],
                                            _dtype_code(x), _dtype_code(y), ctypes.byref(e), _sp(sched),
                                            _ptr(workspace), workspace.numel() * workspace.element_size(),
                                            _stream(stream))
    _check(rc, "alcop_conv2d_igemm_unaligned")
    return y


def alcop_conv2d_igemm_krsc(x, w, y, stride=(1, 1), pad=(0, 0), sched=None, stream=None):
    """x NHWC [N,H,W,C], w KRSC [K,R,S,C], y NPQK [N,P,Q,K]; all contiguous."""
    if _marshal_lib is _lib is not None:
        rc = _marshal.conv(x, w, y, stride, pad, (1, 1), True, sched, stream, 1.0, None, 0)
        if rc is not None:
            if rc:
                raise AlcopError(rc, "alcop_conv2d_igemm_krsc")
            return y
    N, H, W, Cc, K, R, S = _conv_shapes(x, w, y, stride, pad, krsc=True)
    rc = lib().alcop_conv2d_igemm_krsc(_ptr(x), _ptr(w), _ptr(y), N, H, W, Cc, K, R, S,
                                       stride[0], stride[1], pad[0], pad[1],
                                       _dtype_code(x), _dtype_code(y), _sp(sched), _stream(stream))
    _check(rc, "alcop_conv2d_igemm_krsc")
    return y


def problem(op, M, N, K, in_dtype, out_dtype, batch=1, transB=False, conv_C=0, transA=False) -> Problem:
    return Problem(op, batch, M, N, K, int(transB), in_dtype, out_dtype, conv_C, int(transA))


def alcop_sched_supported(prob: Problem, s: Sched) -> int:
    return lib().alcop_sched_supported(ctypes.byref(prob), ctypes.byref(s))


def alcop_sched_space(prob: Problem):
    n = lib().alcop_sched_space(ctypes.byref(prob), None, 0)
    if n < 0:
        raise AlcopError(n, "alcop_sched_space")
    arr = (Sched * max(n, 1))()
    lib().alcop_sched_space(ctypes.byref(prob), arr, n)
    return [Sched(*arr[i].key()) for i in range(n)]


def alcop_sched_variants(prob: Problem):
    """Schedule variants whose feasibility depends on the call (see alcop_sched.variant)."""
    n = lib().alcop_sched_variants(ctypes.byref(prob), None, 0)
    if n < 0:
        raise AlcopError(n, "alcop_sched_variants")
    arr = (Sched * max(n, 1))()
    lib().alcop_sched_variants(ctypes.byref(prob), arr, n)
    return [Sched(*arr[i].key()) for i in range(n)]


def alcop_sched_ranked(prob: Problem, model: int = 0, variants: bool = False, top_k: int = 10):
    """Schedules in the order alcop_tune(top_k, model) would try them."""
    n = lib().alcop_sched_ranked(ctypes.byref(prob), model, int(variants), top_k, None, 0)
    if n < 0:
        raise AlcopError(n, "alcop_sched_ranked")
    arr = (Sched * max(n, 1))()
    lib().alcop_sched_ranked(ctypes.byref(prob), model, int(variants), top_k, arr, n)
    return [Sched(*arr[i].key()) for i in range(n)]


def alcop_sched_auto(prob: Problem) -> Sched:
    """The schedule a None schedule resolves to (tuning cache, else the library's pick)."""
    s = Sched()
    _check(lib().alcop_sched_auto(ctypes.byref(prob), ctypes.byref(s)), "alcop_sched_auto")
    return s


def alcop_cache_save(path: str) -> int:
    n = lib().alcop_cache_save(os.fsencode(path))
    if n < 0:
        raise AlcopError(n, "alcop_cache_save")
    return n


def alcop_cache_load(path: str) -> int:
    n = lib().alcop_cache_load(os.fsencode(path))
    if n < 0:
        raise AlcopError(n, "alcop_cache_load")
    return n


def alcop_model_predict(prob: Problem, s: Sched, model: int = 0):
    """Returns (predicted_us, terms[8])."""
    us = ctypes.c_double()
    terms = (ctypes.c_double * 8)()
    rc = lib().alcop_model_predict(ctypes.byref(prob), ctypes.byref(s), model, ctypes.byref(us), terms)
    _check(rc, "alcop_model_predict")
    return us.value, list(terms)


CORRECTOR_DIM = 10


def alcop_corrector_features(prob: Problem, s: Sched):
    """Features of a (problem, schedule) pair as the learner of alcop_tune(model=2) sees them."""
    x = (ctypes.c_double * CORRECTOR_DIM)()
    _check(lib().alcop_corrector_features(ctypes.byref(prob), ctypes.byref(s), x), "alcop_corrector_features")
    return list(x)


def alcop_corrector_fit(X, measured_us):
    """Weights of the learner after the given trials (X: rows of CORRECTOR_DIM features)."""
    n = len(measured_us)
    flat = (ctypes.c_double * (n * CORRECTOR_DIM))(*[float(v) for row in X for v in row])
    ys = (ctypes.c_double * max(n, 1))(*[float(v) for v in measured_us])
    w = (ctypes.c_double * CORRECTOR_DIM)()
    _check(lib().alcop_corrector_fit(flat, ys, n, w), "alcop_corrector_fit")
    return list(w)


@dataclass
class TuneResult:
    best: Sched
    best_us: float
    trials: int
    space: int
    log: list   # [(Sched, predicted_us, measured_us)] in rank order


def _operands(prob, A, B, C, conv):
    if prob.op == OP_CONV2D:
        cv = (ctypes.c_int * 11)(*conv)
        return cv, (0, 0, 0, 0, 0, 0)
    if prob.op == OP_BMM:
        return None, (A.stride(1), B.stride(1), C.stride(1), A.stride(0), B.stride(0), C.stride(0))
    return None, (A.stride(0), B.stride(0), C.stride(0), 0, 0, 0)


def alcop_tune(prob: Problem, A, B, C, top_k=10, model=0, iters=20, conv=None, stream=None,
               variants=False) -> TuneResult:
    """Model-ranked tuning on the caller's tensors (C is overwritten). top_k=0: exhaustive.
    variants=True also considers the schedule variants that depend on the call's geometry."""
    cv, ld = _operands(prob, A, B, C, conv)
    cap = max(1, lib().alcop_sched_space(ctypes.byref(prob), None, 0) +
              lib().alcop_sched_variants(ctypes.byref(prob), None, 0))
    best, best_us = Sched(), ctypes.c_double()
    trials, space = ctypes.c_int(), ctypes.c_int()
    ls, lp, lm = (Sched * cap)(), (ctypes.c_double * cap)(), (ctypes.c_double * cap)()
    rc = lib().alcop_tune(ctypes.byref(prob), _ptr(A), _ptr(B), _ptr(C), *ld, cv, top_k, model,
                          int(variants), iters,
                          ctypes.byref(best), ctypes.byref(best_us), ctypes.byref(trials),
                          ctypes.byref(space), ls, lp, lm, cap, _stream(stream))
    _check(rc, "alcop_tune")
    log = [(Sched(*ls[i].key()), lp[i], lm[i]) for i in range(trials.value)]
    return TuneResult(Sched(*best.key()), best_us.value, trials.value, space.value, log)


def alcop_tune_splitk(prob: Problem, A, B, C, workspace, top_k=10, iters=20, conv=None, stream=None):
    """Model-ranked tuning over (split-K variant, slices).  Returns (TuneResult, best_split); the
    log entries are (Sched, slices, predicted_us, measured_us)."""
    cv, ld = _operands(prob, A, B, C, conv)
    cap = 16 * max(1, lib().alcop_splitk_space(ctypes.byref(prob), None, 0))
    best, best_us, best_split = Sched(), ctypes.c_double(), ctypes.c_int()
    trials, space = ctypes.c_int(), ctypes.c_int()
    ls, lk = (Sched * cap)(), (ctypes.c_int * cap)()
    lp, lm = (ctypes.c_double * cap)(), (ctypes.c_double * cap)()
    rc = lib().alcop_tune_splitk(ctypes.byref(prob), _ptr(A), _ptr(B), _ptr(C), *ld, cv, _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), top_k, iters,
                                 ctypes.byref(best), ctypes.byref(best_split), ctypes.byref(best_us),
                                 ctypes.byref(trials), ctypes.byref(space), ls, lk, lp, lm, cap,
                                 _stream(stream))
    _check(rc, "alcop_tune_splitk")
    log = [(Sched(*ls[i].key()), lk[i], lp[i], lm[i]) for i in range(trials.value)]
    return TuneResult(Sched(*best.key()), best_us.value, trials.value, space.value, log), best_split.value


def alcop_time(prob: Problem, A, B, C, s: Sched, warmup=3, iters=20, conv=None, stream=None) -> float:
    """Mean microseconds per launch of one schedule, timed with HIP events on the stream."""
    cv, ld = _operands(prob, A, B, C, conv)
    us = ctypes.c_double()
    rc = lib().alcop_time(ctypes.byref(prob), _ptr(A), _ptr(B), _ptr(C), *ld, cv, ctypes.byref(s),
                          warmup, iters, ctypes.byref(us), _stream(stream))
    _check(rc, "alcop_time")
    return us.value
