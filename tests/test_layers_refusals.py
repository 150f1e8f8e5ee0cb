"""Calls of the linear layers, norms and 8-bit rows that are refused: by the C ABI with an error and without a launch
(addresses here are never dereferenced), by the binding with an exception that says why."""
import ctypes

import pytest
import torch

import paper_2210_16691_amd as al

V = ctypes.c_void_p
# 4 GiB apart, so that nothing overlaps by accident
P = [V(k << 32) for k in range(1, 12)]
ODD = V((20 << 32) + 1)
EIGHT = V((20 << 32) + 8)


def linear(A=P[0], W=P[1], C=P[2], M=64, N=64, K=64, lda=64, ldw=64, ldc=64, transB=1, i=al.F16, o=al.F16, alpha=1.0, bias=None,
           act=0, residual=None, ldr=64, pre=None, ldp=64, sa=None, sw=None):
    t = al.LinearTail(alpha, bias, act, residual, ldr, pre, ldp, sa, sw)
    return al.lib().alcop_linear(A, W, C, M, N, K, lda, ldw, ldc, transB, i, o, ctypes.byref(t), None)


@pytest.mark.parametrize("kw,rc", [
    (dict(A=None), al.ERR_NULL), (dict(W=None), al.ERR_NULL), (dict(C=None), al.ERR_NULL),
    (dict(i=al.F32), al.ERR_DTYPE), (dict(i=9), al.ERR_DTYPE), (dict(o=al.E4M3), al.ERR_DTYPE), (dict(o=-1), al.ERR_DTYPE),
    (dict(act=5), al.ERR_UNSUPPORTED), (dict(act=-1), al.ERR_UNSUPPORTED), (dict(i=al.E4M3, transB=0), al.ERR_UNSUPPORTED),
    (dict(M=0), al.ERR_SHAPE), (dict(N=0), al.ERR_SHAPE), (dict(K=0), al.ERR_SHAPE), (dict(M=-1), al.ERR_SHAPE),
    (dict(K=60), al.ERR_SHAPE), (dict(K=56, i=al.E4M3), al.ERR_SHAPE), (dict(N=60, transB=0), al.ERR_SHAPE),
    (dict(lda=56), al.ERR_SHAPE), (dict(ldw=56), al.ERR_SHAPE), (dict(ldc=63), al.ERR_SHAPE),
    (dict(residual=P[3], ldr=63), al.ERR_SHAPE), (dict(pre=P[3], ldp=63), al.ERR_SHAPE),
    (dict(A=EIGHT), al.ERR_ALIGN), (dict(W=EIGHT), al.ERR_ALIGN), (dict(lda=68), al.ERR_ALIGN), (dict(ldw=68), al.ERR_ALIGN),
    (dict(i=al.E4M3, lda=72), al.ERR_ALIGN), (dict(C=ODD), al.ERR_ALIGN), (dict(residual=ODD), al.ERR_ALIGN),
    (dict(pre=ODD), al.ERR_ALIGN), (dict(bias=EIGHT), al.ERR_ALIGN), (dict(sw=EIGHT), al.ERR_ALIGN), (dict(sa=ODD), al.ERR_ALIGN),
    (dict(M=0x7fffffff), al.ERR_SIZE), (dict(N=0x7fffffff, ldc=0x3fffffff), al.ERR_SHAPE),
    (dict(lda=1 << 30), al.ERR_SIZE), (dict(ldc=1 << 30), al.ERR_SIZE), (dict(ldr=1 << 30, residual=P[3]), al.ERR_SIZE),
    (dict(M=256, N=256, lda=1 << 26, ldc=256), al.ERR_SIZE), (dict(transB=0, K=4096, lda=4096, ldw=1 << 20), al.ERR_SIZE),
    # what is written overlaps what is read, or what else is written
    (dict(C=P[0]), al.ERR_UNSUPPORTED), (dict(C=P[1]), al.ERR_UNSUPPORTED), (dict(pre=P[0]), al.ERR_UNSUPPORTED),
    (dict(pre=P[2]), al.ERR_UNSUPPORTED), (dict(bias=P[2]), al.ERR_UNSUPPORTED), (dict(sa=P[2]), al.ERR_UNSUPPORTED),
    (dict(sw=P[3], pre=P[3]), al.ERR_UNSUPPORTED), (dict(residual=P[3], pre=P[3]), al.ERR_UNSUPPORTED),
    (dict(residual=V((3 << 32) + 16)), al.ERR_UNSUPPORTED), (dict(residual=P[2], ldr=72), al.ERR_UNSUPPORTED),
    (dict(C=P[2], ldc=128, pre=V((3 << 32) + 120), ldp=128), al.ERR_UNSUPPORTED),
])
def test_linear_layers_that_are_refused(kw, rc):
    assert linear(**kw) == rc


def backward(dC=P[0], A=P[1], W=P[2], pre=P[3], dA=P[4], dW=P[5], db=P[6], M=64, N=64, K=64, lddc=64, lda=64, ldw=64, ldp=64,
             ldda=64, lddw=64, transB=1, i=al.F16, o=al.F16, alpha=1.0, act=3, ws=P[7], bytes=None):
    if bytes is None:
        bytes = al.lib().alcop_linear_backward_workspace_bytes(64, 64, 64)
    return al.lib().alcop_linear_backward(dC, A, W, pre, dA, dW, db, M, N, K, lddc, lda, ldw, ldp, ldda, lddw, transB, i, o, alpha,
                                          act, ws, bytes, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(dC=None), al.ERR_NULL), (dict(pre=None), al.ERR_NULL), (dict(ws=None), al.ERR_NULL), (dict(A=None), al.ERR_NULL),
    (dict(W=None), al.ERR_NULL), (dict(dA=None, dW=None, db=None), al.ERR_NULL), (dict(ws=None, act=0), al.ERR_NULL),
    (dict(i=al.F32), al.ERR_DTYPE), (dict(i=al.E4M3), al.ERR_DTYPE), (dict(o=al.BF16), al.ERR_DTYPE),
    (dict(act=5), al.ERR_UNSUPPORTED), (dict(M=0), al.ERR_SHAPE), (dict(N=60), al.ERR_SHAPE), (dict(K=60), al.ERR_SHAPE),
    (dict(lddc=56), al.ERR_SHAPE), (dict(lda=56), al.ERR_SHAPE), (dict(ldw=56), al.ERR_SHAPE), (dict(ldp=56), al.ERR_SHAPE),
    (dict(ldda=56), al.ERR_SHAPE), (dict(lddw=56), al.ERR_SHAPE),
    (dict(dC=EIGHT), al.ERR_ALIGN), (dict(A=EIGHT), al.ERR_ALIGN), (dict(W=EIGHT), al.ERR_ALIGN), (dict(pre=EIGHT), al.ERR_ALIGN),
    (dict(dA=EIGHT), al.ERR_ALIGN), (dict(dW=EIGHT), al.ERR_ALIGN), (dict(ws=EIGHT), al.ERR_ALIGN), (dict(db=ODD), al.ERR_ALIGN),
    (dict(lddc=68), al.ERR_ALIGN), (dict(ldda=68), al.ERR_ALIGN), (dict(lddc=1 << 30), al.ERR_SIZE), (dict(bytes=64), al.ERR_SIZE),
    (dict(dA=P[0]), al.ERR_UNSUPPORTED), (dict(dW=P[1]), al.ERR_UNSUPPORTED), (dict(dA=P[5]), al.ERR_UNSUPPORTED),
    (dict(db=P[3]), al.ERR_UNSUPPORTED), (dict(ws=P[3]), al.ERR_UNSUPPORTED), (dict(ws=P[4]), al.ERR_UNSUPPORTED),
])
def test_gradients_that_are_refused(kw, rc):
    assert backward(**kw) == rc


@pytest.mark.parametrize("kw", [
    # 2^20 rows of 1024 columns are the last that fit: the last row starts 2 KiB below 2^31
    dict(M=(1 << 20) + 8, K=1024, lda=1024, ldda=1024, ldw=1024, lddw=1024, dA=None),          # dW: A spans more than 2 GiB
    dict(M=(1 << 20) + 8, N=1024, lddc=1024, ldp=1024, dA=None),                               # dW: dZ does
    dict(N=(1 << 20) + 8, K=1024, lddc=1 << 21, ldp=1 << 21, lda=1024, ldda=1024, ldw=1024, lddw=1024, dW=None),   # dA: W does
])
@pytest.mark.parametrize("db", [None, P[6]])
def test_gradients_whose_products_are_refused_launch_nothing(kw, db):
    # far apart, so that no two overlap; without a GPU a launch would be ALCOP_ERR_LAUNCH
    far = {n: (i + 1) << 40 for i, n in enumerate(("dC", "A", "W", "pre", "dA", "dW", "ws"))}
    kw = {**{n: p for n, p in far.items()}, **kw}
    assert backward(db=db, bytes=1 << 39, **kw) == al.ERR_SIZE


def norm(x=P[0], r=P[1], g=P[2], h=P[3], y=P[4], s=P[5], d=P[6], rows=8, cols=64, ldx=64, ldr=64, ldt=64, ldy=64, eps=1e-6, i=al.F16,
         o=al.F16):
    return al.lib().alcop_rmsnorm(x, r, g, h, y, s, d, rows, cols, ldx, ldr, ldt, ldy, eps, i, o, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(x=None), al.ERR_NULL), (dict(y=None), al.ERR_NULL), (dict(s=None, o=al.E4M3), al.ERR_NULL),
    (dict(i=al.E4M3), al.ERR_DTYPE), (dict(o=4), al.ERR_DTYPE), (dict(rows=0), al.ERR_SHAPE), (dict(cols=0), al.ERR_SHAPE),
    (dict(ldx=63), al.ERR_SHAPE), (dict(ldr=63), al.ERR_SHAPE), (dict(ldt=63), al.ERR_SHAPE), (dict(ldy=63), al.ERR_SHAPE),
    (dict(cols=32769, ldx=40000, ldr=40000, ldt=40000, ldy=40000), al.ERR_SIZE),
    (dict(rows=1 << 25), al.ERR_SIZE), (dict(rows=1 << 23, cols=4096, ldx=4096, ldr=4096, ldt=4096, ldy=4096), al.ERR_SIZE),
    (dict(x=ODD), al.ERR_ALIGN), (dict(r=ODD), al.ERR_ALIGN), (dict(h=ODD), al.ERR_ALIGN), (dict(y=ODD), al.ERR_ALIGN),
    (dict(g=ODD), al.ERR_ALIGN), (dict(d=ODD), al.ERR_ALIGN), (dict(s=ODD, o=al.E4M3), al.ERR_ALIGN),
    (dict(y=P[3]), al.ERR_UNSUPPORTED), (dict(y=P[2]), al.ERR_UNSUPPORTED), (dict(h=P[2]), al.ERR_UNSUPPORTED),
    (dict(y=P[0], ldy=72), al.ERR_UNSUPPORTED), (dict(y=P[0], o=al.E4M3), al.ERR_UNSUPPORTED), (dict(d=P[4]), al.ERR_UNSUPPORTED),
    (dict(h=V((1 << 32) + 2)), al.ERR_UNSUPPORTED), (dict(d=P[5], o=al.E4M3), al.ERR_UNSUPPORTED), (dict(d=P[0]), al.ERR_UNSUPPORTED),
])
def test_norms_that_are_refused(kw, rc):
    assert norm(**kw) == rc


def norm_backward(dy=P[0], h=P[1], g=P[2], d=P[3], dt=P[4], dx=P[5], dg=P[6], rows=8, cols=64, lddy=64, ldt=64, lddt=64, lddx=64, i=al.F16,
                  ws=P[7], bytes=1 << 20):
    return al.lib().alcop_rmsnorm_backward(dy, h, g, d, dt, dx, dg, rows, cols, lddy, ldt, lddt, lddx, i, ws, bytes, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(dy=None), al.ERR_NULL), (dict(h=None), al.ERR_NULL), (dict(d=None), al.ERR_NULL), (dict(dx=None), al.ERR_NULL),
    (dict(ws=None), al.ERR_NULL), (dict(i=al.E4M3), al.ERR_DTYPE), (dict(rows=0), al.ERR_SHAPE), (dict(lddy=63), al.ERR_SHAPE),
    (dict(ldt=63), al.ERR_SHAPE), (dict(lddt=63), al.ERR_SHAPE), (dict(lddx=63), al.ERR_SHAPE), (dict(bytes=8), al.ERR_SIZE),
    (dict(cols=32769, lddy=40000, ldt=40000, lddt=40000, lddx=40000), al.ERR_SIZE), (dict(dx=ODD), al.ERR_ALIGN),
    (dict(ws=EIGHT), al.ERR_ALIGN), (dict(dx=P[1]), al.ERR_UNSUPPORTED), (dict(dx=P[0], lddx=72), al.ERR_UNSUPPORTED),
    (dict(dg=P[2]), al.ERR_UNSUPPORTED), (dict(ws=P[5]), al.ERR_UNSUPPORTED), (dict(ws=P[6]), al.ERR_UNSUPPORTED),
])
def test_norm_gradients_that_are_refused(kw, rc):
    assert norm_backward(**kw) == rc


def test_columns_of_one_matrix_do_not_overlap():
    # past every check of arguments: what is returned is the launch's error (no device) or its success
    f = lambda off: V((3 << 32) + off)
    for kw in (dict(C=f(0), ldc=256, pre=f(128), ldp=256, residual=f(256), ldr=256), dict(residual=P[2])):
        if not torch.cuda.is_available():
            assert linear(**kw) == al.ERR_LAUNCH


def test_workspace_sizes_of_arguments_no_call_accepts():
    L = al.lib()
    assert L.alcop_linear_backward_workspace_bytes(0, 64, 64) == 0 and L.alcop_linear_backward_workspace_bytes(8, 60, 64) == 0
    assert L.alcop_rmsnorm_backward_workspace_bytes(8, 32769) == 0 and L.alcop_rmsnorm_backward_workspace_bytes(0, 8) == 0
    assert L.alcop_linear_backward_workspace_bytes(1 << 30, 65536, 8) > 1 << 47


h = torch.float16


@pytest.mark.parametrize("args,kw,says", [
    ((torch.zeros(4, 8, dtype=h), torch.zeros(8, 16, dtype=h), torch.zeros(4, 8, dtype=h)), {}, "C is"),
    ((torch.zeros(4, 8, dtype=h), torch.zeros(16, 16, dtype=h), torch.zeros(4, 16, dtype=h)), {}, "reduction extents"),
    ((torch.zeros(4, 8, dtype=h), torch.zeros(8, 16), torch.zeros(4, 16, dtype=h)), {}, "W is"),
    ((torch.zeros(2, 4, 8, dtype=h), torch.zeros(8, 16, dtype=h), torch.zeros(4, 16, dtype=h)), {}, "2-D"),
    ((torch.zeros(0, 8, dtype=h), torch.zeros(8, 16, dtype=h), torch.zeros(0, 16, dtype=h)), {}, "at least one"),
    ((torch.zeros(8, 4, dtype=h).t(), torch.zeros(8, 16, dtype=h), torch.zeros(4, 16, dtype=h)), {}, "contiguous"),
    ((torch.zeros(4, 8, dtype=h), torch.zeros(8, 16, dtype=h), torch.zeros(4, 16, dtype=h)), dict(bias=torch.zeros(16, dtype=h)), "bias"),
    ((torch.zeros(4, 8, dtype=h), torch.zeros(8, 16, dtype=h), torch.zeros(4, 16, dtype=h)), dict(bias=torch.zeros(8)), "bias"),
    ((torch.zeros(4, 8, dtype=h), torch.zeros(8, 16, dtype=h), torch.zeros(4, 16, dtype=h)), dict(scale_a=torch.zeros(5)), "scale_a"),
    ((torch.zeros(4, 8, dtype=h), torch.zeros(8, 16, dtype=h), torch.zeros(4, 16, dtype=h)), dict(residual=torch.zeros(4, 16)), "residual"),
    ((torch.zeros(4, 8, dtype=h), torch.zeros(8, 16, dtype=h), torch.zeros(4, 16, dtype=h)), dict(pre=torch.zeros(4, 8, dtype=h)), "pre"),
])
def test_what_the_binding_says(args, kw, says):
    with pytest.raises(ValueError, match=says):
        al.alcop_linear(*args, **kw)


def test_tensors_in_host_memory_are_refused():
    x, w, s8 = torch.zeros(4, 8, dtype=h), torch.zeros(8, 16, dtype=h), torch.zeros(4, 8, dtype=torch.float8_e4m3fn)
    for fn, args in ((al.alcop_linear, (x, w, torch.zeros(4, 16, dtype=h))), (al.alcop_rmsnorm, (x, None, x.clone())),
                     (al.alcop_quantize_rows, (x, s8, torch.zeros(4))),
                     (al.alcop_rmsnorm_backward, (x, x.clone(), None, torch.zeros(4), x.clone())),
                     (al.alcop_linear_backward, (torch.zeros(4, 16, dtype=h), x, w, x.clone()))):
        with pytest.raises(ValueError, match="on a GPU"):
            fn(*args)


def test_what_the_binding_says_of_rows():
    x = torch.zeros(4, 8, dtype=h)
    with pytest.raises(ValueError, match="gain"):
        al.alcop_rmsnorm(x, torch.ones(4), x.clone())
    with pytest.raises(ValueError, match="residual"):
        al.alcop_rmsnorm(x, None, x.clone(), residual=torch.zeros(4, 8))
    with pytest.raises(ValueError, match="e4m3|float8"):
        al.alcop_quantize_rows(x, x.clone(), torch.zeros(4))
    with pytest.raises(ValueError, match="scale"):
        al.alcop_quantize_rows(x, torch.zeros(4, 8, dtype=torch.float8_e4m3fn), torch.zeros(8))
    with pytest.raises(ValueError, match="total"):
        al.alcop_rmsnorm_backward(x, torch.zeros(4, 9, dtype=h), None, torch.zeros(4), x.clone())
    with pytest.raises(ValueError, match="dA"):
        al.alcop_linear_backward(x, x.clone(), torch.zeros(8, 8, dtype=h), dA=torch.zeros(4, 8), dW=torch.zeros(8, 8, dtype=h))
