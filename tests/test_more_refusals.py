"""Calls of the layer norm, the products grouped by expert and the cross entropy that are refused: by the C ABI with an error and
without a launch (addresses here are never dereferenced), by the binding with an exception that says why."""
import ctypes

import pytest
import torch

import paper_2210_16691_amd as al

V = ctypes.c_void_p
# 4 GiB apart, so that nothing overlaps by accident
P = [V(k << 32) for k in range(1, 16)]
ODD = V((20 << 32) + 1)
TWO = V((20 << 32) + 2)
FOUR = V((20 << 32) + 4)
EIGHT = V((20 << 32) + 8)
NULL, DTYPE, SHAPE, ALIGN, SIZE, UNSUPPORTED = (al.ERR_NULL, al.ERR_DTYPE, al.ERR_SHAPE, al.ERR_ALIGN, al.ERR_SIZE, al.ERR_UNSUPPORTED)


def norm(x=P[0], r=P[1], g=P[2], b=P[3], h=P[4], y=P[5], s=P[6], m=P[7], d=P[8], rows=8, cols=64, ldx=64, ldr=64, ldt=64, ldy=64, eps=1e-5,
         i=al.F16, o=al.F16):
    return al.lib().alcop_layernorm(x, r, g, b, h, y, s, m, d, rows, cols, ldx, ldr, ldt, ldy, eps, i, o, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(s=None, o=al.E4M3), NULL), (dict(i=al.E4M3), DTYPE), (dict(o=4), DTYPE),
    (dict(rows=0), SHAPE), (dict(cols=0), SHAPE), (dict(ldx=63), SHAPE), (dict(ldr=63), SHAPE), (dict(ldt=63), SHAPE), (dict(ldy=63), SHAPE),
    (dict(cols=32769, ldx=40000, ldr=40000, ldt=40000, ldy=40000), SIZE), (dict(rows=1 << 25), SIZE),
    (dict(rows=1 << 23, cols=4096, ldx=4096, ldr=4096, ldt=4096, ldy=4096), SIZE),
    (dict(x=ODD), ALIGN), (dict(r=ODD), ALIGN), (dict(h=ODD), ALIGN), (dict(y=ODD), ALIGN), (dict(g=TWO), ALIGN), (dict(b=TWO), ALIGN),
    (dict(m=TWO), ALIGN), (dict(d=TWO), ALIGN), (dict(s=TWO, o=al.E4M3), ALIGN),
    (dict(y=P[4]), UNSUPPORTED), (dict(y=P[2]), UNSUPPORTED), (dict(h=P[3]), UNSUPPORTED), (dict(y=P[0], ldy=72), UNSUPPORTED),
    (dict(y=P[0], o=al.E4M3), UNSUPPORTED), (dict(m=P[8]), UNSUPPORTED), (dict(m=P[0]), UNSUPPORTED), (dict(d=P[5]), UNSUPPORTED),
    (dict(m=P[2]), UNSUPPORTED), (dict(d=P[6], o=al.E4M3), UNSUPPORTED), (dict(h=V((1 << 32) + 2)), UNSUPPORTED),
])
def test_norms(kw, rc):
    assert norm(**kw) == rc


def norm_backward(dy=P[0], h=P[1], g=P[2], m=P[3], d=P[4], dt=P[5], dx=P[6], dg=P[7], ds=P[8], rows=8, cols=64, lddy=64, ldt=64, lddt=64,
                  lddx=64, i=al.F16, ws=P[9], bytes=1 << 20):
    return al.lib().alcop_layernorm_backward(dy, h, g, m, d, dt, dx, dg, ds, rows, cols, lddy, ldt, lddt, lddx, i, ws, bytes, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(dy=None), NULL), (dict(h=None), NULL), (dict(m=None), NULL), (dict(d=None), NULL), (dict(dx=None), NULL), (dict(ws=None), NULL),
    (dict(ws=None, dg=None), NULL), (dict(i=al.E4M3), DTYPE), (dict(rows=0), SHAPE), (dict(lddy=63), SHAPE), (dict(ldt=63), SHAPE),
    (dict(lddt=63), SHAPE), (dict(lddx=63), SHAPE), (dict(bytes=8), SIZE), (dict(cols=32769, lddy=40000, ldt=40000, lddt=40000, lddx=40000), SIZE),
    (dict(dx=ODD), ALIGN), (dict(ws=EIGHT), ALIGN), (dict(dg=TWO), ALIGN), (dict(ds=TWO), ALIGN), (dict(m=TWO), ALIGN),
    (dict(dx=P[1]), UNSUPPORTED), (dict(dx=P[0], lddx=72), UNSUPPORTED), (dict(dg=P[2]), UNSUPPORTED), (dict(dg=P[8]), UNSUPPORTED),
    (dict(ds=P[3]), UNSUPPORTED), (dict(ws=P[6]), UNSUPPORTED), (dict(ws=P[7]), UNSUPPORTED), (dict(ws=P[0]), UNSUPPORTED),
])
def test_gradients_of_norms(kw, rc):
    assert norm_backward(**kw) == rc


def grouped(A=P[0], W=P[1], off=P[2], C=P[3], rows=64, groups=4, N=64, K=64, lda=64, ldw=64, sw_=4096, ldc=64, transB=1, i=al.F16, o=al.F16,
            alpha=1.0, bias=None, act=0, residual=None, ldr=64, pre=None, ldp=64, sa=None, sw=None):
    t = al.LinearTail(alpha, bias, act, residual, ldr, pre, ldp, sa, sw)
    return al.lib().alcop_grouped_linear(A, W, off, C, rows, groups, N, K, lda, ldw, sw_, ldc, transB, i, o, ctypes.byref(t), None)


@pytest.mark.parametrize("kw,rc", [
    (dict(A=None), NULL), (dict(W=None), NULL), (dict(off=None), NULL), (dict(C=None), NULL),
    (dict(i=al.F32), DTYPE), (dict(i=9), DTYPE), (dict(o=al.E4M3), DTYPE), (dict(act=5), UNSUPPORTED), (dict(act=-1), UNSUPPORTED),
    (dict(residual=P[5]), UNSUPPORTED), (dict(i=al.E4M3, transB=0), UNSUPPORTED),
    (dict(rows=0), SHAPE), (dict(groups=0), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(K=60), SHAPE), (dict(K=56, i=al.E4M3), SHAPE),
    (dict(N=60, transB=0), SHAPE), (dict(lda=56), SHAPE), (dict(ldw=56), SHAPE), (dict(ldc=63), SHAPE), (dict(pre=P[5], ldp=63), SHAPE),
    (dict(sw_=-8), SHAPE), (dict(A=EIGHT), ALIGN), (dict(W=EIGHT), ALIGN), (dict(lda=68), ALIGN), (dict(ldw=68), ALIGN), (dict(sw_=4100), ALIGN),
    (dict(i=al.E4M3, sw_=4104), ALIGN), (dict(C=ODD), ALIGN), (dict(pre=ODD), ALIGN), (dict(off=TWO), ALIGN), (dict(bias=TWO), ALIGN),
    (dict(sw=TWO), ALIGN), (dict(sa=TWO), ALIGN), (dict(rows=0x7fffffff), SIZE), (dict(groups=1 << 24), SIZE), (dict(lda=1 << 30), SIZE),
    (dict(ldc=1 << 30), SIZE), (dict(A=V(1 << 44), rows=1024, groups=1, N=256, lda=1 << 26, ldc=256), SIZE),
    (dict(N=0x7ffff000, ldc=0x3fffffff), SHAPE),
    (dict(C=P[0]), UNSUPPORTED), (dict(C=P[1]), UNSUPPORTED), (dict(C=V((2 << 32) + 3 * 8192)), UNSUPPORTED), (dict(C=P[2]), UNSUPPORTED),
    (dict(pre=P[3]), UNSUPPORTED), (dict(bias=P[3]), UNSUPPORTED), (dict(sa=P[3]), UNSUPPORTED), (dict(sw=P[4], pre=P[4]), UNSUPPORTED),
])
def test_grouped_products(kw, rc):
    assert grouped(**kw) == rc


def grouped_backward(dC=P[0], A=P[1], W=P[2], pre=P[3], off=P[4], dA=P[5], dW=P[6], db=P[7], rows=64, groups=4, N=64, K=64, lddc=64, lda=64,
                     ldw=64, sw=4096, ldp=64, ldda=64, lddw=64, sdw=4096, transB=1, i=al.F16, o=al.F16, alpha=1.0, act=3, ws=P[8], bytes=1 << 24):
    return al.lib().alcop_grouped_linear_backward(dC, A, W, pre, off, dA, dW, db, rows, groups, N, K, lddc, lda, ldw, sw, ldp, ldda, lddw, sdw,
                                                  transB, i, o, alpha, act, ws, bytes, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(dC=None), NULL), (dict(off=None), NULL), (dict(pre=None), NULL), (dict(ws=None), NULL), (dict(A=None), NULL), (dict(W=None), NULL),
    (dict(dA=None, dW=None, db=None), NULL), (dict(ws=None, act=0), NULL), (dict(i=al.F32), DTYPE), (dict(i=al.E4M3), DTYPE),
    (dict(o=al.BF16), DTYPE), (dict(act=5), UNSUPPORTED), (dict(rows=0), SHAPE), (dict(groups=0), SHAPE), (dict(N=60), SHAPE), (dict(K=60), SHAPE),
    (dict(lddc=56), SHAPE), (dict(lda=56), SHAPE), (dict(ldw=56), SHAPE), (dict(ldp=56), SHAPE), (dict(ldda=56), SHAPE), (dict(lddw=56), SHAPE),
    (dict(sdw=4088), SHAPE), (dict(sw=-8), SHAPE), (dict(dC=EIGHT), ALIGN), (dict(A=EIGHT), ALIGN), (dict(W=EIGHT), ALIGN), (dict(pre=EIGHT), ALIGN),
    (dict(dA=EIGHT), ALIGN), (dict(dW=EIGHT), ALIGN), (dict(ws=EIGHT), ALIGN), (dict(db=TWO), ALIGN), (dict(off=TWO), ALIGN),
    (dict(lddc=68), ALIGN), (dict(ldda=68), ALIGN), (dict(sw=4100), ALIGN), (dict(sdw=4100), ALIGN), (dict(lddc=1 << 30), SIZE),
    (dict(bytes=64), SIZE), (dict(groups=65536), SIZE), (dict(groups=64001), SIZE),
    (dict(dA=P[0]), UNSUPPORTED), (dict(dW=P[1]), UNSUPPORTED), (dict(dA=P[6]), UNSUPPORTED), (dict(db=P[3]), UNSUPPORTED),
    (dict(ws=P[3]), UNSUPPORTED), (dict(ws=P[5]), UNSUPPORTED), (dict(dA=V((3 << 32) + 3 * 8192)), UNSUPPORTED), (dict(db=P[4]), UNSUPPORTED),
])
def test_gradients_of_grouped_products(kw, rc):
    assert grouped_backward(**kw) == rc


def test_gradients_that_are_too_far_apart_launch_nothing():
    # A or dZ span 2 GiB and more; without a GPU a launch would be ALCOP_ERR_LAUNCH
    far = {n: V((k + 1) << 40) for k, n in enumerate(("dC", "A", "W", "pre", "off", "dA", "dW", "db", "ws"))}
    big = dict(rows=(1 << 20) + 8, K=1024, lda=1024, ldda=1024, ldw=1024, lddw=1024, sw=65536, sdw=65536, bytes=1 << 38)
    assert grouped_backward(**{**far, **big}) == SIZE
    big = dict(rows=(1 << 20) + 8, N=1024, lddc=1024, ldp=1024, sw=65536, sdw=65536, bytes=1 << 38)
    assert grouped_backward(**{**far, **big}) == SIZE


def loss(X=P[0], W=P[1], y=P[2], out=P[3], lse=P[4], rows=64, vocab=100, K=64, ldx=64, ldw=64, alpha=1.0, i=al.F16, ws=P[5], bytes=1 << 20):
    return al.lib().alcop_linear_cross_entropy(X, W, y, out, lse, rows, vocab, K, ldx, ldw, alpha, i, ws, bytes, None)


LOSS = [
    (dict(X=None), NULL), (dict(W=None), NULL), (dict(y=None), NULL), (dict(ws=None), NULL), (dict(i=al.F32), DTYPE), (dict(i=al.E4M3), DTYPE),
    (dict(rows=0), SHAPE), (dict(vocab=0), SHAPE), (dict(K=0), SHAPE), (dict(K=60), SHAPE), (dict(ldx=56), SHAPE), (dict(ldw=56), SHAPE),
    (dict(X=EIGHT), ALIGN), (dict(W=EIGHT), ALIGN), (dict(ldx=68), ALIGN), (dict(ldw=68), ALIGN), (dict(y=FOUR), ALIGN), (dict(lse=TWO), ALIGN),
    (dict(ws=EIGHT), ALIGN), (dict(alpha=0.0), UNSUPPORTED), (dict(alpha=-1.0), UNSUPPORTED), (dict(alpha=float("nan")), UNSUPPORTED),
    (dict(alpha=float("inf")), UNSUPPORTED), (dict(ldx=1 << 30), SIZE), (dict(bytes=64), SIZE), (dict(vocab=0x7fffffff, bytes=1 << 60), SIZE),
    (dict(ws=P[0]), UNSUPPORTED), (dict(ws=P[2]), UNSUPPORTED),
]


@pytest.mark.parametrize("kw,rc", LOSS + [
    (dict(out=None), NULL), (dict(out=TWO), ALIGN), (dict(out=P[4]), UNSUPPORTED), (dict(out=P[0]), UNSUPPORTED), (dict(lse=P[1]), UNSUPPORTED),
    (dict(ws=P[3]), UNSUPPORTED),
])
def test_losses(kw, rc):
    assert loss(**kw) == rc


def loss_backward(X=P[0], W=P[1], y=P[2], lse=P[3], d=P[4], dX=P[6], dW=P[7], rows=64, vocab=100, K=64, ldx=64, ldw=64, lddx=64, lddw=64,
                  alpha=1.0, i=al.F16, o=al.F16, ws=P[5], bytes=1 << 24):
    return al.lib().alcop_linear_cross_entropy_backward(X, W, y, lse, d, dX, dW, rows, vocab, K, ldx, ldw, lddx, lddw, alpha, i, o, ws, bytes, None)


@pytest.mark.parametrize("kw,rc", LOSS + [
    (dict(lse=None), NULL), (dict(dX=None, dW=None), NULL), (dict(o=al.BF16), DTYPE), (dict(lddx=56), SHAPE), (dict(lddw=56), SHAPE),
    (dict(d=TWO), ALIGN), (dict(dX=EIGHT), ALIGN), (dict(dW=EIGHT), ALIGN), (dict(lddx=68), ALIGN), (dict(lddw=68), ALIGN),
    (dict(lddx=1 << 30), SIZE), (dict(dX=P[0]), UNSUPPORTED), (dict(dW=P[1]), UNSUPPORTED), (dict(dX=P[7]), UNSUPPORTED),
    (dict(ws=P[6]), UNSUPPORTED), (dict(dW=P[4]), UNSUPPORTED), (dict(dX=P[3]), UNSUPPORTED),
])
def test_gradients_of_losses(kw, rc):
    assert loss_backward(**kw) == rc


def test_gradients_of_losses_that_are_too_far_apart_launch_nothing():
    far = {n: V((k + 1) << 44) for k, n in enumerate(("X", "W", "y", "lse", "d", "dX", "dW", "ws"))}
    assert loss_backward(**{**far, **dict(rows=(1 << 20) + 8, K=1024, ldx=1024, ldw=1024, lddx=1024, lddw=1024, bytes=1 << 43)}) == SIZE


def test_workspace_sizes():
    L = al.lib()
    for f, ok in ((L.alcop_layernorm_backward_workspace_bytes, (8, 64)), (L.alcop_grouped_linear_backward_workspace_bytes, (8, 2, 64, 64)),
                  (L.alcop_linear_cross_entropy_workspace_bytes, (8, 100, 64)),
                  (L.alcop_linear_cross_entropy_backward_workspace_bytes, (8, 100, 64))):
        assert f(*ok) > 0
        for i in range(len(ok)):
            assert f(*[0 if k == i else v for k, v in enumerate(ok)]) == 0
    assert L.alcop_layernorm_backward_workspace_bytes(8, 32769) == 0
    assert L.alcop_grouped_linear_backward_workspace_bytes(8, 2, 60, 64) == 0 and L.alcop_linear_cross_entropy_workspace_bytes(8, 100, 60) == 0
    # G of a piece, sums of dX: not what a vocabulary's logits take
    assert L.alcop_linear_cross_entropy_backward_workspace_bytes(8192, 1 << 20, 4096) < 600 << 20


h = torch.float16
A, W, offs = torch.zeros(6, 8, dtype=h), torch.zeros(3, 16, 8, dtype=h), torch.zeros(4, dtype=torch.int32)
C, y64 = torch.zeros(6, 16, dtype=h), torch.zeros(6, dtype=torch.int64)
W2, f6 = torch.zeros(40, 8, dtype=h), torch.zeros(6)


@pytest.mark.parametrize("call,says", [
    (lambda: al.alcop_grouped_linear(A, W[0], offs, C, transB=True), "3-D"),
    (lambda: al.alcop_grouped_linear(A, W.float(), offs, C, transB=True), "W is"),
    (lambda: al.alcop_grouped_linear(A, W, offs, C), "reduction extents"),
    (lambda: al.alcop_grouped_linear(A, W, offs[:3], C, transB=True), "offsets"),
    (lambda: al.alcop_grouped_linear(A, W, offs.long(), C, transB=True), "offsets"),
    (lambda: al.alcop_grouped_linear(A, W, offs, C[:, :8], transB=True), "C is"),
    (lambda: al.alcop_grouped_linear(A, W, offs, C, transB=True, bias=torch.zeros(16)), "bias"),
    (lambda: al.alcop_grouped_linear(A, W, offs, C, transB=True, scale_w=torch.zeros(3, 8)), "scale_w"),
    (lambda: al.alcop_grouped_linear(A, W, offs, C, transB=True, scale_a=torch.zeros(3)), "scale_a"),
    (lambda: al.alcop_grouped_linear(A, W, offs, C, transB=True, pre=C.float()), "pre"),
    (lambda: al.alcop_grouped_linear(A, W.transpose(1, 2), offs, C), "contiguous"),
    (lambda: al.alcop_grouped_linear_backward(C, A, W, offs, dW=W[:2], transB=True), "dW"),
    (lambda: al.alcop_grouped_linear_backward(C, A, W, offs, dA=A.float(), dW=W.clone(), transB=True), "dA"),
    (lambda: al.alcop_grouped_linear_backward(C[:, :8], A, W, offs, dA=A.clone(), transB=True), "dC"),
    (lambda: al.alcop_grouped_linear_backward(C, A, W, offs, dbias=torch.zeros(16), transB=True), "dbias"),
    (lambda: al.alcop_linear_cross_entropy(A, W2[:, :4], y64, f6), "contiguous|extents"),
    (lambda: al.alcop_linear_cross_entropy(A, W2.float(), y64, f6), "W is"),
    (lambda: al.alcop_linear_cross_entropy(A, W2, y64.int(), f6), "labels"),
    (lambda: al.alcop_linear_cross_entropy(A, W2, y64[:5], f6), "labels"),
    (lambda: al.alcop_linear_cross_entropy(A, W2, y64, f6[:5]), "loss"),
    (lambda: al.alcop_linear_cross_entropy_backward(A, W2, y64, f6, None, dX=A.float(), dW=W2.clone()), "dX"),
    (lambda: al.alcop_linear_cross_entropy_backward(A, W2, y64, f6, None, dW=W2[:3]), "dW"),
    (lambda: al.alcop_linear_cross_entropy_backward(A, W2, y64, f6, None, dX=A.clone(), dloss=f6.double()), "dloss"),
    (lambda: al.alcop_layernorm(A, torch.ones(4), None, A.clone()), "gain"),
    (lambda: al.alcop_layernorm(A, None, torch.ones(4), A.clone()), "shift"),
    (lambda: al.alcop_layernorm(A, None, None, A.clone(), residual=A.float()), "residual"),
    (lambda: al.alcop_layernorm(A, None, None, A.clone(), mean=torch.zeros(5)), "mean"),
    (lambda: al.alcop_layernorm_backward(A, A[:, :4], None, f6, f6, A.clone()), "contiguous|total"),
    (lambda: al.alcop_layernorm_backward(A, A.clone(), None, f6, f6, A.clone(), dshift=f6), "dshift"),
])
def test_what_the_binding_says(call, says):
    with pytest.raises(ValueError, match=says):
        call()


def test_tensors_in_host_memory_are_refused():
    for call in (lambda: al.alcop_layernorm(A, None, None, A.clone()), lambda: al.alcop_layernorm_backward(A, A.clone(), None, f6, f6, A.clone()),
                 lambda: al.alcop_grouped_linear(A, W, offs, C, transB=True),
                 lambda: al.alcop_grouped_linear_backward(C, A, W, offs, dA=A.clone(), transB=True),
                 lambda: al.alcop_linear_cross_entropy(A, W2, y64, f6, None, torch.zeros(4096)),
                 lambda: al.alcop_linear_cross_entropy_backward(A, W2, y64, f6, torch.zeros(4096), dX=A.clone())):
        with pytest.raises(ValueError, match="on a GPU"):
            call()
