"""Linear layers, norms and 8-bit rows on the GPU against their plain forms in 64 bits (on the CPU): every kernel, types,
layouts, ragged sizes, pitches; results of a captured graph; streams; a transformer's feed-forward block, forward and
backward, out of these operators."""
import os

import pytest
import torch

import paper_2210_16691_amd as al
from gpu_util import DEV
from layers_util import DT, HALF, ULP, check, check_e4m3, linear64, norm64, norm_grad64, slope64

pytestmark = pytest.mark.gpu
F8_KERNELS = 6          # and on e4m3 operands with a 16-bit result (ALCOP_LINEAR_F8)
KERNELS = 11            # per operand type, layout and class of activation (ALCOP_LINEAR_CLASS)


def matrix(rows, cols, dtype, seed, pad=0, scale=1.0, offset=0):
    """Rows cols + pad apart, the first `offset` elements into their buffer; padding holds NaN."""
    g = torch.Generator().manual_seed(seed)
    flat = torch.full((offset + rows * (cols + pad),), float("nan"))
    flat[offset:].view(rows, cols + pad)[:, :cols].copy_(torch.randn(rows, cols, generator=g) * scale)
    return flat.to(DT[dtype]).to(DEV)[offset:].view(rows, cols + pad)[:, :cols]


def vector(n, seed, positive=False):
    v = torch.randn(n, generator=torch.Generator().manual_seed(seed))
    return (v.abs() + 0.5 if positive else v).to(DEV)


def padding(t):
    """The elements between a matrix's rows."""
    r, c, ld = t.shape[0], t.shape[1], t.stride(0)
    return t.as_strided((r - 1, ld - c), (ld, 1), t.storage_offset() + c) if r > 1 and ld > c else t[:0]


def run_linear(M, N, K, dtype, transB, out="bf16", act=0, bias=True, residual=True, pre=True, scales=False, pad=0, alpha=1.0,
               offset=0, in_place=False):
    A, W = matrix(M, K, dtype, 1, pad), matrix(*((N, K) if transB else (K, N)), dtype, 2, pad, scale=K ** -0.5)
    C = matrix(M, N, out, 3, pad, offset=offset)
    b = vector(N, 4) if bias else None
    r = (C if in_place else matrix(M, N, out, 5, pad, offset=offset)) if residual else None
    z = matrix(M, N, out, 6, pad, offset=offset) if pre else None
    sa, sw = (vector(M, 7, True), vector(N, 8, True)) if scales else (None, None)
    ref, zref, ez, ec = linear64(A, W, transB, alpha, b, act, r, sa, sw, dtype == "e4m3" and out != "f32")
    al.alcop_linear(A, W, C, transB=transB, alpha=alpha, bias=b, act=act, residual=r, pre=z, scale_a=sa, scale_w=sw)
    torch.cuda.synchronize()
    what = str((M, N, K, dtype, transB, out, act))
    check(C, ref, ec, "C " + what)
    if pre:
        check(z, zref, ez, "pre " + what)
    for t in (C, z):
        assert t is None or padding(t).isnan().all(), what


@pytest.mark.parametrize("kernel", range(KERNELS))
@pytest.mark.parametrize("dtype,transB", [("f16", False), ("f16", True), ("bf16", False), ("bf16", True), ("e4m3", True)])
def test_every_kernel_of_a_linear_layer(kernel, dtype, transB, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    i = kernel + 10 * transB + 20 * (dtype == "bf16")
    run_linear(300, 408, 208, dtype, transB, out=("f16", "bf16", "f32")[i % 3], act=i % 5, scales=dtype == "e4m3" or i % 2 == 0,
               pad=16)
    run_linear(513, 776, 1040, dtype, transB, out=("f16", "bf16", "f32")[(i + 1) % 3], act=(i + 2) % 5, residual=False)


@pytest.mark.parametrize("kernel", range(KERNELS, KERNELS + F8_KERNELS))
@pytest.mark.parametrize("act", [0, 2, 4])
def test_every_kernel_that_multiplies_8_bits_as_they_are(kernel, act, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    run_linear(300, 413, 720, "e4m3", True, out=("f16", "bf16")[kernel % 2], act=act, scales=True, pad=16)
    run_linear(513, 776, 2064, "e4m3", True, out="bf16", act=act, residual=False)
    with pytest.raises(al.AlcopError):            # fp32 results get fp32 sums
        run_linear(8, 16, 16, "e4m3", True, out="f32")


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("out", ["f16", "bf16", "f32"])
def test_activations_and_output_types(act, out):
    run_linear(70, 96, 64, "bf16" if out == "bf16" else "f16", True, out=out, act=act)


@pytest.mark.parametrize("kernel", range(KERNELS))
@pytest.mark.parametrize("N,pad,offset", [(43, 16, 0), (200, 1, 0), (264, 16, 1), (1, 16, 0)])
def test_results_that_are_not_made_of_chunks(kernel, N, pad, offset, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    A, W = matrix(150, 96, "e4m3" if kernel % 2 else "f16", 1, 16), matrix(N, 96, "e4m3" if kernel % 2 else "f16", 2, 16, scale=0.1)
    for out in ("bf16", "f32"):
        C, r, z = (matrix(150, N, out, s, pad, offset=offset) for s in (3, 4, 5))
        b = vector(N, 6)
        ref, zref, ez, ec = linear64(A, W, True, 1.0, b, 4, r)
        al.alcop_linear(A, W, C, transB=True, bias=b, act=4, residual=r, pre=z)
        torch.cuda.synchronize()
        check(C, ref, ec, "C")
        check(z, zref, ez, "pre")
        assert padding(C).isnan().all() and padding(z).isnan().all()


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 64, 200])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "e4m3"])
def test_few_rows(M, dtype):
    run_linear(M, 776, 1040, dtype, True, act=3, scales=dtype == "e4m3")
    run_linear(M, 1029, 4112, dtype, True, out="f32", pre=False, in_place=True)
    run_linear(M, 64, 16, dtype, True, bias=False, residual=False, pre=False, alpha=-0.5)
    if dtype != "e4m3":
        run_linear(M, 1032, 520, dtype, False, act=2)


@pytest.mark.parametrize("dtype,transB", [("bf16", True), ("f16", False), ("e4m3", True)])
def test_larger_layers(dtype, transB):
    run_linear(2048, 2056, 528, dtype, transB, act=2, scales=dtype == "e4m3")
    run_linear(1111, 4104, 1024, dtype, transB, act=4, pre=False, pad=16)


def test_one_call_gives_the_same_bits_again():
    for M, N, K in ((7, 776, 4096), (700, 776, 1040)):
        A, W = matrix(M, K, "bf16", 1), matrix(N, K, "bf16", 2)
        first = None
        for _ in range(3):
            C = torch.empty(M, N, dtype=torch.float32, device=DEV)
            al.alcop_linear(A, W, C, transB=True, act=4)
            first = C if first is None else first
            assert torch.equal(first, C)


# ---- gradients ---------------------------------------------------------------------------------------------
def run_backward(M, N, K, dtype, transB, act, bias=True, out=None, pad=0, alpha=1.0):
    out = out or dtype
    dC, pre = matrix(M, N, dtype, 1, pad), matrix(M, N, dtype, 2, pad, scale=1.5) if act else None
    A, W = matrix(M, K, dtype, 3, pad), matrix(*((N, K) if transB else (K, N)), dtype, 4, pad, scale=0.2)
    dA, dW, db = matrix(M, K, out, 5, pad), matrix(*W.shape, out, 6, pad), vector(N, 7) if bias else None
    ws = torch.full((al.alcop_linear_backward_workspace_bytes(M, N, K),), 255, dtype=torch.uint8, device=DEV)
    al.alcop_linear_backward(dC, A, W, dA=dA, dW=dW, dbias=db, pre=pre, act=act, alpha=alpha, transB=transB, workspace=ws)
    torch.cuda.synchronize()
    d = dC.cpu().double()
    dz, edz = d, 0 * d
    if act:
        z = pre.cpu().double()
        dz = d * slope64(z, act)
        edz = d.abs() * 16 * ULP * (1 + z.abs())
    e = edz + (HALF[DT[dtype]] * (dz.abs() + edz) + 2.0 ** -25) * (act > 0)
    a, w = A.cpu().double(), W.cpu().double()
    w = w.t() if transB else w
    check(dA, alpha * dz @ w.t(), abs(alpha) * ((e + (N + 4) * ULP * dz.abs()) @ w.t().abs()), "dA")
    ref, err = alpha * a.t() @ dz, abs(alpha) * (a.t().abs() @ (e + (M + 4) * ULP * dz.abs()))
    check(dW, ref.t() if transB else ref, err.t() if transB else err, "dW")
    if bias:
        check(db[None], dz.sum(0)[None], (edz + (M + 4) * ULP * dz.abs()).sum(0)[None], "dbias")


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("dtype,transB", [("f16", False), ("f16", True), ("bf16", False), ("bf16", True)])
def test_gradients_of_a_linear_layer(act, dtype, transB):
    run_backward(333, 776, 520, dtype, transB, act, pad=8, alpha=0.5)


@pytest.mark.parametrize("M", [1, 3, 8, 100, 129, 1021])
def test_gradients_of_any_number_of_rows(M):
    run_backward(M, 264, 136, "f16", True, 3)
    run_backward(M, 1032, 648, "bf16", False, 0, out="f32")


@pytest.mark.parametrize("M,N,K,transB,act", [(5856, 64, 1400, True, 2), (5857, 64, 1400, True, 2), (8192, 256, 264, False, 0),
                                              (16384, 256, 256, True, 4), (7224, 112, 2168, False, 3)])
def test_gradients_of_small_weights_and_many_rows(M, N, K, transB, act):
    # dW's sum is split over blocks if the rows are a multiple of 8; the bias's gradient has few lanes to a row
    run_backward(M, N, K, "bf16", transB, act)


def test_a_split_sum_needs_the_workspace():
    M, N, K = 8192, 256, 264
    dC, A, W = matrix(M, N, "f16", 1), matrix(M, K, "f16", 2), matrix(N, K, "f16", 3)
    dW = [torch.empty(N, K, device=DEV) for _ in range(4)]
    size = al.alcop_linear_backward_workspace_bytes(M, N, K)
    ws = torch.full((size,), 255, dtype=torch.uint8, device=DEV)
    for t, w in zip(dW, (None, ws[: size // 2], ws, ws)):
        al.alcop_linear_backward(dC, A, W, dW=t, transB=True, workspace=w)
    assert torch.equal(dW[0], dW[1]) and torch.equal(dW[2], dW[3])
    ref = dC.cpu().double().t() @ A.cpu().double()
    mag = dC.cpu().double().abs().t() @ A.cpu().double().abs()
    for t in dW:
        check(t, ref, (M + 64) * ULP * mag, "dW")


def test_gradients_agree_with_differences():
    # the loss sum(C * G) along a direction of A, of W and of the bias: central differences of the forward pass in
    # fp32 results; the step's error is its square times the third derivative, below 1 % here, rounding of 16-bit
    # operands is left out by steps that the types hold exactly
    M, N, K, act = 24, 32, 16, 3
    g = torch.Generator().manual_seed(0)
    A, W = (torch.randint(-2, 3, (M, K), generator=g) / 4).to(DEV), (torch.randint(-2, 3, (N, K), generator=g) / 4).to(DEV)
    b, G = torch.zeros(N, device=DEV), torch.randint(-2, 3, (M, N), generator=g).to(DEV).float()
    h = 2.0 ** -5
    DA, DW, Db = (h * torch.randint(-1, 2, t.shape, generator=g).to(DEV).float() for t in (A, W, b))

    def loss(a, w, bias, keep=None):
        C = torch.empty(M, N, device=DEV)
        al.alcop_linear(a.half(), w.half(), C, transB=True, bias=bias, act=act, pre=keep)
        return float((C.double() * G.double()).sum())

    z = torch.empty(M, N, device=DEV)
    loss(A, W, b, z)
    dA, dW, db = torch.empty(M, K, device=DEV), torch.empty(N, K, device=DEV), torch.empty(N, device=DEV)
    ws = torch.empty(al.alcop_linear_backward_workspace_bytes(M, N, K), dtype=torch.uint8, device=DEV)
    al.alcop_linear_backward(G.half(), A.half(), W.half(), dA=dA, dW=dW, dbias=db, pre=z.half(), act=act, transB=True, workspace=ws)
    for args, grad, step in (((DA, 0 * DW, 0 * Db), dA, DA), ((0 * DA, DW, 0 * Db), dW, DW), ((0 * DA, 0 * DW, Db), db, Db)):
        up, down = (loss(A + s * args[0], W + s * args[1], b + s * args[2]) for s in (1, -1))
        slope, want = (up - down) / 2, float((grad.double() * step.double()).sum())
        # third derivative of the activation below 2, times the cubes of what a step moves Z by
        moves = (step.abs().double() @ W.abs().double().t() if grad is dA else A.abs().double() @ step.abs().double().t()
                 if grad is dW else step.abs().double()[None].expand(M, N))
        bound = float((G.abs().double() * moves ** 3).sum()) / 3 + 2.0 ** -8 * float((G.abs().double() * moves * 1.13).sum())
        assert abs(slope - want) <= bound and bound < 0.2 * float((G.abs().double() * moves).sum())


# ---- rows -------------------------------------------------------------------------------------------------
COLS = [1, 7, 8, 64, 511, 512, 520, 768, 1023, 1032, 2048, 2056, 4096, 4101, 5000, 8192, 9000, 16384, 17000, 32768, 32767]


@pytest.mark.parametrize("cols", COLS)
def test_norm_of_every_row_length(cols):
    k = COLS.index(cols)
    for rows, dtype, out, pad, residual, gain in ((5, ("f16", "bf16", "f32")[k % 3], "e4m3" if k % 2 else ("f16", "bf16", "f32")[k % 3],
                                                   (0, 8, 3)[k % 3], True, True),
                                                  (1, ("bf16", "f32", "f16")[k % 3], ("e4m3", "f32")[k % 2], 0, False, k % 4 != 0)):
        x, r = matrix(rows, cols, dtype, 1, pad, 2.0), matrix(rows, cols, dtype, 2, pad) if residual else None
        h, g = matrix(rows, cols, dtype, 3, pad) if residual else None, vector(cols, 4) if gain else None
        y, s, d = matrix(rows, cols, out, 5, pad), vector(rows, 6) if out == "e4m3" else None, vector(rows, 7)
        yref, href, dref = norm64(x, r, g)
        al.alcop_rmsnorm(x, g, y, residual=r, total=h, scale=s, rstd=d)
        torch.cuda.synchronize()
        err = (cols / 2 + 8) * ULP
        check(d[:, None], dref[:, None], err * dref[:, None], "rstd")
        if h is not None:
            check(h, href, ULP * href.abs(), "total")
            assert padding(h).isnan().all()
        if out == "e4m3":
            check_e4m3(y, s, yref, err, "y")
        else:
            eh = ULP * href.abs() * dref[:, None] * (1 if g is None else g.cpu().double().abs())
            check(y, yref, err * yref.abs() + eh, "y")
        assert padding(y).float().isnan().all()
        x = matrix(rows, cols, dtype, 8, pad, 3.0)
        y, s = matrix(rows, cols, "e4m3", 9, pad), vector(rows, 10)
        al.alcop_quantize_rows(x, y, s)
        torch.cuda.synchronize()
        check_e4m3(y, s, x.cpu().double(), 0.0, "quantize")
        assert padding(y).float().isnan().all()


@pytest.mark.parametrize("cols", [7, 200, 1027, 5000])
def test_a_gain_and_sums_that_start_anywhere(cols):
    x, dy = matrix(9, cols, "bf16", 1), matrix(9, cols, "bf16", 2)
    for start in (1, 3):
        g, dg = vector(cols + 4, 3)[start:start + cols], vector(cols + 4, 4)
        y, d = matrix(9, cols, "f32", 5), vector(9, 6)
        al.alcop_rmsnorm(x, g, y, rstd=d)
        yref, href, dref = norm64(x, None, g)
        check(y, yref, (cols / 2 + 8) * ULP * yref.abs(), "y")
        ws = torch.empty(al.alcop_rmsnorm_backward_workspace_bytes(9, cols), dtype=torch.uint8, device=DEV)
        before, dx = dg.clone(), matrix(9, cols, "bf16", 7)
        al.alcop_rmsnorm_backward(dy, x, g, d, dx, dgain=dg[start:start + cols], workspace=ws)
        ref, gref, edx, edg = norm_grad64(dy, x, g, d)
        check(dx, ref, edx, "dx")
        check(dg[None, start:start + cols], gref[None], edg[None], "dgain")
        assert torch.equal(dg[:start], before[:start]) and torch.equal(dg[start + cols:], before[start + cols:])


def test_layers_on_two_streams_at_once():
    jobs = []
    for k, (M, N, K) in enumerate(((300, 520, 1040), (16, 2048, 2048))):
        jobs.append((matrix(M, K, "bf16", 2 * k), matrix(N, K, "bf16", 2 * k + 1), torch.empty(M, N, device=DEV),
                     torch.empty(M, N, device=DEV), torch.cuda.Stream()))
    for A, W, C, D, s in jobs:
        al.alcop_linear(A, W, D, transB=True, act=2)
    torch.cuda.synchronize()
    for _ in range(20):
        for A, W, C, D, s in jobs:
            al.alcop_linear(A, W, C, transB=True, act=2, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(C, D) for _, _, C, D, _ in jobs)


def test_e4m3_of_every_kind_of_value():
    # all numbers of 8 bits, the halfway values between them, and the row's own largest at 448: as torch rounds them
    codes = torch.arange(0x7f, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).float()
    vals = torch.cat([codes, (codes[1:] + codes[:-1]) / 2, torch.tensor([2.0 ** -11, 447.9])])
    x = torch.cat([vals, -vals])[None]
    x = torch.cat([x, x.new_zeros(1, (-x.shape[1]) % 8)], dim=1).to(DEV)
    y, s = torch.empty_like(x, dtype=torch.float8_e4m3fn), torch.empty(1, device=DEV)
    al.alcop_quantize_rows(x, y, s)
    assert float(s) == 1.0
    assert torch.equal(y.view(torch.uint8).cpu(), x.cpu().to(torch.float8_e4m3fn).view(torch.uint8))


def test_rows_of_zeros_tiny_and_infinite_values():
    x = torch.zeros(6, 24)
    x[1] = 1e-42
    x[2, 3] = 1e30
    x[3, 0] = float("inf")
    x[4, 7] = float("nan")
    x[5] = torch.arange(24) - 11.5
    x = x.to(DEV)
    y, s = torch.empty(6, 24, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(6, device=DEV)
    al.alcop_quantize_rows(x, y, s)
    y, s = y.float().cpu(), s.cpu()
    assert y[0].eq(0).all() and s[0] == 2.0 ** -126 and s[1] == 2.0 ** -126 and y[1].eq(0).all()
    assert y[2, 3] == 448 and y[2].sum() == 448
    assert s[3] == float("inf") and y[3, 0].isnan() and y[3, 1:].eq(0).all()
    assert s[4].isnan() and y[4].isnan().all() and y[5].isfinite().all()


@pytest.mark.parametrize("cols", COLS)
def test_norm_gradient_of_every_row_length(cols):
    k = COLS.index(cols)
    for rows, dtype, gain, dtotal, dgain, pad in ((7, ("bf16", "f16", "f32")[k % 3], True, True, True, (0, 3, 8)[k % 3]),
                                                  (1, ("f32", "bf16", "f16")[k % 3], k % 2 == 0, False, k % 3 == 0, 0)):
        dy, h = matrix(rows, cols, dtype, 1, pad), matrix(rows, cols, dtype, 2, pad, 2.0)
        g = vector(cols, 3) if gain else None
        rstd = (h.double().square().mean(1) + 1e-6).rsqrt().float()
        dt, dx = matrix(rows, cols, dtype, 4, pad) if dtotal else None, matrix(rows, cols, dtype, 5, pad)
        dg = vector(cols, 6) if dgain else None
        ws = torch.full((al.alcop_rmsnorm_backward_workspace_bytes(rows, cols),), 255, dtype=torch.uint8, device=DEV)
        al.alcop_rmsnorm_backward(dy, h, g, rstd, dx, dgain=dg, dtotal=dt, workspace=ws)
        torch.cuda.synchronize()
        ref, gref, edx, edg = norm_grad64(dy, h, g, rstd, dt)
        check(dx, ref, edx, "dx")
        assert padding(dx).isnan().all()
        if dgain:
            check(dg[None], gref[None], edg[None], "dgain")


@pytest.mark.parametrize("rows,cols", [(5000, 72), (3001, 1000), (2500, 1027), (1536, 2048), (1535, 2048), (2001, 1603), (2100, 4096)])
def test_norm_gradient_of_many_rows(rows, cols):
    dy, h, g = matrix(rows, cols, "bf16", 1), matrix(rows, cols, "bf16", 2), vector(cols, 3)
    rstd = (h.double().square().mean(1) + 1e-6).rsqrt().float()
    dg = vector(cols, 4)
    ws = torch.full((al.alcop_rmsnorm_backward_workspace_bytes(rows, cols),), 255, dtype=torch.uint8, device=DEV)
    dx = dy.clone()
    ref, gref, edx, edg = norm_grad64(dy, h, g, rstd, dy)
    al.alcop_rmsnorm_backward(dx, h, g, rstd, dx, dgain=dg, dtotal=dy, workspace=ws)        # in place
    torch.cuda.synchronize()
    check(dx, ref, edx, "dx")
    check(dg[None], gref[None], edg[None], "dgain")


# ---- together ---------------------------------------------------------------------------------------------
def test_a_feed_forward_block_in_8_bits():
    T, D, F = 300, 512, 2048
    x, r, g = matrix(T, D, "bf16", 1), matrix(T, D, "bf16", 2), vector(D, 3, True)
    w1, w2, b1 = matrix(F, D, "bf16", 4, scale=D ** -0.5), matrix(D, F, "bf16", 5, scale=F ** -0.5), vector(F, 6)
    f8 = lambda rows, cols: (torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(rows, device=DEV))
    (q1, s1), (q2, s2), (q3, s3), (q4, s4) = f8(F, D), f8(D, F), f8(T, D), f8(T, F)
    h, u, out = torch.empty_like(x), torch.empty(T, F, dtype=torch.bfloat16, device=DEV), torch.empty_like(x)
    al.alcop_quantize_rows(w1, q1, s1)
    al.alcop_quantize_rows(w2, q2, s2)

    def block():
        al.alcop_rmsnorm(x, g, q3, residual=r, total=h, scale=s3)
        al.alcop_linear(q3, q1, u, transB=True, bias=b1, act=4, scale_a=s3, scale_w=s1)
        al.alcop_quantize_rows(u, q4, s4)
        al.alcop_linear(q4, q2, out, transB=True, residual=h, scale_a=s4, scale_w=s2)

    block()
    torch.cuda.synchronize()
    ref, _, _, ec = linear64(q3, q1, True, 1.0, b1, 4, None, s3, s1)
    check(u, ref, ec)
    ref, _, _, ec = linear64(q4, q2, True, 1.0, None, 0, h, s4, s2)
    check(out, ref, ec)
    # captured, replayed with other inputs and eager work between the replays
    al.alcop_init()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block()
    for k in range(4):
        x.copy_(matrix(T, D, "bf16", 10 + k))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        block()
        torch.cuda.synchronize()
        assert torch.equal(got, out)


def test_a_feed_forward_block_in_training():
    T, D, F = 200, 256, 520
    x, r, g = matrix(T, D, "bf16", 1), matrix(T, D, "bf16", 2), vector(D, 3, True)
    w1, w2, b1 = matrix(F, D, "bf16", 4, scale=D ** -0.5), matrix(D, F, "bf16", 5, scale=F ** -0.5), vector(F, 6)
    dout = matrix(T, D, "bf16", 7)
    e = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device=DEV)
    f32 = torch.float32
    y, h, rstd, u, z, out = e(T, D), e(T, D), e(T, dt=f32), e(T, F), e(T, F), e(T, D)
    du, dw2, dy, dw1, db1, dx, dg = e(T, F), e(D, F, dt=f32), e(T, D), e(F, D, dt=f32), e(F, dt=f32), e(T, D), e(D, dt=f32)
    dy = e(T, D)
    ws1 = torch.empty(al.alcop_linear_backward_workspace_bytes(T, F, D), dtype=torch.uint8, device=DEV)
    ws2 = torch.empty(al.alcop_rmsnorm_backward_workspace_bytes(T, D), dtype=torch.uint8, device=DEV)

    def step():
        al.alcop_rmsnorm(x, g, y, residual=r, total=h, rstd=rstd)
        al.alcop_linear(y, w1, u, transB=True, bias=b1, act=3, pre=z)
        al.alcop_linear(u, w2, out, transB=True, residual=h)
        al.alcop_linear_backward(dout, u, w2, dA=du, transB=True)
        al.alcop_linear_backward(dout, u, w2, dW=dw2, transB=True)
        al.alcop_linear_backward(du, y, w1, dA=dy, dbias=db1, pre=z, act=3, transB=True, workspace=ws1)
        al.alcop_linear_backward(du, y, w1, dW=dw1, pre=z, act=3, transB=True, workspace=ws1)
        al.alcop_rmsnorm_backward(dy, h, g, rstd, dx, dgain=dg, dtotal=dout, workspace=ws2)

    step()
    torch.cuda.synchronize()
    # the whole in 64 bits by autograd; every stored tensor is rounded to bf16, half a step each, and a sum of n terms
    # whose errors are independent grows by their root: some ten roundings on the way, at 2^-8 of the values' size
    p = [t.cpu().double().requires_grad_(True) for t in (x, g, w1, b1, w2)]
    hh = p[0] + r.cpu().double()
    yy = hh * (hh.square().mean(1, keepdim=True) + 1e-6).rsqrt() * p[1]
    oo = torch.nn.functional.gelu(yy @ p[2].t() + p[3], approximate="tanh") @ p[4].t() + hh
    oo.backward(dout.cpu().double())
    for got, ref, name in zip((out, dx, dg, dw1, db1, dw2), (oo.detach(), *(p[i].grad for i in (0, 1, 2, 3, 4))),
                              ("out", "dx", "dgain", "dw1", "db1", "dw2")):
        err = float((got.cpu().double() - ref).norm() / ref.norm())
        assert err <= 10 * 2.0 ** -8, (name, err)
    # captured beside a second capture with a workspace of its own: both replay to the eager bits
    want = [t.clone() for t in (out, dx, dg, dw1, db1, dw2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in (out, dx, dg, dw1, db1, dw2):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (out, dx, dg, dw1, db1, dw2)))


def test_on_a_stream_of_the_callers():
    A, W = matrix(100, 512, "f16", 1), matrix(136, 512, "f16", 2)
    C, D = torch.empty(100, 136, device=DEV), torch.empty(100, 136, device=DEV)
    al.alcop_linear(A, W, D, transB=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    al.alcop_linear(A, W, C, transB=True, stream=s)
    s.synchronize()
    with torch.cuda.stream(s):
        E = torch.empty_like(C)
        al.alcop_linear(A, W, E, transB=True)
    s.synchronize()
    assert torch.equal(C, D) and torch.equal(E, D)
