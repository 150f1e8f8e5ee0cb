"""On the GPU: rows to 8 bits are those of the definition, bit for bit; activations and slopes are near relative to
their size; sums of layers on e4m3 operands are within the bound of the 8-bit matrix instruction, or fp32."""
import pytest
import torch

import paper_2210_16691_amd as al
from gpu_util import DEV
from layers_util import ULP, check, check_e4m3, linear64, norm64, norm_grad64
from sums8_util import cancelling, check_sums, quantized_pair
from test_gpu_z11_layers import matrix, padding, run_backward, vector
from test_layers_accuracy import check_activation, check_slope
from test_rows_exact import plain, same, values

pytestmark = pytest.mark.gpu


def quantized(x):
    y, s = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(x.shape[0], device=DEV)
    al.alcop_quantize_rows(x.to(DEV), y, s)
    torch.cuda.synchronize()
    return y.cpu(), s.cpu()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(3000, 72), (700, 1000), (1700, 1600), (60, 1603), (200, 4096), (50, 9000), (30, 32767)])
def test_quotients_are_rounded_once_to_fp32(dtype, rows, cols):
    x = values(rows, cols, dtype, cols)
    same(quantized(x), plain(x))


@pytest.mark.parametrize("dtype,scale", [("f32", 1e-42), ("f32", 3e-38), ("f32", 1e-36), ("f32", 1e-20), ("f32", 1e-18), ("f32", 1e37),
                                         ("bf16", 1e-38), ("bf16", 1e-36), ("bf16", 1e-19), ("bf16", 6e37), ("f16", 1e-7), ("f16", 1e4)])
def test_quotients_of_tiny_and_huge_rows(dtype, scale):
    x = values(300, 520, dtype, 7, scale)
    x[:, 3], x[:, 4] = 0.0, -0.0
    x[5] = x[5].sign() * x[5].abs().amax()
    same(quantized(x), plain(x))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(9, 1032), (1600, 1536), (300, 4096)])
def test_an_8_bit_norm_is_its_fp32_norm_divided(dtype, rows, cols):
    x, r = values(rows, cols, dtype, 1, 2.0).to(DEV), values(rows, cols, dtype, 2).to(DEV)
    g = torch.randn(cols, generator=torch.Generator().manual_seed(3)).to(DEV)
    y32, s = torch.empty(rows, cols, device=DEV), torch.empty(rows, device=DEV)
    y = torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device=DEV)
    al.alcop_rmsnorm(x, g, y32, residual=r)
    al.alcop_rmsnorm(x, g, y, residual=r, scale=s)
    torch.cuda.synchronize()
    same((y.cpu(), s.cpu()), plain(y32.cpu()))


def on_the_gpu(fn, *args, reads=None, writes=None, **kw):
    fn(*args, **kw)
    torch.cuda.synchronize()


@pytest.mark.parametrize("act", [2, 3, 4])
def test_activations_are_near_relative_to_their_value(act):
    check_activation(on_the_gpu, act, DEV)


@pytest.mark.parametrize("act", [2, 3, 4])
def test_slopes_are_near_relative_to_their_terms(act):
    check_slope(on_the_gpu, act, DEV)


KERNELS, F8_KERNELS = 11, 6


@pytest.mark.parametrize("kernel", range(KERNELS, KERNELS + F8_KERNELS))
def test_sums_of_the_8_bit_instruction(kernel, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    M, N, K = 513, 776, 2064
    A, W, sa, sw = quantized_pair(M, N, K, kernel, DEV)
    for out, act in ((torch.float16, 0), (torch.float16, 2), (torch.bfloat16, 4)):
        C, z = torch.empty(M, N, dtype=out, device=DEV), torch.empty(M, N, dtype=out, device=DEV)
        al.alcop_linear(A, W, C, transB=True, act=act, pre=z, scale_a=sa, scale_w=sw)
        torch.cuda.synchronize()
        check_sums(C, z, A, W, act=act, sa=sa, sw=sw)
    A, W, exact = cancelling(300, 264, 1024, DEV)
    C = torch.empty(300, 264, dtype=torch.float16, device=DEV)
    al.alcop_linear(A, W, C, transB=True)
    torch.cuda.synchronize()
    check_sums(C, None, A, W, random=False)
    assert C.eq(0).all()


def test_sums_of_every_8_bit_number(monkeypatch):
    # all exponents, numbers below 2^-6 among them
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(KERNELS))
    g = torch.Generator().manual_seed(1)
    for low, span in ((0, 127), (0, 24), (70, 57)):
        A, W = ((torch.randint(0, span, (256, 512), generator=g) + low + 128 * torch.randint(0, 2, (256, 512), generator=g))
                .to(torch.uint8).view(torch.float8_e4m3fn).to(DEV) for _ in range(2))
        C = torch.empty(256, 256, dtype=torch.bfloat16, device=DEV)
        al.alcop_linear(A, W, C, transB=True)
        torch.cuda.synchronize()
        check_sums(C, None, A, W, random=False)


@pytest.mark.parametrize("M,N,K", [(1, 264, 1024), (40, 264, 1024), (300, 520, 1024), (2048, 2056, 1040)])
def test_fp32_sums_that_are_asked_for(M, N, K):
    A, W, exact = cancelling(M, N, K // 8 * 8, DEV)
    for act in (0, 4):
        C, z = torch.empty(M, N, dtype=torch.float16, device=DEV), torch.empty(M, N, dtype=torch.float16, device=DEV)
        al.alcop_linear(A, W, C, transB=True, act=act, pre=z, fp32_sums=True)
        torch.cuda.synchronize()
        assert z.eq(exact).all()
        check(C, *linear64(A, W, True, act=act)[::3])
    A, W, sa, sw = quantized_pair(M, N, K, 3, DEV)
    C = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    al.alcop_linear(A, W, C, transB=True, scale_a=sa, scale_w=sw, fp32_sums=True)
    torch.cuda.synchronize()
    check(C, *linear64(A, W, True, sa=sa, sw=sw)[::3])


# ---- rows that have a wave each --------------------------------------------------------------------------
@pytest.mark.parametrize("rows,cols", [(1535, 2048), (1536, 2048), (1537, 1025), (2001, 1603), (3000, 1536)])
@pytest.mark.parametrize("dtype,out", [("f16", "e4m3"), ("bf16", "e4m3"), ("f32", "e4m3"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "f32"),
                                       ("bf16", "f32")])
def test_norms_of_many_rows(rows, cols, dtype, out):
    pad = 3 if cols % 8 else 8
    x, r, h = (matrix(rows, cols, dtype, s, pad, 2.0) for s in (1, 2, 3))
    g, d, s = vector(cols, 4), vector(rows, 5), vector(rows, 6) if out == "e4m3" else None
    y = matrix(rows, cols, out, 7, pad)
    yref, href, dref = norm64(x, r, g)
    al.alcop_rmsnorm(x, g, y, residual=r, total=h, scale=s, rstd=d)
    torch.cuda.synchronize()
    err = (cols / 2 + 8) * ULP
    check(d[:, None], dref[:, None], err * dref[:, None], "rstd")
    check(h, href, ULP * href.abs(), "total")
    if out == "e4m3":
        # h is rounded once to fp32 before its norm
        check_e4m3(y, s, yref, err + ULP, "y")
    else:
        check(y, yref, err * yref.abs() + ULP * href.abs() * dref[:, None] * g.cpu().double().abs(), "y")
    for t in (h, y):
        assert padding(t).float().isnan().all()
    # without residual, sum and gain; the sum in the residual's place
    y32, total = torch.empty(rows, cols, device=DEV), r.clone()
    al.alcop_rmsnorm(x, None, y32)
    check(y32, norm64(x)[0], err * norm64(x)[0].abs(), "y")
    al.alcop_rmsnorm(x, g, matrix(rows, cols, out, 8, pad), residual=total, total=total, scale=s)
    assert torch.equal(total, h)


def test_rows_that_have_a_wave_each_in_a_captured_graph():
    rows, cols = 2000, 1600
    x, r, h, y = (matrix(rows, cols, "bf16", s) for s in (1, 2, 3, 4))
    g, q, s = vector(cols, 5), torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device=DEV), vector(rows, 6)
    al.alcop_init()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        al.alcop_rmsnorm(x, g, y, residual=r, total=h)
        al.alcop_quantize_rows(y, q, s)
    for k in range(3):
        x.copy_(matrix(rows, cols, "bf16", 10 + k))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (h, y, s)] + [q.view(torch.uint8).clone()]
        al.alcop_rmsnorm(x, g, y, residual=r, total=h)
        al.alcop_quantize_rows(y, q, s)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (h, y, s, q.view(torch.uint8))))


# ---- split sums ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("M,N,K,transB,act", [(5856, 64, 1400, True, 0), (8192, 256, 264, False, 3), (16384, 256, 256, True, 2)])
@pytest.mark.parametrize("alpha", [0.5, -1.75])
def test_split_weight_gradients_with_a_factor(M, N, K, transB, act, alpha):
    run_backward(M, N, K, "bf16", transB, act, alpha=alpha)
    run_backward(M, N, K, "f16", transB, act, out="f32", alpha=alpha, bias=False)


# ---- every kernel there is ---------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,transB", [("f16", False), ("f16", True), ("bf16", False), ("bf16", True), ("e4m3", True)])
@pytest.mark.parametrize("act", [1, 2, 3])        # one of each class of activation: a kernel each
def test_every_kernel_of_every_class_of_activation(dtype, transB, act, monkeypatch):
    M, N, K = 270, 264, 208
    A, W = matrix(M, K, dtype, 1, 16), matrix(*((N, K) if transB else (K, N)), dtype, 2, 16, scale=K ** -0.5)
    b, r = vector(N, 3), {o: matrix(M, N, o, 4) for o in ("f16", "bf16", "f32")}
    for kernel in range(KERNELS + (F8_KERNELS if dtype == "e4m3" else 0)):
        monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
        for out in ("f16", "bf16", "f32"):
            if kernel >= KERNELS and out == "f32":
                continue
            C, z = matrix(M, N, out, 5, 8), matrix(M, N, out, 6, 8)
            al.alcop_linear(A, W, C, transB=transB, bias=b, act=act, residual=r[out], pre=z)
            torch.cuda.synchronize()
            what = "kernel %d %s" % (kernel, out)
            if kernel >= KERNELS:
                check_sums(C, z, A, W, bias=b, act=act, residual=r[out], random=False, what=what)
            else:
                ref, zref, ez, ec = linear64(A, W, transB, 1.0, b, act, r[out])
                check(C, ref, ec, "C " + what)
                check(z, zref, ez, "pre " + what)
            assert padding(C).isnan().all() and padding(z).isnan().all()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("rows,cols", [(9, 512), (9, 1024), (5, 2048), (1536, 2048), (5, 4096), (5, 8192), (3, 16384), (3, 32768)])
def test_every_kernel_of_rows(dtype, whole, rows, cols):
    cols -= 0 if whole else 3
    x, r, h = (matrix(rows, cols, dtype, s, 5, 2.0) for s in (1, 2, 3))
    g, d = vector(cols, 4), vector(rows, 5)
    err = (cols / 2 + 8) * ULP
    yref, href, dref = norm64(x, r, g)
    for out in ("f16", "bf16", "f32", "e4m3"):
        y, s = matrix(rows, cols, out, 6, 5), vector(rows, 7) if out == "e4m3" else None
        al.alcop_rmsnorm(x, g, y, residual=r, total=h, scale=s, rstd=d)
        torch.cuda.synchronize()
        if out == "e4m3":
            check_e4m3(y, s, yref, err + ULP, out)
        else:
            check(y, yref, err * yref.abs() + ULP * href.abs() * dref[:, None] * g.cpu().double().abs(), out)
        assert padding(y).float().isnan().all()
    check(h, href, ULP * href.abs(), "total")
    dy, dt, dx, dg = matrix(rows, cols, dtype, 8, 5), matrix(rows, cols, dtype, 9, 5), matrix(rows, cols, dtype, 10, 5), vector(cols, 11)
    ws = torch.full((al.alcop_rmsnorm_backward_workspace_bytes(rows, cols),), 255, dtype=torch.uint8, device=DEV)
    al.alcop_rmsnorm_backward(dy, h, g, d, dx, dgain=dg, dtotal=dt, workspace=ws)
    torch.cuda.synchronize()
    ref, gref, edx, edg = norm_grad64(dy, h, g, d, dt)
    check(dx, ref, edx, "dx")
    check(dg[None], gref[None], edg[None], "dgain")
    assert padding(dx).isnan().all()
