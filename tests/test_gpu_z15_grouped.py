"""Products grouped by expert and their gradients on the GPU against their plain forms in 64 bits (on the CPU): every kernel,
types, layouts, ragged groups, captured graphs, streams."""
import os

import pytest
import torch

import paper_2210_16691_amd as al
from gpu_util import DEV
from layers_util import DT, check
from more_util import grouped64, grouped_grad64
from test_gpu_z11_layers import matrix, padding, vector
from test_grouped_emulated import F8_KERNELS, GRADIENT_KERNELS, KERNELS, groups_of, offsets_of, rows_of

pytestmark = pytest.mark.gpu


def run_grouped(sizes, N, K, dtype, transB, out="bf16", act=0, bias=True, pre=True, scales=False, pad=0, alpha=1.0, first=0, behind=0,
                offset=0):
    G, rows = len(sizes), first + sum(sizes) + behind
    A = matrix(rows, K, dtype, 1, pad)
    W = groups_of(matrix(G * (N if transB else K), K if transB else N, dtype, 2, pad, scale=K ** -0.5), G)
    offs = offsets_of(sizes, first).to(DEV)
    C = matrix(rows, N, out, 3, pad, offset=offset)
    z = matrix(rows, N, out, 4, pad, offset=offset) if pre else None
    b = vector(G * N, 5).view(G, N) if bias else None
    sa, sw = (vector(rows, 6, True), vector(G * N, 7, True).view(G, N)) if scales else (None, None)
    before = C.clone()
    c, zr, ez, ec = grouped64(A, W, sizes, first, transB, alpha, b, act, sa, sw, dtype == "e4m3" and out != "f32")
    al.alcop_grouped_linear(A, W, offs, C, transB=transB, alpha=alpha, bias=b, act=act, pre=z, scale_a=sa, scale_w=sw)
    torch.cuda.synchronize()
    part = rows_of(sizes, first)
    what = str((sizes, N, K, dtype, transB, out, act))
    if sum(sizes):
        check(C[part], c[part], ec[part], "C " + what)
    assert padding(C).isnan().all(), what
    if pre and sum(sizes):
        check(z[part], zr[part], ez[part], "pre " + what)
        assert padding(z).isnan().all(), what
    for rest in (slice(0, first), slice(part.stop, rows)):
        assert torch.equal(C[rest], before[rest])


@pytest.mark.parametrize("kernel", range(KERNELS))
@pytest.mark.parametrize("dtype,transB", [("f16", False), ("f16", True), ("bf16", False), ("bf16", True), ("e4m3", True)])
def test_every_kernel(kernel, dtype, transB, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    i = kernel + 10 * transB + 20 * (dtype == "bf16")
    run_grouped([0, 1, 17, 130, 0, 16, 256, 3, 300], 408, 208, dtype, transB, out=("f16", "bf16", "f32")[i % 3], act=i % 5,
                scales=dtype == "e4m3" or i % 2 == 0, pad=16, first=i % 3, behind=5)
    run_grouped([513, 0, 65], 776, 1040, dtype, transB, out=("f16", "bf16", "f32")[(i + 1) % 3], act=(i + 2) % 5)


@pytest.mark.parametrize("kernel,dtype,transB", [(KERNELS - 1, "f16", False), (KERNELS - 1, "bf16", True), (KERNELS - 1, "e4m3", True),
                                                 (KERNELS - 2, "f16", True), (KERNELS - 2, "bf16", False), (KERNELS - 2, "e4m3", True),
                                                 (KERNELS + F8_KERNELS - 1, "e4m3", True), (KERNELS + F8_KERNELS - 2, "e4m3", True)])
def test_whole_turns_of_the_large_tiles_and_quarters_behind_them(kernel, dtype, transB, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    run_grouped([(3, 130, 0, 257, 1)[g % 5] for g in range(256)] + [5, 300, 129], 264, 208, dtype, transB, act=2, pad=16, first=2,
                behind=5)
    run_grouped([1] * 256, 256, 80, dtype, transB, pre=False)
    run_grouped([2] * 257, 200, 80, dtype, transB, pre=False)


@pytest.mark.parametrize("kernel", range(KERNELS, KERNELS + F8_KERNELS))
@pytest.mark.parametrize("act", [0, 2, 4])
def test_every_kernel_that_multiplies_8_bits_as_they_are(kernel, act, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    run_grouped([5, 0, 267, 128], 413, 720, "e4m3", True, out=("f16", "bf16")[kernel % 2], act=act, scales=True, pad=16)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "e4m3"])
def test_few_rows_and_many_groups(dtype):
    run_grouped([1], 776, 1040, dtype, True, act=3)
    run_grouped([(5 * g) % 4 for g in range(64)], 1029, 528, dtype, True, out="f32", pre=False, scales=True)
    run_grouped([(7 * g) % 5 for g in range(200)], 72, 64, dtype, True, first=3, behind=4)
    run_grouped([0] * 7, 72, 64, dtype, True, first=3, behind=4)


@pytest.mark.parametrize("N,pad,offset", [(43, 16, 0), (200, 8, 1), (1, 16, 0)])
def test_results_that_are_not_made_of_chunks(N, pad, offset):
    for sizes in ([5, 0, 18], [300, 0, 217]):
        run_grouped(sizes, N, 96, "f16", True, out="bf16", act=4, pad=pad, offset=offset)


def test_larger_products():
    run_grouped([700, 0, 1300, 48], 2056, 528, "bf16", True, act=2)
    run_grouped([1111, 900], 1032, 1024, "f16", False, act=4, pre=False, pad=16)
    run_grouped([500, 3, 1500], 2048, 1024, "e4m3", True, scales=True, pre=False)


def run_backward(sizes, N, K, dtype, transB, out=None, act=0, pad=0, alpha=1.0, first=0, behind=0, parts="AWb"):
    G, rows = len(sizes), first + sum(sizes) + behind
    dC, A = matrix(rows, N, dtype, 1, pad), matrix(rows, K, dtype, 2, pad)
    w_shape = (N, K) if transB else (K, N)
    W = groups_of(matrix(G * w_shape[0], w_shape[1], dtype, 3, pad, scale=K ** -0.5), G)
    pre = matrix(rows, N, dtype, 4, pad) if act else None
    offs = offsets_of(sizes, first).to(DEV)
    dA = matrix(rows, K, out or dtype, 5, pad) if "A" in parts else None
    dWm = matrix(G * w_shape[0], w_shape[1], out or dtype, 6, pad) if "W" in parts else None
    dW = None if dWm is None else groups_of(dWm, G)
    db = vector(G * N, 7).view(G, N) if "b" in parts else None
    ws = torch.empty(al.alcop_grouped_linear_backward_workspace_bytes(rows, G, N, K), dtype=torch.uint8, device=DEV).fill_(255)
    before = None if dA is None else dA.clone()
    ra, rw, rb, ea, ew, eb = grouped_grad64(dC, A, W, sizes, first, transB, pre, act, alpha)
    al.alcop_grouped_linear_backward(dC, A, W, offs, dA=dA, dW=dW, dbias=db, pre=pre, act=act, alpha=alpha, transB=transB, workspace=ws)
    torch.cuda.synchronize()
    part = rows_of(sizes, first)
    if dA is not None:
        if sum(sizes):
            check(dA[part], ra[part], ea[part], "dA")
        assert padding(dA).isnan().all()
        for rest in (slice(0, first), slice(part.stop, rows)):
            assert torch.equal(dA[rest], before[rest])
    if dW is not None:
        for g in range(G):
            check(dW[g], rw[g], ew[g], "dW of group %d" % g)
        assert padding(dWm).isnan().all()
    if db is not None:
        check(db, rb, eb, "dbias")


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("dtype,transB", [("f16", False), ("f16", True), ("bf16", False), ("bf16", True)])
def test_gradients(act, dtype, transB):
    run_backward([3, 0, 41, 1, 70, 333], 200, 136, dtype, transB, act=act, pad=8, first=2, behind=3)


@pytest.mark.parametrize("kernel", range(GRADIENT_KERNELS))
@pytest.mark.parametrize("dtype,transB", [("f16", True), ("bf16", False)])
def test_gradients_of_every_kernel(kernel, dtype, transB, monkeypatch):
    # the weights' gradients by their own kernels, the rows' by those of the product
    monkeypatch.setenv("ALCOP_GRADIENT_KERNEL", str(kernel))
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel + 4))
    run_backward([3, 0, 41, 1, 270, 700], 328, 264, dtype, transB, act=4, pad=8, first=2, behind=3)


def test_gradients_of_larger_products():
    run_backward([700, 0, 900, 17], 520, 264, "bf16", True, act=4)
    run_backward([300, 2, 2500], 1032, 520, "f16", False, act=2, out="f32", alpha=0.5)
    run_backward([(3 * g) % 40 for g in range(150)], 72, 64, "bf16", True, act=1)


def test_gradients_left_out():
    for parts in ("A", "W", "b", "Ab", "Wb"):
        run_backward([3, 0, 120], 72, 40, "f16", True, act=2, parts=parts)
        run_backward([3, 0, 120], 72, 40, "f16", False, act=0, parts=parts, out="f32", alpha=-0.5)
    run_backward([0, 0], 24, 40, "f16", True, act=2, first=1, behind=2)


def test_gradients_against_differences():
    # fp32 results of products of small fp16 integers and steps of 2^-5: the quadratic form is exact, so its differences are too
    g = torch.Generator().manual_seed(5)
    sizes, N, K = [3, 0, 5], 8, 16
    A, W = torch.randint(-3, 4, (8, K), generator=g), torch.randint(-3, 4, (3, N, K), generator=g)
    A, W = A.to(DEV, torch.float16), W.to(DEV, torch.float16)
    dC = torch.randint(-3, 4, (8, N), generator=g).to(DEV, torch.float16)
    offs = offsets_of(sizes).to(DEV)

    def value(A, W):
        C = torch.zeros(8, N, device=DEV)
        al.alcop_grouped_linear(A, W, offs, C, transB=True)
        return float((C.double() * dC.double()).sum())

    dA, dW = torch.zeros(8, K, device=DEV), torch.zeros(3, N, K, device=DEV)
    al.alcop_grouped_linear_backward(dC, A, W, offs, dA=dA, dW=dW, transB=True)
    for t, grad, i in ((A, dA, 0), (W, dW, 1)):
        for at in range(0, t.numel(), 7):
            v = []
            for h in (1.0, -1.0):
                args = [A.clone(), W.clone()]
                args[i].view(-1)[at] += h
                v.append(value(*args))
            assert (v[0] - v[1]) / 2 == float(grad.view(-1)[at])


def test_a_captured_graph_follows_the_offsets():
    rows, G, N, K = 600, 5, 264, 136
    A, dC, pre = matrix(rows, K, "bf16", 1), matrix(rows, N, "bf16", 2), matrix(rows, N, "bf16", 3)
    W, b = groups_of(matrix(G * N, K, "bf16", 4, scale=0.1), G), vector(G * N, 5).view(G, N)
    offs = offsets_of([100, 100, 100, 100, 200]).to(DEV)
    ws = torch.empty(al.alcop_grouped_linear_backward_workspace_bytes(rows, G, N, K), dtype=torch.uint8, device=DEV)

    def outputs():
        return (torch.zeros(rows, N, dtype=torch.bfloat16, device=DEV), torch.zeros(rows, K, dtype=torch.bfloat16, device=DEV),
                torch.zeros(G, N, K, dtype=torch.bfloat16, device=DEV), torch.zeros(G, N, device=DEV))

    def step(C, dA, dW, db):
        al.alcop_grouped_linear(A, W, offs, C, transB=True, bias=b, act=4)
        al.alcop_grouped_linear_backward(dC, A, W, offs, dA=dA, dW=dW, dbias=db, pre=pre, act=4, transB=True, workspace=ws)

    al.alcop_init()
    caught, graph = outputs(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        step(*caught)
    for sizes in ([0, 600, 0, 0, 0], [1, 2, 3, 4, 590], [120] * 5, [300, 0, 0, 0, 300]):
        offs.copy_(offsets_of(sizes))
        eager = outputs()
        step(*eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, e) for a, e in zip(caught, eager)), sizes


def test_two_streams_and_the_same_bits_again():
    rows, G, N, K = 200, 8, 520, 264
    A, W = matrix(rows, K, "f16", 1), groups_of(matrix(G * N, K, "f16", 2, scale=0.1), G)
    offs = offsets_of([25] * 8).to(DEV)
    first = torch.zeros(rows, N, dtype=torch.float16, device=DEV)
    al.alcop_grouped_linear(A, W, offs, first, transB=True, act=3)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.zeros_like(first) for _ in range(2)]
    for s, o in zip(streams, outs):
        al.alcop_grouped_linear(A, W, offs, o, transB=True, act=3, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in outs)


def test_as_many_groups_as_gradients_take():
    # rows of 8 against 8 x 8 weights, a few of every eight groups without any
    G, sizes = 64000, torch.tensor([(0, 1, 3, 0, 2, 1, 1, 1)[g % 8] for g in range(64000)])
    offs = torch.cat([torch.zeros(1, dtype=torch.int64), sizes.cumsum(0)])
    rows = int(offs[-1])
    A, dC, W = matrix(rows, 8, "f16", 1), matrix(rows, 8, "f16", 2), matrix(G * 8, 8, "f16", 3, scale=0.3).view(G, 8, 8)
    dA, dW, db = torch.full_like(A, float("nan")), torch.full_like(W, float("nan")), torch.full((G, 8), float("nan"), device=DEV)
    ws = torch.empty(al.alcop_grouped_linear_backward_workspace_bytes(rows, G, 8, 8), dtype=torch.uint8, device=DEV)
    al.alcop_grouped_linear_backward(dC, A, W, offs.to(DEV, torch.int32), dA=dA, dW=dW, dbias=db, transB=True, workspace=ws)
    torch.cuda.synchronize()
    of = torch.repeat_interleave(torch.arange(G), sizes)
    a, c, w = A.cpu().double(), dC.cpu().double(), W.cpu().double()
    # half a step of fp16 beside fp32 sums of 8 products, or of 3 rows
    for got, exact, size in (
            (dA, (c[:, :, None] * w[of]).sum(1), (c.abs()[:, :, None] * w[of].abs()).sum(1)),
            (dW, torch.zeros(G, 8, 8, dtype=torch.float64).index_add_(0, of, c[:, :, None] * a[:, None, :]),
             torch.zeros(G, 8, 8, dtype=torch.float64).index_add_(0, of, (c[:, :, None] * a[:, None, :]).abs())),
            (db, torch.zeros(G, 8, dtype=torch.float64).index_add_(0, of, c), torch.zeros(G, 8, dtype=torch.float64).index_add_(0, of, c.abs()))):
        bound = exact.abs() * (2.0 ** -11 if got.dtype == torch.float16 else 2.0 ** -24) + size * 16 * 2.0 ** -24 + 2.0 ** -25
        assert ((got.cpu().double() - exact).abs() <= bound).all()
