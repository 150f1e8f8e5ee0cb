"""The layer norm and its gradients on the GPU against their plain forms in 64 bits (on the CPU): every kernel, types, pitches,
rows far from zero, captured graphs, streams."""
import pytest
import torch

import paper_2210_16691_amd as al
from gpu_util import DEV
from layers_util import DT, ULP, check, check_e4m3
from more_util import layernorm64, layernorm_grad64
from test_gpu_z11_layers import matrix, padding, vector

pytestmark = pytest.mark.gpu
# columns that between them reach every kernel, whole chunks and not
COLS = [1, 40, 512, 513, 1024, 1111, 2048, 2049, 4096, 5001, 8192, 9000, 16384, 20001, 32768]


def run_norm(rows, cols, dtype, out, residual=True, gain=True, shift=True, total=True, pad=0, offset=0, far=0.0):
    x = matrix(rows, cols, dtype, 1, pad, offset=offset)
    x += far
    r = matrix(rows, cols, dtype, 2, pad, offset=offset) if residual else None
    g, b = vector(cols, 3) if gain else None, vector(cols, 4) if shift else None
    h = matrix(rows, cols, dtype, 5, pad, offset=offset) if total else None
    y = matrix(rows, cols, "bf16" if out == "e4m3" else out, 6, pad, offset=offset)
    if out == "e4m3":
        y = torch.zeros(rows, cols + pad, dtype=DT[out], device=DEV)[:, :cols]
    s = vector(rows, 7) if out == "e4m3" else None
    mean, rstd = vector(rows, 8), vector(rows, 9)
    yr, hr, mr, rr, ey, em, er = layernorm64(x, r, g, b)
    al.alcop_layernorm(x, g, b, y, residual=r, total=h, scale=s, mean=mean, rstd=rstd)
    torch.cuda.synchronize()
    check(mean[None], mr[None], em[None], "mean")
    check(rstd[None], rr[None], (er * rr)[None], "rstd")
    if total:
        check(h, hr, ULP * hr.abs(), "total")
        assert padding(h).isnan().all()
    if out == "e4m3":
        top = yr.abs().amax(dim=1, keepdim=True).clamp_min(1e-30)
        check_e4m3(y, s, yr, float((ey / top).max()) + 4 * ULP, "y")
    else:
        check(y, yr, ey, "y")
        assert padding(y).isnan().all()


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f16", "e4m3"), ("f32", "f32")])
def test_norms(cols, dtype, out):
    run_norm(37, cols, dtype, out, pad=3, offset=1)
    run_norm(1, cols, dtype, out, residual=False, total=False)


def test_norms_of_many_rows():
    run_norm(1536, 2048, "bf16", "bf16")
    run_norm(5000, 1200, "f16", "f16", residual=False, pad=8)
    run_norm(20000, 72, "bf16", "e4m3")


@pytest.mark.parametrize("cols", [64, 100, 128, 129, 250, 256])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f16", "e4m3"), ("f32", "f32")])
def test_short_rows(cols, dtype, out):
    for rows in (1, 4, 5, 15, 17, 3001):
        run_norm(rows, cols, dtype, out, pad=3 * (rows % 2), offset=rows % 2)
        x, g, r, b = matrix(rows, cols, dtype, 1), vector(cols, 2), matrix(rows, cols, dtype, 3), vector(cols, 4)
        y, h = torch.empty_like(x), torch.empty_like(x)
        al.alcop_layernorm(x, g, b, y, residual=r, total=h)
        al.alcop_layernorm(x, g, b, r, residual=r, total=x)
        torch.cuda.synchronize()
        assert torch.equal(x, h) and torch.equal(r, y)


def test_rows_far_from_zero():
    for cols in (1000, 4096, 16384):
        run_norm(9, cols, "f32", "f32", residual=False, far=3000.0)


def run_grad(rows, cols, dtype, dtotal=True, gain=True, dgain=True, dshift=True, pad=0, offset=0, in_place=False):
    dy = matrix(rows, cols, dtype, 1, pad, offset=offset)
    h = matrix(rows, cols, dtype, 2, pad, scale=2.0, offset=offset)
    dt = matrix(rows, cols, dtype, 3, pad, offset=offset) if dtotal else None
    g = vector(cols, 4) if gain else None
    mean, rstd = 0.1 * vector(rows, 5), vector(rows, 6, True)
    dg, ds = vector(cols, 8) if dgain else None, vector(cols, 9) if dshift else None
    ws = torch.empty(al.alcop_layernorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    dxr, dgr, dsr, edx, edg, eds = layernorm_grad64(dy, h, g, mean, rstd, dt)
    dx = (dt if dtotal else dy) if in_place else matrix(rows, cols, dtype, 7, pad, offset=offset)
    al.alcop_layernorm_backward(dy, h, g, mean, rstd, dx, dgain=dg, dshift=ds, dtotal=dt, workspace=ws)
    torch.cuda.synchronize()
    check(dx, dxr, edx, "dx")
    assert padding(dx).isnan().all()
    if dgain:
        check(dg[None], dgr[None], edg[None], "dgain")
    if dshift:
        check(ds[None], dsr[None], eds[None], "dshift")


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_gradients(cols, dtype):
    run_grad(37, cols, dtype, pad=3, offset=1)
    run_grad(1, cols, dtype, dtotal=False, gain=False)


@pytest.mark.parametrize("cols", [64, 100, 128, 129, 250, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_gradients_of_short_rows(cols, dtype):
    for rows in (1, 4, 5, 35, 3001, 9001):
        run_grad(rows, cols, dtype, pad=3 * (rows % 2), offset=rows % 2)
        run_grad(rows, cols, dtype, in_place=True)
        run_grad(rows, cols, dtype, dtotal=False, dgain=False)


def test_gradients_of_many_rows():
    run_grad(1536, 2048, "bf16")
    run_grad(6000, 1200, "f16", pad=8)
    run_grad(20000, 72, "f32")


def test_gradients_left_out_or_in_place():
    for kw in (dict(dgain=False), dict(dshift=False, in_place=True), dict(dgain=False, dshift=False, dtotal=False, in_place=True)):
        run_grad(300, 1000, "f16", **kw)


def test_gradients_against_differences():
    g = torch.Generator().manual_seed(3)
    rows, cols, step = 3, 24, 2.0 ** -7
    x, gain, shift, dy = (torch.randn(s, generator=g).to(DEV) for s in ((rows, cols), (cols,), (cols,), (rows, cols)))
    ws = torch.empty(al.alcop_layernorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)

    def loss(x, gain, shift):
        y = torch.empty_like(x)
        al.alcop_layernorm(x, gain, shift, y)
        return float((y.double() * dy.double()).sum())

    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    al.alcop_layernorm(x, gain, shift, y, mean=mean, rstd=rstd)
    dx, dg, ds = torch.empty_like(x), torch.empty_like(gain), torch.empty_like(shift)
    al.alcop_layernorm_backward(dy, x, gain, mean, rstd, dx, dgain=dg, dshift=ds, workspace=ws)
    for i, (t, grad) in enumerate(((x, dx), (gain, dg), (shift, ds))):
        for at in range(0, t.numel(), 5):
            v = []
            for h in (step, -step):
                args = [x.clone(), gain.clone(), shift.clone()]
                args[i].view(-1)[at] += h
                v.append(loss(*args))
            # the difference quotient: fp32 outputs of 72 terms below 8 each, off by 2^-22 of them, over 2^-6; the third derivative
            # of a row's norm, below 40 here, times step^2 / 6
            assert abs((v[0] - v[1]) / (2 * step) - float(grad.view(-1)[at])) < 72 * 8 * 2.0 ** -22 * 64 + 40 * step ** 2 / 6


def test_a_captured_graph_gives_the_eager_bits():
    rows, cols = 700, 1111
    x, r, dy = (matrix(rows, cols, "bf16", s) for s in (1, 2, 3))
    g, b = vector(cols, 4), vector(cols, 5)
    ws = torch.empty(al.alcop_layernorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)

    def outputs():
        return [torch.zeros_like(x) for _ in range(3)] + [torch.zeros(rows, device=DEV) for _ in range(2)] + \
            [torch.zeros(cols, device=DEV) for _ in range(2)]

    def step(y, h, dx, mean, rstd, dg, ds):
        al.alcop_layernorm(x, g, b, y, residual=r, total=h, mean=mean, rstd=rstd)
        al.alcop_layernorm_backward(dy, h, g, mean, rstd, dx, dgain=dg, dshift=ds, workspace=ws)

    al.alcop_init()
    caught, graph, side = outputs(), torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        step(*caught)
    for seed in (11, 12, 13):
        x.copy_(matrix(rows, cols, "bf16", seed))
        eager = outputs()
        step(*eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, e) for a, e in zip(caught, eager))


def test_a_stream_of_the_callers_own():
    x, y = matrix(64, 1000, "bf16", 1), torch.zeros(64, 1000, dtype=torch.bfloat16, device=DEV)
    ref = torch.zeros_like(y)
    al.alcop_layernorm(x, None, None, ref)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    al.alcop_layernorm(x, None, None, y, stream=s)
    s.synchronize()
    assert torch.equal(y, ref)
