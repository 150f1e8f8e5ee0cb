"""The layer norm and its gradients on the CPU model of the hardware (tests/emu): bounds of every access, barriers, results
against the plain forms in 64 bits."""
import pytest
import torch

import emu_util as emu
import paper_2210_16691_amd as al
from layers_util import DT, ULP, check, check_e4m3
from more_util import layernorm64, layernorm_grad64
from test_layers_emulated import matrix, some, vector


def run_norm(rows, cols, dtype, out, residual=True, gain=True, shift=True, total=True, pad=0, offset=0, far=0.0, policy=(1, 0)):
    x = matrix(rows, cols, dtype, 1, pad, offset=offset)
    x += far
    r = matrix(rows, cols, dtype, 2, pad, offset=offset) if residual else None
    g = vector(cols, 3) if gain else None
    b = vector(cols, 4) if shift else None
    h = matrix(rows, cols, dtype, 5, pad, offset=offset) if total else None
    y = matrix(rows, cols, out, 6, pad, offset=0 if out == "e4m3" else offset)
    s = vector(rows, 7) if out == "e4m3" else None
    mean, rstd = vector(rows, 8), vector(rows, 9)
    yr, hr, mr, rr, ey, em, er = layernorm64(x, r, g, b)
    errs = emu.call(al.alcop_layernorm, x, g, b, y, residual=r, total=h, scale=s, mean=mean, rstd=rstd, reads=some(x, r, g, b),
                    writes=some(h, y, s, mean, rstd), policy=policy)
    assert not errs, errs[:4]
    check(mean[None], mr[None], em[None], "mean")
    check(rstd[None], rr[None], (er * rr)[None], "rstd")
    if total:
        check(h, hr, ULP * hr.abs(), "total")
    if out == "e4m3":
        top = yr.abs().amax(dim=1, keepdim=True)
        check_e4m3(y, s, yr, float((ey / top).max()) + 4 * ULP, "y")
    else:
        check(y, yr, ey, "y")


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (2, 8), (5, 513), (3, 1024), (2, 1111), (1, 4096), (2, 2049)])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f16", "f32"), ("f32", "e4m3")])
def test_norms(rows, cols, dtype, out):
    run_norm(rows, cols, dtype, out, pad=3, offset=1)


@pytest.mark.parametrize("rows,cols", [(1, 64), (4, 100), (5, 128), (15, 129), (17, 256), (35, 250)])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("f16", "e4m3"), ("f32", "f32")])
def test_short_rows(rows, cols, dtype, out):
    run_norm(rows, cols, dtype, out)
    run_norm(rows, cols, dtype, out, pad=3, offset=1)
    x, g = matrix(rows, cols, dtype, 1), vector(cols, 2)
    r, b = matrix(rows, cols, dtype, 3), vector(cols, 4)
    y = torch.empty(rows, cols, dtype=DT[dtype])
    h = torch.empty_like(y)
    assert not emu.call(al.alcop_layernorm, x, g, b, y, residual=r, total=h, reads=[x, g, b, r], writes=[y, h])
    assert not emu.call(al.alcop_layernorm, x, g, b, r, residual=r, total=x, reads=[x, g, b, r], writes=[x, r])
    assert torch.equal(x, h) and torch.equal(r, y)


def test_norms_of_long_rows():
    run_norm(2, 9000, "bf16", "bf16")
    run_norm(1, 20001, "f16", "e4m3", pad=5)


@pytest.mark.parametrize("policy", emu.POLICIES)
def test_norms_under_every_timing(policy):
    run_norm(3, 2056, "bf16", "e4m3", policy=policy)


def test_parts_that_are_left_out():
    run_norm(4, 100, "f16", "f16", residual=False, gain=False, shift=False, total=False)
    run_norm(4, 100, "f16", "f16", residual=False, gain=True, shift=False)


def test_rows_far_from_zero():
    # a spread of 1 beside a mean of a thousand: a variance from sums of squares would have no digits left
    run_norm(3, 1000, "f32", "f32", residual=False, far=3000.0)
    run_norm(2, 4096, "f32", "f32", residual=False, far=3000.0)


def test_a_row_of_equal_numbers_is_its_shift():
    x = torch.full((2, 40), 3.25)
    b, y = vector(40, 1), torch.empty(2, 40)
    g = vector(40, 2)
    errs = emu.call(al.alcop_layernorm, x, g, b, y, reads=[x, g, b], writes=[y])
    assert not errs and torch.equal(y, b.expand(2, 40))


def test_infinities_and_nan_stay_in_their_row():
    x = matrix(4, 96, "f16", 1)
    x[1, 5] = float("inf")
    x[2, 7] = float("nan")
    y = torch.empty(4, 96, dtype=torch.float16)
    assert not emu.call(al.alcop_layernorm, x, None, None, y, reads=[x], writes=[y])
    assert torch.isfinite(y[[0, 3]]).all() and y[1:3].isnan().all()


def run_grad(rows, cols, dtype, dtotal=True, gain=True, dgain=True, dshift=True, pad=0, offset=0, in_place=False, policy=(1, 0)):
    dy = matrix(rows, cols, dtype, 1, pad, offset=offset)
    h = matrix(rows, cols, dtype, 2, pad, scale=2.0, offset=offset)
    dt = matrix(rows, cols, dtype, 3, pad, offset=offset) if dtotal else None
    g = vector(cols, 4) if gain else None
    mean, rstd = 0.1 * vector(rows, 5), vector(rows, 6).abs() + 0.1
    dx = (dt if dtotal else dy) if in_place else matrix(rows, cols, dtype, 7, pad, offset=offset)
    dg, ds = vector(cols, 8) if dgain else None, vector(cols, 9) if dshift else None
    ws = torch.empty(al.alcop_layernorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8)
    dxr, dgr, dsr, edx, edg, eds = layernorm_grad64(dy, h, g, mean, rstd, dt)
    errs = emu.call(al.alcop_layernorm_backward, dy, h, g, mean, rstd, dx, dgain=dg, dshift=ds, dtotal=dt, workspace=ws,
                    reads=some(dy, h, g, mean, rstd, dt), writes=some(dx, dg, ds, ws), policy=policy)
    assert not errs, errs[:4]
    check(dx, dxr, edx, "dx")
    if dgain:
        check(dg[None], dgr[None], edg[None], "dgain")
    if dshift:
        check(ds[None], dsr[None], eds[None], "dshift")


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (9, 8), (13, 513), (5, 1024), (3, 1111), (3, 4096), (4, 2049)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_gradients(rows, cols, dtype):
    run_grad(rows, cols, dtype, pad=3, offset=1)


@pytest.mark.parametrize("rows,cols", [(1, 64), (4, 100), (50, 128), (15, 129), (35, 256), (33, 250)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_gradients_of_short_rows(rows, cols, dtype):
    run_grad(rows, cols, dtype)
    run_grad(rows, cols, dtype, pad=3, offset=1, in_place=True)
    run_grad(rows, cols, dtype, dgain=False, dtotal=False)


def test_gradients_of_long_rows_and_many():
    run_grad(3, 9000, "bf16")
    run_grad(3, 17001, "f16", pad=1)
    run_grad(40, 72, "f32")


@pytest.mark.parametrize("policy", emu.POLICIES)
def test_gradients_under_every_timing(policy):
    run_grad(5, 2056, "bf16", policy=policy)
    run_grad(30, 72, "bf16", policy=policy)


def test_gradients_that_are_left_out_or_in_place():
    run_grad(20, 100, "f16", dtotal=False, gain=False, dgain=False, dshift=False)
    run_grad(20, 100, "f16", dgain=False)
    run_grad(20, 100, "f16", dshift=False, in_place=True)
    run_grad(20, 100, "bf16", dtotal=False, in_place=True)
