"""Layer norm of rows whose mean is a million times their spread and more, on the CPU model of the hardware (tests/emu): the variance keeps
its digits, and rows beside such a row keep their bits."""
import pytest
import torch

import paper_2210_16691_amd as al
from layers_util import ULP, check
from test_loss_confident import emulated

COLS = [40, 250, 1000, 1024, 2049, 4096, 20001]


def far64(x, eps):
    """(y, mean, rstd, bounds of their errors; rstd's is relative) of fp32 rows without a residual.

    A sum over a row takes no more than S = 100 steps: up to 64 numbers of a thread, six exchanges, sixteen waves, its mean.  m is within
    e1 = (S ULP + 2^-13) mean|h| of the mean and h - m exact, or rounded where the row is not far.  Its mean is off by e2 = S ULP (mean|d| + e1).
    Where e1^2 is above the variance the row is moved once more, to a point e2 away, and that mean is off by S ULP (mean|d| + e2); else
    e1 is at most about the spread.  The variance: S + 8 roundings of mean(d^2) = var + the square of the distance left, which counts twice."""
    h = x.cpu().double()
    S = 100
    mean = h.mean(dim=1, keepdim=True)
    d = h - mean
    size = d.abs().mean(dim=1, keepdim=True)
    var = d.square().mean(dim=1, keepdim=True)
    rstd = (var + eps).rsqrt()
    e1 = (S * ULP + 2.0 ** -13) * h.abs().mean(dim=1, keepdim=True)
    e2 = S * ULP * (size + e1)
    left = torch.minimum(e1, torch.maximum(1.5 * var.sqrt(), 2 * e2))
    em = S * ULP * (size + left) + 2 * ULP * mean.abs()
    ed = S * ULP * (size + left) + 2 * ULP * (d.abs() + left)
    er = (S + 8) * ULP * (var + 2 * left ** 2) / (var + eps) + (ed * d.abs()).mean(dim=1, keepdim=True) / (var + eps) + 6 * ULP
    y = d * rstd
    return y, mean[:, 0], rstd[:, 0], ed * rstd + y.abs() * (er + 3 * ULP), em[:, 0], er[:, 0]


def check_far(call, rows, cols, far, spread=1.0, dev="cpu", eps=1e-5):
    g = torch.Generator().manual_seed(cols)
    x = (torch.randn(rows, cols, generator=g) * spread + far * (1 + torch.rand(rows, 1, generator=g))).to(dev)
    y, mean, rstd = torch.zeros_like(x), torch.zeros(rows, device=dev), torch.zeros(rows, device=dev)
    call(al.alcop_layernorm, x, None, None, y, mean=mean, rstd=rstd, eps=eps)
    yr, mr, rr, ey, em, er = far64(x, eps)
    check(mean[None], mr[None], em[None], "mean")
    check(rstd[None], rr[None], (er * rr)[None], "rstd")
    check(y, yr, ey, "y")


def check_beside(call, dev="cpu"):
    # four rows to a wave: the second and the last of them far away
    g = torch.Generator().manual_seed(1)
    near = torch.randn(8, 72, generator=g).to(dev)
    mixed = near.clone()
    mixed[[1, 3, 7]] += 3e6
    out = [torch.zeros_like(near) for _ in range(2)]
    for x, y in zip((near, mixed), out):
        call(al.alcop_layernorm, x, None, None, y)
    assert torch.equal(out[0][[0, 2, 4, 5, 6]], out[1][[0, 2, 4, 5, 6]])


@pytest.mark.parametrize("cols", COLS)
def test_rows_a_million_spreads_from_zero(cols):
    for far in (1e4, 1e6, -4e6):
        check_far(emulated, 3, cols, far)


@pytest.mark.parametrize("cols", [72, 4096])
def test_rows_of_equal_numbers_far_from_zero(cols):
    check_far(emulated, 3, cols, 1e6, spread=0.0)


def test_rows_beside_a_far_one_keep_their_bits():
    check_beside(emulated)
