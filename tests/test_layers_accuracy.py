"""Activations and their slopes on the CPU model: how near they are relative to their own size, far from 0 too.

A layer of zeros has Z = bias, any fp32 numbers; the bias's gradient of a single row with dC = 1 is the slope, in fp32.  u = 2^-24."""
import math

import pytest
import torch

import emu_util as emu
import paper_2210_16691_amd as al
from layers_util import act64, slope64

U = 2.0 ** -24


def relative(z, act):
    """Bound of the activation's error relative to its value, z in 64 bits.

    GELU (erf): the fit 13 u; t = 1 / (1 + p z) 3 u (sum 1, reciprocal 2) times the tail's sensitivity to t, at most 2.3; seven steps
    of the polynomial, whose terms' magnitudes are at most 1.8 times their sum, 12 u; three products and exp2 5 u: below 40.  The exponent
    z^2 / 2 has two roundings and the constant's: 1.5 z^2 / 2 u and half of that again in reserve.
    z sigmoid(v), v = z (a + b z^2) or z: the exponent's roundings and constants 8 |v| u; exp2, a sum, the reciprocal, the product 8 u."""
    if act == 2:
        return (40 + 1.5 * z * z) * U
    v = z if act == 4 else 2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)
    return (8 + 8 * v.abs()) * U


def exact(z, act):
    # the tails of the sigmoid without 1 + exp, those of the normal distribution from the scaled function
    if act == 2:
        tail = 0.5 * torch.special.erfcx(z.abs() / math.sqrt(2.0)) * torch.exp(-0.5 * z * z)
        return torch.where(z < 0, z * tail, z - z * tail)
    return act64(z, act)


def points(act):
    # as far left as the results are normal fp32 numbers
    left = {2: -12.5, 3: -9.0, 4: -80.0}[act]
    return torch.cat([torch.linspace(left, 10.0, 1531), torch.tensor([-1e-3, 1e-3, -1e-30, 1e-30, 50.0])])


def check_activation(call, act, dev="cpu"):
    z = points(act)
    A, W = torch.zeros(1, 8, dtype=torch.float16, device=dev), torch.zeros(len(z), 8, dtype=torch.float16, device=dev)
    C, b = torch.empty(1, len(z), device=dev), z.to(dev)
    call(al.alcop_linear, A, W, C, reads=[A, W, b], writes=[C], transB=True, bias=b, act=act)
    ref = exact(z.double(), act)
    off = (C[0].cpu().double() - ref).abs() / (relative(z.double(), act) * ref.abs())
    assert float(off.max()) <= 1.0, (float(off.max()), float(z[off.argmax()]))


def check_slope(call, act, dev="cpu"):
    left = {2: -12.5, 3: -8.0, 4: -80.0}[act]
    z = torch.linspace(left, 10.0, 1528).to(torch.bfloat16)[None]
    dC, pre = torch.ones_like(z).to(dev), z.to(dev)
    A, W = torch.zeros(1, 8, dtype=torch.bfloat16, device=dev), torch.zeros(z.shape[1], 8, dtype=torch.bfloat16, device=dev)
    db = torch.empty(z.shape[1], device=dev)
    ws = torch.empty(al.alcop_linear_backward_workspace_bytes(1, z.shape[1], 8), dtype=torch.uint8, device=dev)
    call(al.alcop_linear_backward, dC, A, W, reads=[dC, A, W, pre], writes=[db, ws], dbias=db, pre=pre, act=act, transB=True, workspace=ws)
    v = z[0].double()
    ref = slope64(v, act)
    if act == 2:                  # the two terms' sizes
        size = 0.5 * torch.special.erfcx(v.abs() / math.sqrt(2.0)) * torch.exp(-0.5 * v * v)
        size = torch.where(v < 0, size, 1 - size) + v.abs() * torch.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)
        ref = torch.where(v < 0, 0.5 * torch.special.erfcx(v.abs() / math.sqrt(2.0)) * torch.exp(-0.5 * v * v)
                          + v * torch.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi), ref)
    else:                         # s + z s (1 - s) v': 1 - s is off by a unit of 1, s as above
        c = 2.0 * math.sqrt(2.0 / math.pi)
        s = torch.sigmoid(v if act == 4 else c * (v + 0.044715 * v ** 3))
        size = s * (1 + v.abs() * (1.0 if act == 4 else c * (1 + 0.134145 * v * v)))
    off = (db.cpu().double() - ref).abs() / ((relative(v, act) + 16 * U) * size)
    assert float(off.max()) <= 1.0, (float(off.max()), float(v[off.argmax()]))


def on_the_model(fn, *args, **kw):
    assert not emu.call(fn, *args, **kw)


@pytest.mark.parametrize("act", [2, 3, 4])
def test_activations_are_near_relative_to_their_value(act):
    check_activation(on_the_model, act)


@pytest.mark.parametrize("act", [2, 3, 4])
def test_slopes_are_near_relative_to_their_terms(act):
    check_slope(on_the_model, act)
