"""Plain forms of the linear layers, norms and 8-bit rows in 64 bits, and how far results may be off.

Half a step of a type, relative to the value: HALF.  A sum of n fp32 terms is off by at most (n + 4) 2^-24 times the
sum of the terms' magnitudes (n - 1 additions, a product, the scales' two, the bias)."""
import math

import torch

HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24, torch.float8_e4m3fn: 2.0 ** -4}
# below the smallest normal number the steps stay as they are: half of one
LEAST = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150, torch.float8_e4m3fn: 2.0 ** -10}
DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
ULP = 2.0 ** -24
TINY = 2.0 ** -126


def act64(z, act):
    if act == 1:
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == 2:
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    if act == 3:
        return z * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
    if act == 4:
        return z * torch.sigmoid(z)
    return z


def slope64(z, act):
    if act == 1:
        return (z > 0).to(z.dtype)
    if act == 2:
        return 0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == 3:
        c = 2.0 * math.sqrt(2.0 / math.pi)
        s = torch.sigmoid(c * (z + 0.044715 * z ** 3))
        return s + z * s * (1.0 - s) * c * (1.0 + 3.0 * 0.044715 * z * z)
    if act == 4:
        s = torch.sigmoid(z)
        return s + z * s * (1.0 - s)
    return torch.ones_like(z)


def act_error(z):
    """What the activation adds in fp32: 1 + erf and the sigmoid are within 4 units of 2^-24 (erf 1, exp2 and the
    reciprocal 1 each, the argument's roundings times its size, which decays against exp(-u)); times |z|, and the slope
    of at most 1.13 carries Z's own error on."""
    return 16 * ULP * z.abs()


def linear64(A, W, transB, alpha=1.0, bias=None, act=0, residual=None, sa=None, sw=None, as_they_are=False):
    """(C, Z, bound of Z's error, bound of C's error before the rounding).  as_they_are: sums of the 8-bit matrix
    instruction, which cuts off what lies below 2^-13 of the largest product among those it adds, from each of them and
    from what it adds up of them: 2^-12 of the largest product for each term."""
    a, w = A.cpu().double(), W.cpu().double()
    if transB:
        w = w.t()
    s = abs(alpha) * torch.ones(a.shape[0], w.shape[1], dtype=torch.float64)
    if sa is not None:
        s = s * sa.cpu().double()[:, None]
    if sw is not None:
        s = s * sw.cpu().double()
    z = a @ w * s * math.copysign(1.0, alpha)
    mag = a.abs() @ w.abs() * s
    if bias is not None:
        z = z + bias.cpu().double()
        mag = mag + bias.cpu().double().abs()
    ez = (a.shape[1] + 4) * ULP * mag
    if as_they_are:
        top = a.abs().amax(dim=1)[:, None] * w.abs().amax(dim=0)[None] * s
        ez = ez + 2.0 ** -12 * a.shape[1] * torch.minimum(top, mag)
    c, ec = act64(z, act), 1.13 * ez + (act_error(z) if act > 1 else 0)
    if residual is not None:
        c = c + residual.cpu().double()
        ec = ec + ULP * (c.abs() + residual.cpu().double().abs())
    return c, z, ez, ec


def check(got, ref, err, what=""):
    """got is ref rounded once, ref being known up to err."""
    g = got.detach().cpu().double()
    assert g.shape == ref.shape, what
    assert bool(torch.isfinite(g).all()), what + ": not finite"
    half, least = HALF[got.dtype], LEAST[got.dtype]
    bound = err + half * (ref.abs() + err) + least
    off = (g - ref).abs()
    worst = float((off / bound).max())
    assert worst <= 1.0, "%s: %.3f times the bound at %s" % (what, worst, divmod(int((off / bound).argmax()), g.shape[-1]))


def norm64(x, residual=None, gain=None, eps=1e-6):
    """(y, h, rstd), all in 64 bits."""
    h = x.cpu().double()
    if residual is not None:
        h = h + residual.cpu().double()
    rstd = (h.square().mean(dim=1) + eps).rsqrt()
    y = h * rstd[:, None]
    if gain is not None:
        y = y * gain.cpu().double()
    return y, h, rstd


def check_e4m3(q, scale, y, err, what=""):
    """q and scale are rows y (known up to the relative error err of their values) in 8 bits.  y / scale is off by
    err and by the scale's error, then rounded; below 2^-6 the step of e4m3 is 2^-9."""
    s = (y.abs().amax(dim=1) / 448.0).clamp_min(TINY)
    es = float((((scale.cpu().double() - s).abs()) / s).max())
    assert es <= err + 2 * ULP, "%s: scale off by %.3g" % (what, es)
    check(q, y / s[:, None], (2 * err + 4 * ULP) * (y / s[:, None]).abs(), what)


def norm_grad64(dy, total, gain, rstd, dtotal=None):
    """(dx, dgain, bound of dx's error, bound of dgain's)."""
    d, h, r = dy.cpu().double(), total.cpu().double(), rstd.cpu().double()[:, None]
    g = torch.ones(d.shape[1], dtype=torch.float64) if gain is None else gain.cpu().double()
    n = d.shape[1]
    xh, t = h * r, d * g
    mean = (t * xh).mean(dim=1, keepdim=True)
    dx = r * (t - xh * mean)
    size = r * (t.abs() + xh.abs() * (t * xh).abs().mean(dim=1, keepdim=True))
    edx = (n + 8) * ULP * r * xh.abs() * (t * xh).abs().mean(dim=1, keepdim=True) + 8 * ULP * size
    if dtotal is not None:
        dx = dx + dtotal.cpu().double()
        edx = edx + ULP * (dx.abs() + dtotal.cpu().double().abs())
    return dx, (d * xh).sum(dim=0), edx, (d.shape[0] + 4) * ULP * (d * xh).abs().sum(dim=0)
