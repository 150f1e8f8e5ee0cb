"""Plain forms of layer norm, products grouped by expert and cross entropy in 64 bits, and how far results may be off
(half a step of a type and of a sum's error: layers_util)."""
import torch

from layers_util import ULP, act64, act_error, slope64


def layernorm64(x, residual=None, gain=None, shift=None, eps=1e-5):
    """(y, h, mean, rstd, bound of y's error before the rounding, of the mean's, of rstd's relative one).

    The mean: m = sum / n is off by e <= (n + 2) ULP mean|h|, and mean(h - m) by (n + 2) ULP of the mean of |h - m|, itself at most
    mean|h - mean| + e; what is left of e is its product with that, so E = (n + 4) ULP (mean|d| + e) + 2 ULP |mean|.
    h is rounded once on the way in where a residual is added.  The variance: n + 6 roundings, halved by the root, and E^2."""
    h = x.cpu().double()
    eh = 0.0
    if residual is not None:
        r = residual.cpu().double()
        h = h + r
        eh = ULP * h.abs()
    n = h.shape[1]
    mean = h.mean(dim=1, keepdim=True)
    d = h - mean
    var = d.square().mean(dim=1, keepdim=True)
    rstd = (var + eps).rsqrt()
    first = (n + 2) * ULP * h.abs().mean(dim=1, keepdim=True)
    em = (n + 4) * ULP * (d.abs().mean(dim=1, keepdim=True) + first) + 2 * ULP * mean.abs()
    if residual is not None:
        em = em + eh.mean(dim=1, keepdim=True)
    # h - m and the correction are rounded relative to themselves, the mean's own rounding is not part of y
    ed = em + 2 * ULP * (d.abs() + first) + (eh if residual is not None else 0)
    spread = ((var + first ** 2) / (var + eps)).clamp_min(1.0)
    er = (n + 8) * ULP * spread + (ed * d.abs()).mean(dim=1, keepdim=True) / (var + eps) + 6 * ULP
    y = d * rstd
    ey = (ed * rstd + y.abs() * (er + 3 * ULP))
    if gain is not None:
        g = gain.cpu().double()
        y, ey = y * g, ey * g.abs()
    if shift is not None:
        y = y + shift.cpu().double()
    return y, h, mean[:, 0], rstd[:, 0], ey + ULP * y.abs(), em[:, 0], er[:, 0]


def layernorm_grad64(dy, total, gain, mean, rstd, dtotal=None):
    """(dx, dgain, dshift, bounds of their errors)."""
    d, h = dy.cpu().double(), total.cpu().double()
    m, r = mean.cpu().double()[:, None], rstd.cpu().double()[:, None]
    g = torch.ones(d.shape[1], dtype=torch.float64) if gain is None else gain.cpu().double()
    n = d.shape[1]
    xh, t = (h - m) * r, d * g
    mt, mx = t.mean(dim=1, keepdim=True), (t * xh).mean(dim=1, keepdim=True)
    at, ax = t.abs().mean(dim=1, keepdim=True), (t * xh).abs().mean(dim=1, keepdim=True)
    dx = r * (t - mt - xh * mx)
    # two sums of n + 4 roundings each, xh of two, then the terms' own
    edx = r * ((n + 8) * ULP * (at + xh.abs() * ax) + 8 * ULP * (t.abs() + at + xh.abs() * ax))
    if dtotal is not None:
        dx = dx + dtotal.cpu().double()
        edx = edx + ULP * (dx.abs() + dtotal.cpu().double().abs())
    rows = d.shape[0]
    return (dx, (d * xh).sum(dim=0), d.sum(dim=0), edx, (rows + 8) * ULP * (d * xh).abs().sum(dim=0),
            (rows + 4) * ULP * d.abs().sum(dim=0))
