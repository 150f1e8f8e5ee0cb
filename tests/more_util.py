"""Plain forms of layer norm, products grouped by expert and cross entropy in 64 bits, and how far results may be off
(half a step of a type and of a sum's error: layers_util)."""
import torch

from layers_util import ULP, act64, act_error, slope64


def layernorm64(x, residual=None, gain=None, shift=None, eps=1e-5):
    """(y, h, mean, rstd, bound of y's error before the rounding, of the mean's, of rstd's relative one).

    The mean: the point m is within e = (n + 2) ULP mean|h| + 2^-13 mean|h| of it (a sum, and half of a step of 2^-12), and
    mean(h - m) is off by (n + 2) ULP of the mean of |h - m|, itself at most mean|h - mean| + e: E = (n + 4) ULP (mean|d| + e) + 2 ULP
    |mean|.  h is rounded once on the way in where a residual is added.  The variance: n + 8 roundings of mean(d^2) = var + e^2 at most."""
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
    first = ((n + 2) * ULP + 2.0 ** -13) * h.abs().mean(dim=1, keepdim=True)
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


def grouped64(A, W, sizes, first, transB, alpha=1.0, bias=None, act=0, sa=None, sw=None, as_they_are=False):
    """(C, Z, bound of Z's error, of C's before the rounding) of every group's rows, which start at `first`; the rows of no
    group are NaN.  as_they_are: as for layers_util.linear64."""
    from layers_util import linear64
    rows, N = A.shape[0], W.shape[1] if transB else W.shape[2]
    out = [torch.full((rows, N), float("nan"), dtype=torch.float64) for _ in range(4)]
    at = first
    for g, n in enumerate(sizes):
        if n:
            part = slice(at, at + n)
            ref = linear64(A[part], W[g], transB, alpha, None if bias is None else bias[g], act, None,
                           None if sa is None else sa[part], None if sw is None else sw[g], as_they_are)
            for o, r in zip(out, ref):
                o[part] = r
        at += n
    return out


def grouped_grad64(dC, A, W, sizes, first, transB, pre=None, act=0, alpha=1.0):
    """(dA, dW, dbias, bounds of their errors before the rounding); dA of rows of no group is NaN.  dZ is rounded to the operands'
    type in front of the two products: half a step of each of their terms, beside a sum's error and the slope's."""
    from layers_util import HALF, LEAST
    half, least = HALF[dC.dtype], LEAST[dC.dtype]
    w = W.cpu().double()
    w = w.transpose(1, 2) if transB else w                     # groups x K x N
    G, K, N = w.shape
    rows = A.shape[0]
    dA = torch.full((rows, K), float("nan"), dtype=torch.float64)
    edA = dA.clone()
    dW, db = torch.zeros(G, K, N, dtype=torch.float64), torch.zeros(G, N, dtype=torch.float64)
    edW, edb = torch.zeros_like(dW), torch.zeros_like(db)
    at = first
    for g, n in enumerate(sizes):
        if n:
            part = slice(at, at + n)
            z, ez = dC[part].cpu().double(), 0.0
            if act:
                p = pre[part].cpu().double()
                ez = 16 * ULP * z.abs() * (1 + p.abs()) + ULP * z.abs()
                z = z * slope64(p, act)
            a = A[part].cpu().double()
            off = ez + (half * z.abs() + least if act else 0)      # dC itself is an operand where there is no activation
            dA[part] = alpha * (z @ w[g].t())
            edA[part] = abs(alpha) * (off @ w[g].t().abs() if act else 0) + (N + 4) * ULP * abs(alpha) * (z.abs() @ w[g].t().abs())
            dW[g] = alpha * (a.t() @ z)
            edW[g] = abs(alpha) * (a.t().abs() @ off if act else 0) + (n + 4) * ULP * abs(alpha) * (a.t().abs() @ z.abs())
            db[g] = z.sum(dim=0)
            edb[g] = (ez.sum(dim=0) if act else 0) + (n + 8) * ULP * z.abs().sum(dim=0)
        at += n
    if transB:
        dW, edW = dW.transpose(1, 2), edW.transpose(1, 2)
    return dA, dW, db, edA, edW, edb


def loss64(X, W, labels, alpha=1.0):
    """(loss, lse, bounds of their errors before the rounding).

    z is off by ez, a product's sum.  A term of sum(exp(z - shift)) has its exponent rounded (2^-24 of |z - shift|, which the term's own
    size outweighs: below 2 ULP), exp2's error and, on its way through a lane (64 terms), two lanes, four waves, a run of strips and 32
    runs, an addition and where shifts differ a product with an exp2 each: 4 ULP a step."""
    x, w = X.cpu().double(), W.cpu().double()
    z = alpha * (x @ w.t())
    ez = (x.shape[1] + 4) * ULP * alpha * (x.abs() @ w.abs().t())
    V = w.shape[0]
    lse = torch.logsumexp(z, dim=1)
    p = torch.exp(z - lse[:, None])
    steps = 64 + 1 + 4 + V / (64 * 32) + 32
    elses = (p * ez).sum(dim=1) + (4 * steps + 8) * ULP + 4 * ULP * (lse.abs() + z.abs().amax(dim=1))
    y = labels.cpu()
    there = (y >= 0) & (y < V)
    at = torch.where(there, y, torch.zeros_like(y))[:, None]
    loss = torch.where(there, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse))
    eloss = torch.where(there, elses + ez.gather(1, at)[:, 0] + 2 * ULP * (lse.abs() + z.gather(1, at)[:, 0].abs()), torch.zeros_like(lse))
    return loss, lse, eloss, elses


def loss_grad64(X, W, labels, lse, dloss=None, alpha=1.0):
    """(dX, dW, bounds of their errors before the rounding): G is rounded to the operands' type (fp16: in steps of 2^-25 of
    S |dloss| at most 2^15, S at least 2^14 over the largest |dloss|), beside a sum's error."""
    from layers_util import HALF, LEAST
    x, w = X.cpu().double(), W.cpu().double()
    z = alpha * (x @ w.t())
    ez = (x.shape[1] + 4) * ULP * alpha * (x.abs() @ w.abs().t())
    l = lse.cpu().double()[:, None]
    p = torch.exp(z - l)
    ep = p * (ez + 2 * ULP * (l.abs() + z.abs()) + 6 * ULP)
    y = labels.cpu()
    there = (y >= 0) & (y < w.shape[0])
    d = torch.ones(x.shape[0], dtype=torch.float64) if dloss is None else dloss.cpu().double()
    d = torch.where(there, d, torch.zeros_like(d))[:, None]
    one = torch.zeros_like(p)
    one[there, y[there]] = 1.0
    g = (p - one) * d
    top = float((torch.ones(1) if dloss is None else dloss.cpu().abs()).max())
    eg = (ep + 2 * ULP) * d.abs()
    eg = eg + HALF[X.dtype] * (g.abs() + eg) + LEAST[X.dtype] * (top * 2.0 ** -14 if X.dtype == torch.float16 else 1.0) * (d != 0)
    V, T = w.shape[0], x.shape[0]
    dX, dW = alpha * (g @ w), alpha * (g.t() @ x)
    return (dX, dW, alpha * (eg @ w.abs() + (V + 8) * ULP * (g.abs() @ w.abs())),
            alpha * (eg.t() @ x.abs() + (T + 8) * ULP * (g.abs().t() @ x.abs())))
