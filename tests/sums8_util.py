"""How far a layer on e4m3 operands may be off where the 8-bit matrix instruction sums it.

Of each eight products k = 8g .. 8g+7 every one is cut off, towards 0, at 2^-13 of the largest 2^(sum of the operands' exponents)
among them, numbers below 2^-6 counting as 2^-6.  The largest product itself has eight bits and is not cut, so the eight lose at most
7 * 2^-13 top_g, with top_g = max |a| |w| (each at least 2^-6, products of 0 left out) and never less than that power of two.
Truncation errors of random numbers have the products' random signs and at most a step's length: their mean square is at most
a third of its square each."""
import math

import torch

from layers_util import HALF, ULP, act64, check, linear64

CUT = 2.0 ** -13


def tops(A, W):
    """(sum_g top_g, sum_g top_g^2) for every element of A.W^T, in fp32: each is one product of e4m3 numbers, exact."""
    a, w = A.float(), W.float()
    K = a.shape[1]
    one, two = (torch.zeros(a.shape[0], w.shape[0], device=a.device) for _ in range(2))
    fa, fw = (torch.where(t == 0, t, t.abs().clamp_min(2.0 ** -6)) for t in (a, w))
    for g in range(0, K, 8):
        top = torch.zeros_like(one)
        for k in range(g, min(g + 8, K)):
            top = torch.maximum(top, fa[:, k, None] * fw[None, :, k])
        one += top
        two += top * top
    return one.cpu().double(), two.cpu().double()


def check_sums(C, pre, A, W, alpha=1.0, bias=None, act=0, residual=None, sa=None, sw=None, random=True, what=""):
    """C and pre within the bound element by element and, of random numbers, the root of the mean square too: 1.1 times that of
    the rounding (uniform within half a step: its square a third) and of the cuts together."""
    ref, zref, ez, ec = linear64(A, W, True, alpha, bias, act, residual, sa, sw)
    s = abs(alpha) * torch.ones_like(ref)
    if sa is not None:
        s = s * sa.cpu().double()[:, None]
    if sw is not None:
        s = s * sw.cpu().double()
    one, two = tops(A, W)
    most, square = 7 * CUT * one * s, 7 / 3 * CUT ** 2 * two * s * s
    # the eights' sums and the accumulator are added as fp32, towards 0 at worst: a step each instead of half of one
    for got, exact, err, slope, name in ((C, ref, ec + ez, 1.13, "C "), (pre, zref, 2 * ez, 1.0, "pre ")):
        if got is None:
            continue
        check(got, exact, err + slope * most, name + what)
        if random:
            off = (got.cpu().double() - exact).square().mean().sqrt()
            allow = ((HALF[got.dtype] * exact).square() / 3 + slope ** 2 * square).mean().sqrt()
            assert float(off) <= 1.1 * float(allow), "%s%s: root mean square %.3g, %.3g expected" % (name, what, off, allow)


def quantized_pair(M, N, K, seed, device="cpu"):
    """e4m3 operands and scales as rows of normal numbers have them."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for rows, scale in ((M, 1.0), (N, K ** -0.5)):
        v = torch.randn(rows, K, generator=g) * scale
        s = v.abs().amax(dim=1) / 448.0
        out += [(v / s[:, None]).to(torch.float8_e4m3fn).to(device), s.to(device)]
    return out[0], out[2], out[1], out[3]


def cancelling(M, N, K, device="cpu"):
    """Operands whose sums the 8-bit instruction gets wrong: in every eight 2^14, -2^14 and six of 2^-1, each below 2^-13 of the
    largest: Z = 6 K / 16 exactly in fp32, 0 with the cuts."""
    row = torch.tensor([128.0, -128.0, 2.0 ** -8, 2.0 ** -8, 2.0 ** -8, 2.0 ** -8, 2.0 ** -8, 2.0 ** -8]).repeat(K // 8)
    return (row.repeat(M, 1).to(torch.float8_e4m3fn).to(device),
            torch.full((N, K), 128.0).to(torch.float8_e4m3fn).to(device), 6 * (K // 8) * 0.5)
