"""The loss of rows that are predicted well, on the CPU model of the hardware (tests/emu): small beside lse, of which it must not be the
rounded rest."""
import pytest
import torch

import emu_util as emu
import paper_2210_16691_amd as al
from layers_util import ULP

ROWS, VOCAB, K = 60, 300, 64


def confident(dtype, behind=None, alpha=1.0):
    """(X, W, labels, loss in 64 bits).  Row r has the logit L = 15 .. 60 at column r, -32 elsewhere, with `behind` L - behind at column
    100 + r too; 16ths, which the types and the sums hold exactly (times 1 / alpha, a power of two)."""
    L = torch.round((15 + 45 * torch.arange(ROWS) / (ROWS - 1)) * 16) / 16
    X, W = torch.zeros(ROWS, K), torch.zeros(VOCAB, K)
    # z = X[r, r] W[v, r] - 32 with X[r, r] = 1: W holds what the column needs, in two parts of few bits each
    for r in range(ROWS):
        X[r, r] = 1.0
        W[r, r] = torch.floor(L[r] + 32)
        if behind is not None:
            W[100 + r, r] = torch.floor(L[r] + 32) - behind
    X[:, 61], W[:ROWS, 61] = 1.0, L - torch.floor(L)
    if behind is not None:
        W[100:100 + ROWS, 61] = L - torch.floor(L)
    X[:, 60], W[:, 60] = 1.0 / alpha, -32.0
    X[:, :60], X[:, 61] = X[:, :60] / alpha, X[:, 61] / alpha
    X, W = X.to(dtype), W.to(dtype)
    z = alpha * (X.double() @ W.double().t())
    # (other rows' fractions move a logit of -32 by less than 1)
    y = torch.arange(ROWS)
    assert torch.equal(z[y, y], L.double()) and z.amax() <= 63
    return X, W, y, z


def loss_of(call, X, W, y, alpha, dev="cpu"):
    loss, lse = torch.zeros(ROWS, device=dev), torch.zeros(ROWS, device=dev)
    ws = torch.empty(al.alcop_linear_cross_entropy_workspace_bytes(ROWS, VOCAB, K), dtype=torch.uint8, device=dev)
    call(al.alcop_linear_cross_entropy, X, W, y, loss, lse, ws, alpha=alpha)
    return loss.cpu().double()


def check_confident(call, dtype, behind, alpha, dev="cpu"):
    X, W, y, z = confident(dtype, behind, alpha)
    if behind is not None and behind < 0:
        y = y + 100                                # the larger one of the two
        behind = -behind
    ref = -torch.log_softmax(z, dim=1)[torch.arange(ROWS), y]
    got = loss_of(call, X.to(dev), W.to(dev), y.to(dev), alpha, dev)
    # ln 2 (log2(sum) - d): two terms of the sum count, whose exponents are at most 5 apart and off by 4 ULP of that times p < 0.05 (1 ULP),
    # exp2 by 2 ULP, their sum by 1, log2 by 2 of a number below 1; d by ULP of itself, the difference and its product with ln 2 by 3 of
    # the loss.  The logits below -31 are less than 2^-66 of the largest
    bound = (8 + 8 * ref) * ULP
    assert bool(((got - ref).abs() <= bound).all()), float((got - ref).abs().max())
    assert bool((got >= 0).all())


def emulated(fn, *args, **kw):
    ts = [t for t in list(args) + list(kw.values()) if isinstance(t, torch.Tensor)]
    errs = emu.call(fn, *args, reads=ts, writes=ts, **kw)
    assert not errs, errs[:3]


@pytest.mark.parametrize("behind", [None, 3, -3])
@pytest.mark.parametrize("dtype,alpha", [(torch.float16, 1.0), (torch.bfloat16, 1.0), (torch.float16, 0.25)])
def test_the_loss_of_confident_rows(dtype, alpha, behind, monkeypatch):
    check_confident(emulated, dtype, behind, alpha)
