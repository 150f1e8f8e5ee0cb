"""Gradients of the cross entropy in fp16 for losses that weigh next to nothing or enormously, on the CPU model of the hardware (tests/emu):
the power of two that G carries reaches all of fp32."""
import pytest
import torch

import paper_2210_16691_amd as al
from layers_util import check
from more_util import loss_grad64
from test_loss_confident import emulated


def check_scale(call, size, rows=40, vocab=300, K=40, dev="cpu"):
    g = torch.Generator().manual_seed(2)
    X, W = (torch.randn(n, K, generator=g).half() for n in (rows, vocab))
    W = (W.float() * K ** -0.5).half()
    y = torch.randint(0, vocab, (rows,), generator=g)
    d = torch.randn(rows, generator=g) * size
    lse = torch.logsumexp(X.double() @ W.double().t(), dim=1).float()
    rx, rw, ex, ew = loss_grad64(X, W, y, lse, d)
    dX, dW = torch.zeros(rows, K, device=dev), torch.zeros(vocab, K, device=dev)
    ws = torch.empty(al.alcop_linear_cross_entropy_backward_workspace_bytes(rows, vocab, K), dtype=torch.uint8, device=dev)
    call(al.alcop_linear_cross_entropy_backward, X.to(dev), W.to(dev), y.to(dev), lse.to(dev), ws, dX=dX, dW=dW, dloss=d.to(dev))
    check(dX, rx, ex, "dX")
    check(dW, rw, ew, "dW")


@pytest.mark.parametrize("size", [1e-33, 1e-30, 1.0, 1e30, 2e36])
def test_losses_of_every_weight(size):
    check_scale(emulated, size)
