"""An infinite logit beside large finite ones in other strips of the vocabulary, on the CPU model of the hardware (tests/emu): the loss and
lse are infinite, whichever strip comes first."""
import pytest
import torch

import paper_2210_16691_amd as al
from test_loss_confident import emulated
from test_loss_emulated import KERNELS

INF = float("inf")


def check_infinite(call, dtype, dev="cpu"):
    rows, vocab, K = 6, 700, 8
    for at in (9, 350, 699):
        X, W = torch.zeros(rows, K, dtype=dtype), torch.zeros(vocab, K, dtype=dtype)
        X[:, 0] = 1.0
        W[:, 0], W[3, 0], W[340, 0], W[600, 0] = -200.0, 300.0, 300.0, 400.0
        W[100:200, 0] = -INF
        W[at, 0] = INF
        y = torch.tensor([3, 600, 340, 150, at, -1])
        loss, lse = torch.zeros(rows, device=dev), torch.zeros(rows, device=dev)
        ws = torch.empty(al.alcop_linear_cross_entropy_workspace_bytes(rows, vocab, K), dtype=torch.uint8, device=dev)
        call(al.alcop_linear_cross_entropy, X.to(dev), W.to(dev), y.to(dev), loss, lse, ws)
        assert (lse == INF).all(), lse
        assert (loss[:4] == INF).all() and loss[4].isnan() and loss[5] == 0.0, loss


@pytest.mark.parametrize("kernel", range(KERNELS))
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_an_infinite_logit_beside_large_ones(dtype, kernel, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    check_infinite(emulated, dtype)
