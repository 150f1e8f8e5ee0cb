"""The cross entropy's gradients on the GPU where the vocabulary is long: pieces of several slices, vectors that span more than 2 GiB."""
import pytest
import torch

import paper_2210_16691_amd as al
from gpu_util import DEV
from layers_util import ULP
from test_gpu_z16_loss import run_gradients
from test_gpu_z17_block import big

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("out", [None, "f32"])
def test_several_pieces_of_several_slices(dtype, out, monkeypatch):
    monkeypatch.setenv("ALCOP_LOSS_PIECE", "8192")
    run_gradients(200, 17000, 136, dtype, out=out, pad=8)         # three pieces of two slices
    monkeypatch.setenv("ALCOP_LOSS_PIECE", "4096")
    run_gradients(33, 34700, 40, dtype, out=out)                  # eight of two slices and one of one


@pytest.mark.parametrize("out", [None, "f32"])
def test_one_piece_of_several_slices(out):
    run_gradients(33, 8200, 264, "bf16", out=out, pad=8)


@pytest.mark.parametrize("rows,vocab,K", [(40, 140000, 16384), (600, 70000, 16384), (1, 262144, 5376)])
def test_vectors_that_span_more_than_2_gib(rows, vocab, K):
    """(The first: eight slices of a piece; the second: one slice of a piece, which what a slice spans makes narrower; the third: a token.)"""
    big()
    # z is exact: sums of up to 2^14 products of -1, 0, 1 with 64ths; W has a mean, so that a slice that is lost or added twice shows in dX
    g = torch.Generator(device=DEV).manual_seed(5)
    alpha = 1.0 / 32
    X = torch.randint(-1, 2, (rows, K), generator=g, device=DEV).to(torch.bfloat16)
    W = torch.empty(vocab, K, dtype=torch.bfloat16, device=DEV)
    for w in W.split(5000):
        w.copy_(torch.randint(0, 65, w.shape, generator=g, device=DEV, dtype=torch.int16).to(torch.bfloat16) / 64)
    y = torch.randint(0, vocab, (rows,), device=DEV)
    y[:1] = vocab - 1
    # in 64 bits on the GPU, a part of the vocabulary at a time
    z = alpha * torch.cat([X.double() @ w.double().t() for w in W.split(5000)], dim=1)
    lse = torch.logsumexp(z, dim=1).float()
    dX, dW = torch.empty_like(X), torch.empty_like(W)
    ws = torch.empty(al.alcop_linear_cross_entropy_backward_workspace_bytes(rows, vocab, K), dtype=torch.uint8, device=DEV)
    al.alcop_linear_cross_entropy_backward(X, W, y, lse, ws, dX=dX, dW=dW, alpha=alpha)
    torch.cuda.synchronize()
    # G = p - one(label), rounded by 2^-8 of itself; p's exponent is off by the roundings of alpha log2(e), of lse log2(e) and of itself,
    # exp2 and p - 1 by two more: e of p, which is |G|, at the label |G| + 1.  dX: vocab + 8 roundings of a sum and one of 2^-8; dW likewise
    e = 4 * ULP * float(lse.abs().max() + z.abs().max()) + 6 * ULP
    G = torch.exp(z - lse.double()[:, None])
    G.scatter_add_(1, y[:, None], -torch.ones(rows, 1, dtype=torch.float64, device=DEV))
    del z
    want, size = torch.zeros(rows, K, dtype=torch.float64, device=DEV), torch.zeros(rows, K, dtype=torch.float64, device=DEV)
    for at in range(0, vocab, 5000):
        part, w = G[:, at:at + 5000], W[at:at + 5000].double()
        want += alpha * (part @ w)
        size += alpha * (part.abs() @ w)
    bound = (2.0 ** -8 + (vocab + 8) * ULP) * size + 2 * e * (size + alpha * W[y].double()) + 2.0 ** -8 * want.abs()
    assert bool(((dX.double() - want).abs() <= bound).all())
    for at in (0, 5120, 32511, 32512, 65535, 65536, vocab - 1, int(y[-1])):
        at = min(at, vocab - 1)
        want, size = alpha * (G[:, at] @ X.double()), alpha * (G[:, at].abs() @ X.double().abs())
        hits = alpha * ((y == at).double() @ X.double().abs())
        assert bool(((dW[at].double() - want).abs() <= (2.0 ** -8 + (rows + 8) * ULP) * size + 2 * e * (size + hits) + 2.0 ** -8 * want.abs()).all())
