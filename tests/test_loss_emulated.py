"""The cross entropy of a vocabulary's product and its gradients on the CPU model of the hardware (tests/emu): bounds of every access,
waits and barriers, results against the plain forms in 64 bits."""
import pytest
import torch

import emu_util as emu
import paper_2210_16691_amd as al
from layers_util import check
from more_util import loss64, loss_grad64
from test_layers_emulated import matrix, some, vector

KERNELS = 5             # of each step (ALCOP_LOSS_KERNELS)


def labels_of(rows, vocab, seed, ignored=True):
    y = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(seed))
    if ignored and rows > 3:
        y[1], y[2], y[3] = -100, vocab, 2 ** 32
    return y


def run_loss(rows, vocab, K, dtype, alpha=1.0, pad=0, policy=(1, 0), lse=True, scale=2.0):
    X, W = matrix(rows, K, dtype, 1, pad), matrix(vocab, K, dtype, 2, pad, scale=scale * K ** -0.5)
    y = labels_of(rows, vocab, 3)
    loss, l = vector(rows, 4), vector(rows, 5) if lse else None
    with emu._swapped():
        ws = torch.empty(al.alcop_linear_cross_entropy_workspace_bytes(rows, vocab, K), dtype=torch.uint8)
    ref, lref, e, el = loss64(X, W, y, alpha)
    errs = emu.call(al.alcop_linear_cross_entropy, X, W, y, loss, l, ws, alpha=alpha, reads=[X, W, y], writes=some(loss, l, ws), policy=policy)
    assert not errs, errs[:4]
    check(loss[None], ref[None], e[None], "loss")
    if lse:
        check(l[None], lref[None], el[None], "lse")


@pytest.mark.parametrize("kernel", range(KERNELS))
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_every_kernel(kernel, dtype, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    run_loss(70, 300, 72, dtype, pad=8, policy=emu.POLICIES[kernel % 4])
    run_loss(5, 131, 16, dtype, alpha=0.25)


def test_a_vocabulary_of_one_and_a_single_row():
    run_loss(1, 1, 8, "f16")
    run_loss(1, 65, 8, "f16", lse=False)
    run_loss(33, 2, 16, "bf16", alpha=3.0)


def test_many_strips():
    run_loss(3, 64 * 70 + 5, 8, "bf16")


def test_logits_far_apart():
    # one logit of some hundreds: the others vanish beside it
    run_loss(20, 200, 64, "f16", scale=60.0)


def test_infinite_and_masked_logits():
    rows, vocab, K = 4, 300, 8
    X, W = torch.zeros(rows, K, dtype=torch.float16), torch.zeros(vocab, K, dtype=torch.float16)
    X[:, 0], X[:, 1] = 1.0, torch.tensor([0.0, 1.0, 0.0, 1.0], dtype=torch.float16)
    W[:, 0] = torch.randn(vocab, generator=torch.Generator().manual_seed(1)) - 300.0
    y = torch.tensor([5, 6, 7, 8])
    W[64:192, 0] = -float("inf")          # columns that are masked out, a whole tile among them
    z = W[:, 0].double()                  # rows 0 and 2 with x = (1, 0): 0 times W's zeros adds nothing
    lse = torch.logsumexp(z, 0)
    loss, l = vector(rows, 4), vector(rows, 5)
    ws = torch.empty(al.alcop_linear_cross_entropy_workspace_bytes(rows, vocab, K), dtype=torch.uint8)
    errs = emu.call(al.alcop_linear_cross_entropy, X, W, y, loss, l, ws, reads=[X, W, y], writes=[loss, l, ws])
    assert not errs, errs[:3]
    for r in range(rows):
        assert abs(float(l[r]) - float(lse)) < 2e-4 and abs(float(loss[r]) - float(lse - z[y[r]])) < 4e-4
    W[9, 0] = float("nan")
    assert not emu.call(al.alcop_linear_cross_entropy, X, W, y, loss, l, ws, reads=[X, W, y], writes=[loss, l, ws])
    assert l.isnan().all() and loss.isnan().all()
    W[9, 0] = float("inf")
    assert not emu.call(al.alcop_linear_cross_entropy, X, W, y, loss, l, ws, reads=[X, W, y], writes=[loss, l, ws])
    assert (l == float("inf")).all()
    W[:, 0] = -float("inf")
    assert not emu.call(al.alcop_linear_cross_entropy, X, W, y, loss, l, ws, reads=[X, W, y], writes=[loss, l, ws])
    assert (l == -float("inf")).all()


def run_gradients(rows, vocab, K, dtype, out=None, alpha=1.0, pad=0, policy=(1, 0), parts="XW", dloss=True, mean=True, scale=2.0):
    X, W = matrix(rows, K, dtype, 1, pad), matrix(vocab, K, dtype, 2, pad, scale=scale * K ** -0.5)
    y = labels_of(rows, vocab, 3)
    lse = torch.logsumexp(alpha * (X.double() @ W.double().t()), dim=1).float()
    d = (vector(rows, 4) / rows if mean else vector(rows, 4) * 100) if dloss else None
    dX = matrix(rows, K, out or dtype, 5, pad) if "X" in parts else None
    dW = matrix(vocab, K, out or dtype, 6, pad) if "W" in parts else None
    with emu._swapped():
        ws = torch.empty(al.alcop_linear_cross_entropy_backward_workspace_bytes(rows, vocab, K), dtype=torch.uint8).fill_(255)
    rx, rw, ex, ew = loss_grad64(X, W, y, lse, d, alpha)
    errs = emu.call(al.alcop_linear_cross_entropy_backward, X, W, y, lse, ws, dX=dX, dW=dW, dloss=d, alpha=alpha,
                    reads=some(X, W, y, lse, d), writes=some(dX, dW, ws), policy=policy)
    assert not errs, errs[:4]
    if dX is not None:
        check(dX, rx, ex, "dX")
    if dW is not None:
        check(dW, rw, ew, "dW")


@pytest.mark.parametrize("kernel", range(KERNELS))
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_gradients_of_every_kernel(kernel, dtype, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    run_gradients(70, 300, 72, dtype, pad=8, policy=emu.POLICIES[kernel % 4])
    run_gradients(5, 131, 16, dtype, alpha=0.25, mean=False)


@pytest.mark.parametrize("dtype,out", [("f16", None), ("bf16", None), ("f16", "f32"), ("bf16", "f32")])
def test_gradients_in_pieces(dtype, out, monkeypatch):
    monkeypatch.setenv("ALCOP_LOSS_PIECE", "256")
    run_gradients(20, 256 * 2 + 43, 40, dtype, out=out, pad=8)
    run_gradients(20, 257, 40, dtype, out=out, parts="X")
    run_gradients(3, 512, 40, dtype, out=out, parts="W")


def test_gradients_left_out_and_small():
    run_gradients(1, 1, 8, "f16")
    run_gradients(9, 65, 24, "f16", dloss=False)
    run_gradients(9, 65, 24, "bf16", parts="X", dloss=False)
    run_gradients(9, 65, 24, "f16", parts="W", out="f32")


def test_rows_that_do_not_count_have_no_gradient():
    X, W = matrix(6, 16, "f16", 1), matrix(40, 16, "f16", 2)
    y = torch.tensor([-1, -100, 40, 41, 2 ** 40, -2 ** 63])
    dX, dW = matrix(6, 16, "f16", 3), matrix(40, 16, "f16", 4)
    lse, d = vector(6, 5), vector(6, 6)
    ws = torch.empty(al.alcop_linear_cross_entropy_backward_workspace_bytes(6, 40, 16), dtype=torch.uint8)
    errs = emu.call(al.alcop_linear_cross_entropy_backward, X, W, y, lse, ws, dX=dX, dW=dW, dloss=d, reads=[X, W, y, lse, d],
                    writes=[dX, dW, ws])
    assert not errs and not dX.any() and not dW.any()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_what_rows_that_do_not_count_or_are_lost_hold_does_not_reach_the_others(dtype):
    X, W, d = matrix(6, 16, dtype, 1), matrix(40, 16, dtype, 2), torch.tensor([1e-6, 0.0, 0.0, -1e-3, 0.0, 1e-4])
    y = torch.tensor([3, -100, 40, 0, 2 ** 33, 39])
    lse = torch.logsumexp(X.double() @ W.double().t(), dim=1).float()
    with emu._swapped():
        ws = torch.empty(al.alcop_linear_cross_entropy_backward_workspace_bytes(6, 40, 16), dtype=torch.uint8).fill_(255)

    def gradients(d, lse):
        dX, dW = matrix(6, 16, dtype, 3), matrix(40, 16, dtype, 4)
        errs = emu.call(al.alcop_linear_cross_entropy_backward, X, W, y, lse, ws, dX=dX, dW=dW, dloss=d, reads=[X, W, y, lse, d],
                        writes=[dX, dW, ws])
        assert not errs, errs[:3]
        return dX, dW

    clean, rest = gradients(d, lse), [0, 3, 5]
    assert clean[0][rest].any(dim=1).all()
    masked, their = d.clone(), lse.clone()
    masked[[1, 2, 4]], their[1] = torch.tensor([float("nan"), float("inf"), 1e30]), float("nan")
    for a, b in zip(clean, gradients(masked, their)):
        assert torch.equal(a, b)
    for lost in (float("inf"), float("nan")):
        bad = d.clone()
        bad[5] = lost
        dX = gradients(bad, lse)[0]
        assert torch.equal(dX[[0, 1, 2, 3, 4]], clean[0][[0, 1, 2, 3, 4]]) and not dX[5].isfinite().any()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_norms_experts_and_loss_together(dtype):
    from block_util import run_block

    def call(fn, *args, **kw):
        ts = [t for t in list(args) + list(kw.values()) if isinstance(t, torch.Tensor)]
        errs = emu.call(fn, *args, reads=ts, writes=ts, **kw)
        assert not errs, errs[:3]

    run_block(call, "cpu", dtype, 40, 40, 24, [0, 9, 21, 7], 131, behind=3)
