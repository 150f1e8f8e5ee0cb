"""The cross entropy of a vocabulary's product and its gradients on the GPU against their plain forms in 64 bits (on the CPU): every
kernel, types, pieces, pitches, captured graphs, streams; a run of norm, experts and loss, forward and backward."""
import pytest
import torch

import paper_2210_16691_amd as al
from gpu_util import DEV
from layers_util import HALF, check
from more_util import loss64, loss_grad64
from test_gpu_z11_layers import matrix, padding, vector
from test_loss_emulated import KERNELS, labels_of

pytestmark = pytest.mark.gpu


def workspace(bytes):
    return torch.empty(bytes, dtype=torch.uint8, device=DEV).fill_(255)


def run_loss(rows, vocab, K, dtype, alpha=1.0, pad=0, lse=True, scale=2.0):
    X, W = matrix(rows, K, dtype, 1, pad), matrix(vocab, K, dtype, 2, pad, scale=scale * K ** -0.5)
    y = labels_of(rows, vocab, 3).to(DEV)
    loss, l = vector(rows, 4), vector(rows, 5) if lse else None
    ref, lref, e, el = loss64(X, W, y, alpha)
    al.alcop_linear_cross_entropy(X, W, y, loss, l, workspace(al.alcop_linear_cross_entropy_workspace_bytes(rows, vocab, K)), alpha=alpha)
    torch.cuda.synchronize()
    check(loss[None], ref[None], e[None], "loss")
    if lse:
        check(l[None], lref[None], el[None], "lse")


@pytest.mark.parametrize("kernel", range(KERNELS))
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_every_kernel(kernel, dtype, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    run_loss(300, 1003, 136, dtype, pad=8)
    run_loss(5, 131, 16, dtype, alpha=0.25)
    run_loss(513, 5000, 520, dtype)


@pytest.mark.parametrize("rows", [1, 2, 31, 33, 200])
def test_sizes(rows):
    run_loss(rows, 1, 8, "f16")
    run_loss(rows, 65, 8, "f16", lse=False)
    run_loss(rows, 30011, 264, "bf16", alpha=0.5)


def test_logits_far_apart():
    run_loss(100, 2000, 64, "f16", scale=60.0)


def run_gradients(rows, vocab, K, dtype, out=None, alpha=1.0, pad=0, parts="XW", dloss=True, mean=True, scale=2.0):
    X, W = matrix(rows, K, dtype, 1, pad), matrix(vocab, K, dtype, 2, pad, scale=scale * K ** -0.5)
    y = labels_of(rows, vocab, 3).to(DEV)
    lse = torch.logsumexp(alpha * (X.double() @ W.double().t()), dim=1).float()
    d = (vector(rows, 4) / rows if mean else vector(rows, 4) * 100) if dloss else None
    dX = matrix(rows, K, out or dtype, 5, pad) if "X" in parts else None
    dW = matrix(vocab, K, out or dtype, 6, pad) if "W" in parts else None
    rx, rw, ex, ew = loss_grad64(X, W, y, lse, d, alpha)
    al.alcop_linear_cross_entropy_backward(X, W, y, lse, workspace(al.alcop_linear_cross_entropy_backward_workspace_bytes(rows, vocab, K)),
                                           dX=dX, dW=dW, dloss=d, alpha=alpha)
    torch.cuda.synchronize()
    for got, ref, e, what in ((dX, rx, ex, "dX"), (dW, rw, ew, "dW")):
        if got is not None:
            check(got, ref, e, what)
            assert padding(got).isnan().all()


@pytest.mark.parametrize("kernel", range(KERNELS))
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_gradients_of_every_kernel(kernel, dtype, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    run_gradients(300, 1003, 136, dtype, pad=8)
    run_gradients(5, 131, 16, dtype, alpha=0.25, mean=False)
    run_gradients(600, 3000, 264, dtype)


@pytest.mark.parametrize("dtype,out", [("f16", None), ("bf16", None), ("f16", "f32"), ("bf16", "f32")])
def test_gradients_in_pieces(dtype, out, monkeypatch):
    monkeypatch.setenv("ALCOP_LOSS_PIECE", "512")
    run_gradients(200, 512 * 3 + 43, 136, dtype, out=out, pad=8)
    run_gradients(200, 513, 40, dtype, out=out, parts="X")
    run_gradients(3, 1024, 40, dtype, out=out, parts="W")


def test_gradients_left_out_and_small():
    run_gradients(1, 1, 8, "f16")
    run_gradients(9, 65, 24, "f16", dloss=False)
    run_gradients(1, 30011, 264, "bf16", parts="X", dloss=False)
    run_gradients(70, 5003, 24, "f16", parts="W", out="f32")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_what_rows_that_do_not_count_hold_does_not_reach_the_others(dtype):
    rows, vocab, K = 1100, 3001, 136
    X, W, d = matrix(rows, K, dtype, 1), matrix(vocab, K, dtype, 2, scale=0.2), vector(rows, 4) / rows
    y, lse = labels_of(rows, vocab, 3).to(DEV), torch.logsumexp(X.float() @ W.float().t(), dim=1)
    wb = workspace(al.alcop_linear_cross_entropy_backward_workspace_bytes(rows, vocab, K))
    out = []
    for masked in (0.0, float("nan"), float("inf"), 1e30):
        for r in (5, 900, 1099):
            y[r], d[r], lse[r] = -100, masked, masked
        dX, dW = torch.zeros_like(X), torch.zeros_like(W)
        al.alcop_linear_cross_entropy_backward(X, W, y, lse, wb, dX=dX, dW=dW, dloss=d)
        out.append((dX, dW))
    assert out[0][0].isfinite().all() and out[0][1].isfinite().all() and out[0][1].any()
    for dX, dW in out[1:]:
        assert torch.equal(dX, out[0][0]) and torch.equal(dW, out[0][1])


def test_gradients_against_differences():
    # loss in fp32 of logits below 8: off by 2^-20; the third derivative of a log-sum of 40 logits along one weight is below 2 |x|^3
    g = torch.Generator().manual_seed(7)
    rows, vocab, K, step = 6, 40, 8, 2.0 ** -4
    X = (torch.randint(-8, 9, (rows, K), generator=g) / 8).to(DEV, torch.float16)
    W = (torch.randint(-8, 9, (vocab, K), generator=g) / 8).to(DEV, torch.float16)
    y = labels_of(rows, vocab, 3).to(DEV)
    d = vector(rows, 4)
    ws = workspace(al.alcop_linear_cross_entropy_workspace_bytes(rows, vocab, K))
    loss, lse = vector(rows, 5), vector(rows, 6)

    def value(X, W):
        al.alcop_linear_cross_entropy(X, W, y, loss, lse, ws)
        return float((loss.double() * d.double()).sum())

    value(X, W)
    dX, dW = torch.zeros(rows, K, device=DEV), torch.zeros(vocab, K, device=DEV)
    wb = workspace(al.alcop_linear_cross_entropy_backward_workspace_bytes(rows, vocab, K))
    al.alcop_linear_cross_entropy_backward(X, W, y, lse, wb, dX=dX, dW=dW, dloss=d)
    size = float(d.abs().sum())
    for t, grad, i in ((X, dX, 0), (W, dW, 1)):
        for at in range(0, t.numel(), 11):
            v = []
            for h in (step, -step):            # steps of 1/16 beside eighths are exact in fp16
                args = [X.clone(), W.clone()]
                args[i].view(-1)[at] += h
                v.append(value(*args))
            diff = (v[0] - v[1]) / (2 * step)
            # + G in fp16: 2^-11 of each of its numbers, at most size of them times |W|, |X| <= 1
            assert abs(diff - float(grad.view(-1)[at])) < size * (2.0 ** -20 / step + 2 * step ** 2 / 6 + 2 * HALF[torch.float16])


def test_a_captured_graph_gives_the_eager_bits(monkeypatch):
    monkeypatch.setenv("ALCOP_LOSS_PIECE", "512")
    rows, vocab, K = 200, 1500, 136
    for dtype in ("f16", "bf16"):
        X, W, y, d = matrix(rows, K, dtype, 1), matrix(vocab, K, dtype, 2, scale=0.2), labels_of(rows, vocab, 3).to(DEV), vector(rows, 4)
        ws = workspace(max(al.alcop_linear_cross_entropy_workspace_bytes(rows, vocab, K),
                           al.alcop_linear_cross_entropy_backward_workspace_bytes(rows, vocab, K)))

        def outputs():
            return (torch.zeros(rows, device=DEV), torch.zeros(rows, device=DEV), torch.zeros_like(X), torch.zeros_like(W))

        def step(loss, lse, dX, dW):
            al.alcop_linear_cross_entropy(X, W, y, loss, lse, ws)
            al.alcop_linear_cross_entropy_backward(X, W, y, lse, ws, dX=dX, dW=dW, dloss=d)

        al.alcop_init()
        caught, graph = outputs(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            step(*caught)
        for seed in (11, 12, 13):
            X.copy_(matrix(rows, K, dtype, seed))
            y.copy_(labels_of(rows, vocab, seed))
            d.copy_(vector(rows, seed) * seed)
            eager = outputs()
            step(*eager)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, e) for a, e in zip(caught, eager))


def test_a_stream_of_the_callers_own():
    rows, vocab, K = 64, 3001, 136
    X, W, y = matrix(rows, K, "bf16", 1), matrix(vocab, K, "bf16", 2, scale=0.2), labels_of(rows, vocab, 3).to(DEV)
    ws = [workspace(al.alcop_linear_cross_entropy_workspace_bytes(rows, vocab, K)) for _ in range(3)]
    outs = [torch.zeros(rows, device=DEV) for _ in range(3)]
    al.alcop_linear_cross_entropy(X, W, y, outs[0], None, ws[0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s, o, w in zip(streams, outs[1:], ws[1:]):
        al.alcop_linear_cross_entropy(X, W, y, o, None, w, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
