"""Norms, experts and loss together on the GPU, forward and backward (block_util); the operators on matrices of more than 2^31 elements;
another device than the current one where there is one."""
import pytest
import torch

import paper_2210_16691_amd as al
from block_util import run_block
from gpu_util import DEV
from layers_util import ULP, check
from more_util import grouped64, layernorm64, layernorm_grad64, loss64
from test_gpu_z13_layers_far import normal

pytestmark = pytest.mark.gpu


def direct(fn, *args, **kw):
    fn(*args, **kw)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_norms_experts_and_loss_together(dtype):
    run_block(direct, DEV, dtype, 300, 136, 264, [0, 90, 7, 130, 0, 53], 1003, behind=20)
    run_block(direct, DEV, dtype, 33, 512, 520, [33], 4099)


def test_the_run_gives_the_same_bits_again():
    runs = [run_block(direct, DEV, torch.bfloat16, 200, 72, 136, [50, 0, 140], 700, behind=10) for _ in range(3)]
    assert all(torch.equal(a, b) for run in runs[1:] for a, b in zip(runs[0], run))


def big():
    free, _ = torch.cuda.mem_get_info()
    if free < 60 << 30:
        pytest.skip("needs 60 GB")


def test_norms_of_more_than_2_31_elements():
    big()
    rows, cols = 70000, 32768
    some = [0, 1, 32767, 32768, 65535, 65536, 65537, 69999]
    x, g, b = normal(rows, cols, seed=1), torch.randn(cols, device=DEV), torch.randn(cols, device=DEV)
    y, h = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    al.alcop_layernorm(x, g, b, y, residual=x, total=h, mean=mean, rstd=rstd)
    torch.cuda.synchronize()
    ref = layernorm64(x[some], x[some], g, b)
    check(y[some], ref[0], ref[4], "y")
    del x
    dy, dx, dg = y, torch.empty_like(y), torch.empty(cols, device=DEV)
    ws = torch.empty(al.alcop_layernorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    al.alcop_layernorm_backward(dy, h, g, mean, rstd, dx, dgain=dg, workspace=ws)
    torch.cuda.synchronize()
    ref = layernorm_grad64(dy[some], h[some], g, mean[some], rstd[some])
    check(dx[some], ref[0], ref[3], "dx")


def test_grouped_products_of_more_than_2_31_results_and_weights():
    big()
    rows, N, K, G = 70000, 32768, 64, 1100         # 2.29e9 results, 2.31e9 weights
    A, W = normal(rows, K, seed=1), normal(G * N, K, scale=0.125, seed=2).view(G, N, K)
    sizes = [60] * (G - 1) + [rows - 60 * (G - 1)]
    offs = torch.tensor([0] + sizes).cumsum(0).to(torch.int32).to(DEV)
    C = torch.empty(rows, N, dtype=torch.bfloat16, device=DEV)
    al.alcop_grouped_linear(A, W, offs, C, transB=True, act=4)
    torch.cuda.synchronize()
    for g in (0, 1, 545, 546, 1023, 1024, 1025, G - 1):
        at = 60 * g
        ref, _, _, e = grouped64(A[at:at + 60], W[g:g + 1], [60], 0, True, act=4)
        check(C[at:at + 60], ref, e, "group %d" % g)


def test_a_vocabulary_of_more_than_2_31_numbers():
    big()
    rows, vocab, K = 40, 140000, 16384             # W: 2.29e9 numbers
    X, W = normal(rows, K, seed=1), normal(vocab, K, scale=2.0 * K ** -0.5, seed=2)
    y = torch.randint(0, vocab, (rows,), device=DEV)
    y[:3] = torch.tensor([vocab - 1, 131072, 65535])
    loss, lse = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    ws = torch.empty(al.alcop_linear_cross_entropy_workspace_bytes(rows, vocab, K), dtype=torch.uint8, device=DEV)
    al.alcop_linear_cross_entropy(X, W, y, loss, lse, ws)
    dW = torch.empty(vocab, K, dtype=torch.bfloat16, device=DEV)
    wb = torch.empty(al.alcop_linear_cross_entropy_backward_workspace_bytes(rows, vocab, K), dtype=torch.uint8, device=DEV)
    al.alcop_linear_cross_entropy_backward(X, W, y, lse, wb, dW=dW)
    torch.cuda.synchronize()
    # in 64 bits on the GPU, a part of the vocabulary at a time
    z = torch.cat([X.double() @ w.double().t() for w in W.split(10000)], dim=1)
    ref = torch.logsumexp(z, dim=1)
    hit = z.gather(1, y[:, None])[:, 0]
    # a product's sum is off by K 2^-24 of its terms' magnitudes, here 2 |x| |w| ~ 2 * 0.64 * sqrt(K) each
    e = (K + 4) * ULP * 2 * 0.64 * K ** 0.5 * torch.ones(rows, dtype=torch.float64) + 2.0 ** -14
    check(lse[None], ref.cpu()[None], e[None], "lse")
    check(loss[None], (ref - hit).cpu()[None], 2 * e[None], "loss")
    for at in (0, 131071, 131072, vocab - 1, int(y[5])):
        p = torch.exp(z[:, at] - lse.double()) - (y == at).double()
        got, want = dW[at].double(), p @ X.double()
        # G and dW are rounded to 2^-8 each, z's error in the exponent
        bound = (2 ** -7 + 2 * float(e[0])) * (p.abs() @ X.double().abs()) + 2.0 ** -30
        assert bool(((got - want).abs() <= bound).all())


def test_tensors_on_another_device_than_the_current_one():
    if torch.cuda.device_count() < 2:
        pytest.skip("one device")
    with torch.cuda.device(0):
        run_block(lambda fn, *a, **k: (fn(*a, **k), torch.cuda.synchronize("cuda:1")), "cuda:1", torch.float16, 60, 72, 64, [20, 40], 100)
