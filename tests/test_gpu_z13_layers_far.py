"""Layers, norms and their gradients on matrices of more than 2^31 elements: rows at both ends, and around the places where an offset
passes 31 and 32 bits of elements and of bytes, against the plain forms in 64 bits."""
import pytest
import torch

import paper_2210_16691_amd as al
from gpu_util import DEV
from layers_util import HALF, ULP, check, check_e4m3, linear64, norm64, norm_grad64, slope64

pytestmark = pytest.mark.gpu
ROWS, COLS = 70000, 32768
# 2^31 elements are 65536 rows; 2^31 bytes of 16 bits 32768
SOME = [0, 1, 16383, 16384, 32767, 32768, 32769, 65535, 65536, 65537, 69998, 69999]


@pytest.fixture(autouse=True)
def memory():
    free, _ = torch.cuda.mem_get_info()
    if free < 60 << 30:
        pytest.skip("needs 60 GB")
    yield
    torch.cuda.empty_cache()


def normal(rows, cols, dtype=torch.bfloat16, scale=1.0, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = torch.empty(rows, cols, dtype=dtype, device=DEV)
    for r in range(0, rows, 8192):
        t[r:r + 8192] = (torch.randn(min(8192, rows - r), cols, generator=g, device=DEV) * scale).to(dtype)
    return t


@pytest.mark.parametrize("dtype,N", [("bf16", COLS), ("e4m3", COLS), ("bf16", COLS - 3)])
def test_a_layer_with_more_than_2_31_results(dtype, N):
    dt = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[dtype]
    A, W, b = normal(ROWS, 64, dt, seed=1), normal(N, 64, dt, 0.125, 2), torch.randn(N, device=DEV)
    C, r, z = torch.empty(ROWS, COLS, dtype=torch.bfloat16, device=DEV)[:, :N], normal(ROWS, COLS, seed=3)[:, :N], \
        torch.empty(ROWS, COLS, dtype=torch.bfloat16, device=DEV)[:, :N]
    al.alcop_linear(A, W, C, transB=True, bias=b, act=4, residual=r, pre=z, fp32_sums=True)
    torch.cuda.synchronize()
    ref, zref, ez, ec = linear64(A[SOME], W, True, 1.0, b, 4, r[SOME])
    check(C[SOME], ref, ec, "C")
    check(z[SOME], zref, ez, "pre")


def test_norms_of_more_than_2_31_elements():
    x, r, g = normal(ROWS, COLS, seed=1), normal(ROWS, COLS, seed=2), torch.randn(COLS, device=DEV)
    h, y, s = torch.empty_like(x), torch.empty(ROWS, COLS, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(ROWS, device=DEV)
    rstd = torch.empty(ROWS, device=DEV)
    al.alcop_rmsnorm(x, g, y, residual=r, total=h, scale=s, rstd=rstd)
    torch.cuda.synchronize()
    yref, href, dref = norm64(x[SOME], r[SOME], g)
    check(h[SOME], href, ULP * href.abs(), "total")
    check_e4m3(y[SOME], s[SOME], yref, (COLS / 2 + 9) * ULP, "y")
    del x, y
    dy, dx, dg = r, torch.empty_like(r), torch.empty(COLS, device=DEV)
    ws = torch.empty(al.alcop_rmsnorm_backward_workspace_bytes(ROWS, COLS), dtype=torch.uint8, device=DEV)
    al.alcop_rmsnorm_backward(dy, h, g, rstd, dx, dgain=dg, workspace=ws)
    torch.cuda.synchronize()
    ref, _, edx, _ = norm_grad64(dy[SOME], h[SOME], g, rstd[SOME])
    check(dx[SOME], ref, edx, "dx")
    some = slice(0, COLS, 4099)
    xh = dy[:, some].cpu().double() * (h[:, some].cpu().double() * rstd.cpu().double()[:, None])
    check(dg[None, some], xh.sum(0)[None], ((ROWS + 4) * ULP * xh.abs().sum(0))[None], "dgain")


def test_gradients_of_a_layer_with_more_than_2_31_results():
    K = 64
    dC, pre, W = normal(ROWS, COLS, seed=1), normal(ROWS, COLS, scale=1.5, seed=2), normal(COLS, K, scale=0.02, seed=3)
    A, dA, db = normal(ROWS, K, seed=4), torch.empty(ROWS, K, dtype=torch.bfloat16, device=DEV), torch.empty(COLS, device=DEV)
    ws = torch.empty(al.alcop_linear_backward_workspace_bytes(ROWS, COLS, K), dtype=torch.uint8, device=DEV)
    al.alcop_linear_backward(dC, A, W, dA=dA, dbias=db, pre=pre, act=3, transB=True, workspace=ws)
    torch.cuda.synchronize()
    d, z = dC[SOME].cpu().double(), pre[SOME].cpu().double()
    dz, edz = d * slope64(z, 3), d.abs() * 16 * ULP * (1 + z.abs())
    e = edz + HALF[torch.bfloat16] * (dz.abs() + edz) + 2.0 ** -25
    w = W.cpu().double()
    check(dA[SOME], dz @ w, (e + (COLS + 4) * ULP * dz.abs()) @ w.abs(), "dA")
    some = slice(0, COLS, 4099)
    d, z = dC[:, some].cpu().double(), pre[:, some].cpu().double()
    dz, edz = d * slope64(z, 3), d.abs() * 16 * ULP * (1 + z.abs())
    check(db[None, some], dz.sum(0)[None], (edz + (ROWS + 4) * ULP * dz.abs()).sum(0)[None], "dbias")
    with pytest.raises(al.AlcopError) as err:      # dW's operands span more than 2 GiB
        al.alcop_linear_backward(dC, A, W, dW=torch.empty_like(W), pre=pre, act=3, transB=True, workspace=ws)
    assert err.value.code == al.ERR_SIZE
