"""On the GPU: rows to 8 bits are those of the definition, bit for bit; activations and slopes are near relative to their size."""
import pytest
import torch

import paper_2210_16691_amd as al
from gpu_util import DEV
from test_layers_accuracy import check_activation, check_slope
from test_rows_exact import plain, same, values

pytestmark = pytest.mark.gpu


def quantized(x):
    y, s = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(x.shape[0], device=DEV)
    al.alcop_quantize_rows(x.to(DEV), y, s)
    torch.cuda.synchronize()
    return y.cpu(), s.cpu()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(3000, 72), (700, 1000), (1700, 1600), (60, 1603), (200, 4096), (50, 9000), (30, 32767)])
def test_quotients_are_rounded_once_to_fp32(dtype, rows, cols):
    x = values(rows, cols, dtype, cols)
    same(quantized(x), plain(x))


@pytest.mark.parametrize("dtype,scale", [("f32", 1e-42), ("f32", 3e-38), ("f32", 1e-36), ("f32", 1e-20), ("f32", 1e-18), ("f32", 1e37),
                                         ("bf16", 1e-38), ("bf16", 1e-36), ("bf16", 1e-19), ("bf16", 6e37), ("f16", 1e-7), ("f16", 1e4)])
def test_quotients_of_tiny_and_huge_rows(dtype, scale):
    x = values(300, 520, dtype, 7, scale)
    x[:, 3], x[:, 4] = 0.0, -0.0
    x[5] = x[5].sign() * x[5].abs().amax()
    same(quantized(x), plain(x))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(9, 1032), (1600, 1536), (300, 4096)])
def test_an_8_bit_norm_is_its_fp32_norm_divided(dtype, rows, cols):
    x, r = values(rows, cols, dtype, 1, 2.0).to(DEV), values(rows, cols, dtype, 2).to(DEV)
    g = torch.randn(cols, generator=torch.Generator().manual_seed(3)).to(DEV)
    y32, s = torch.empty(rows, cols, device=DEV), torch.empty(rows, device=DEV)
    y = torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device=DEV)
    al.alcop_rmsnorm(x, g, y32, residual=r)
    al.alcop_rmsnorm(x, g, y, residual=r, scale=s)
    torch.cuda.synchronize()
    same((y.cpu(), s.cpu()), plain(y32.cpu()))


def on_the_gpu(fn, *args, reads=None, writes=None, **kw):
    fn(*args, **kw)
    torch.cuda.synchronize()


@pytest.mark.parametrize("act", [2, 3, 4])
def test_activations_are_near_relative_to_their_value(act):
    check_activation(on_the_gpu, act, DEV)


@pytest.mark.parametrize("act", [2, 3, 4])
def test_slopes_are_near_relative_to_their_terms(act):
    check_slope(on_the_gpu, act, DEV)
