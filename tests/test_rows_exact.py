"""Rows to 8 bits on the CPU model: scales and 8-bit numbers are those of the definition, bit for bit, as every step of
it is one rounding of fp32.  And which of the rows' kernels alcop_init loads."""
import ctypes

import pytest
import torch

import emu_util as emu
import paper_2210_16691_amd as al
from test_layers_emulated import run_norm

DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
TINY = 2.0 ** -126


def plain(x):
    """(e4m3(x / scale), scale) of rows in fp32."""
    s = (x.float().abs().amax(dim=1) / 448.0).clamp_min(TINY)
    return (x.float() / s[:, None]).to(torch.float8_e4m3fn), s


def values(rows, cols, dtype, seed, scale=1.0):
    return (torch.randn(rows, cols, generator=torch.Generator().manual_seed(seed)) * scale).to(DT[dtype])


def quantized(x):
    y, s = torch.empty(x.shape, dtype=torch.float8_e4m3fn), torch.empty(x.shape[0])
    assert not emu.call(al.alcop_quantize_rows, x, y, s, reads=[x], writes=[y, s])
    return y, s


def same(got, want):
    assert torch.equal(got[1], want[1])
    assert torch.equal(got[0].view(torch.uint8), want[0].view(torch.uint8))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("cols", [1000, 4096])
def test_quotients_are_rounded_once_to_fp32(dtype, cols):
    x = values(24, cols, dtype, cols)
    # the product with the scale's reciprocal lies on the other side of a tie for some of these numbers
    s = plain(x)[1]
    assert not torch.equal((x.float() * (1.0 / s)[:, None]).to(torch.float8_e4m3fn).view(torch.uint8), plain(x)[0].view(torch.uint8)) \
        or dtype == "f32"
    same(quantized(x), plain(x))


@pytest.mark.parametrize("dtype,scale", [("f32", 1e-42), ("f32", 3e-38), ("f32", 1e-36), ("f32", 1e-20), ("f32", 1e-18), ("f32", 1e37),
                                         ("bf16", 1e-38), ("bf16", 1e-36), ("bf16", 1e-19), ("bf16", 6e37), ("f16", 1e-7), ("f16", 1e4)])
def test_quotients_of_tiny_and_huge_rows(dtype, scale):
    # scales at the lowest one, below and above where rows are scaled up first, near the end of the fp32 range; zeros of both signs
    x = values(12, 520, dtype, 7, scale)
    x[:, 3], x[:, 4] = 0.0, -0.0
    x[5] = x[5].sign() * x[5].abs().amax()
    assert x.isfinite().all()
    same(quantized(x), plain(x))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_an_8_bit_norm_is_its_fp32_norm_divided(dtype):
    x, r = values(9, 1032, dtype, 1, 2.0), values(9, 1032, dtype, 2)
    g = torch.randn(1032, generator=torch.Generator().manual_seed(3))
    y32, y, s = torch.empty(9, 1032), torch.empty(9, 1032, dtype=torch.float8_e4m3fn), torch.empty(9)
    assert not emu.call(al.alcop_rmsnorm, x, g, y32, residual=r, reads=[x, r, g], writes=[y32])
    assert not emu.call(al.alcop_rmsnorm, x, g, y, residual=r, scale=s, reads=[x, r, g], writes=[y, s])
    same((y, s), plain(y32))


def test_every_kernel_of_rows_is_loaded_ahead():
    # what alcop_init loads against what calls of any number of rows and columns launch
    sizes = [(r, c) for r in (1, 3, 4, 511, 1535, 1536, 5000) for c in
             (1, 511, 512, 513, 1024, 1025, 1600, 2047, 2048, 2049, 4096, 4097, 8192, 8193, 16384, 16385, 32768)]
    L = emu.lib()
    L.emu_rows_kernels.argtypes, L.emu_rows_kernels.restype = [ctypes.POINTER(ctypes.c_int), ctypes.c_int,
                                                               ctypes.POINTER(ctypes.c_int)], None
    flat, out = (ctypes.c_int * (2 * len(sizes)))(*[v for s in sizes for v in s]), (ctypes.c_int * 3)()
    L.emu_rows_kernels(flat, len(sizes), out)
    assert list(out) == [48, 48, 0]


@pytest.mark.parametrize("dtype,out,rows,cols", [("f16", "e4m3", 1536, 1032), ("f32", "f32", 1537, 1025), ("bf16", "bf16", 1536, 2048)])
def test_norms_of_rows_that_have_a_wave_each(dtype, out, rows, cols):
    # 1025 to 2048 columns are a block's row, but a wave's from 1536 rows on
    run_norm(rows, cols, dtype, out, pad=3 if cols % 8 else 8)
