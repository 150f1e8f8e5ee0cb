"""Sums of layers on e4m3 operands on the CPU model, which cuts products off as the 8-bit matrix instruction does: within the
bound of it, and fp32 where that is asked for.  And that the check sees sums kept in too few bits, the model stores that
are not aligned."""
import ctypes

import pytest
import torch

import emu_util as emu
import paper_2210_16691_amd as al
from layers_util import check, linear64
from sums8_util import cancelling, check_sums, quantized_pair

KERNELS, F8_KERNELS = 11, 6


def some(*ts):
    return [t for t in ts if t is not None]


@pytest.mark.parametrize("kernel", range(KERNELS, KERNELS + F8_KERNELS))
def test_sums_of_the_8_bit_instruction(kernel, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    M, N, K = 133, 72, 336
    A, W, sa, sw = quantized_pair(M, N, K, kernel)
    for out, act in ((torch.float16, 0), (torch.bfloat16, 4)):
        C, z = torch.empty(M, N, dtype=out), torch.empty(M, N, dtype=out)
        assert not emu.call(al.alcop_linear, A, W, C, transB=True, act=act, pre=z, scale_a=sa, scale_w=sw, reads=[A, W, sa, sw], writes=[C, z])
        check_sums(C, z, A, W, act=act, sa=sa, sw=sw)
    A, W, exact = cancelling(70, 24, 64)
    C = torch.empty(70, 24, dtype=torch.float16)
    assert not emu.call(al.alcop_linear, A, W, C, transB=True, reads=[A, W], writes=[C])
    check_sums(C, None, A, W, random=False)
    assert C.eq(0).all()


@pytest.mark.parametrize("kernel", range(KERNELS))
def test_fp32_sums_that_are_asked_for(kernel, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    A, W, exact = cancelling(70, 24, 64)
    for act in (0, 1, 4):
        C, z = torch.empty(70, 24, dtype=torch.float16), torch.empty(70, 24, dtype=torch.float16)
        assert not emu.call(al.alcop_linear, A, W, C, transB=True, act=act, pre=z, fp32_sums=True, reads=[A, W], writes=[C, z])
        assert z.eq(exact).all()
        check(C, *linear64(A, W, True, act=act)[::3])


def test_no_kernel_of_the_8_bit_instruction_has_fp32_sums(monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(KERNELS))
    A, W, _ = cancelling(70, 24, 64)
    C = torch.empty(70, 24, dtype=torch.float16)
    with pytest.raises(al.AlcopError) as e:
        emu.call(al.alcop_linear, A, W, C, transB=True, fp32_sums=True, reads=[A, W], writes=[C])
    assert e.value.code == al.ERR_SCHED


def test_fp32_sums_of_other_operands_are_what_they_were():
    A, W = torch.randn(9, 64).half(), torch.randn(24, 64).half()
    C, D = torch.empty(9, 24), torch.empty(9, 24)
    for out, f in ((C, False), (D, True)):
        assert not emu.call(al.alcop_linear, A, W, out, transB=True, act=2, fp32_sums=f, reads=[A, W], writes=[out])
    assert torch.equal(C, D)


@pytest.mark.parametrize("act", [-1, 5, 15, 16 + 5, 32])
def test_activations_that_do_not_exist(act):
    A, W, C = torch.zeros(8, 8, dtype=torch.float16), torch.zeros(8, 8, dtype=torch.float16), torch.zeros(8, 8, dtype=torch.float16)
    with pytest.raises(al.AlcopError) as e:
        emu.call(al.alcop_linear, A, W, C, transB=True, act=act, reads=[A, W], writes=[C])
    assert e.value.code == al.ERR_UNSUPPORTED


def test_the_check_sees_sums_in_too_few_bits():
    M, N, K = 130, 120, 2064
    A, W, sa, sw = quantized_pair(M, N, K, 5)
    a, w = A.double() * sa.double()[:, None], W.double() * sw.double()[:, None]
    exact = a @ w.t()
    check_sums(exact.half(), None, A, W, sa=sa, sw=sw)
    running = torch.zeros(M, N)
    for k in range(0, K, 64):                      # what a running sum in bf16 makes of it
        running = (running.double() + a[:, k:k + 64] @ w[:, k:k + 64].t()).to(torch.bfloat16).float()
    short = exact - a[:, -16:] @ w[:, -16:].t()    # the last products left out
    for bad in (running, short, exact * 1.03):
        for t in (torch.float16, torch.bfloat16):
            with pytest.raises(AssertionError):
                check_sums(bad.to(t), None, A, W, sa=sa, sw=sw)


def test_stores_that_have_to_be_aligned_are_checked():
    L = emu.lib()
    L.emu_store16.argtypes, L.emu_store16.restype = [ctypes.c_void_p, ctypes.c_int], None
    buf = torch.zeros(16, dtype=torch.int64)
    at = buf.data_ptr() + (-buf.data_ptr()) % 16
    for kind, anywhere in enumerate((False, False, False, True, True)):
        for off, ok in ((0, True), (16, True), (8, anywhere), (2, anywhere), (1, False)):
            L.emu_reset(1, 0)
            L.emu_register_buffer(buf.data_ptr(), 128, 1)
            L.emu_store16(at + off, kind)
            assert (L.emu_error_count() == 0) == ok, (kind, off)
