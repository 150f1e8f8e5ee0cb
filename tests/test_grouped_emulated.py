"""Products grouped by expert and their gradients on the CPU model of the hardware (tests/emu): bounds of every access, waits and
barriers, results against the plain forms in 64 bits."""
import pytest
import torch

import emu_util as emu
import paper_2210_16691_amd as al
from layers_util import DT, check
from more_util import grouped64, grouped_grad64
from test_layers_emulated import matrix, some, vector

KERNELS = 9             # per operand type, layout and class of activation (ALCOP_GROUPED_CLASS)
GRADIENT_KERNELS = 5    # of the weights' gradients, per operand type (ALCOP_GROUPED_GRAD)
F8_KERNELS = 5          # and on e4m3 operands with a 16-bit result (ALCOP_GROUPED_F8)


def groups_of(m, G):
    """A matrix of G * n rows as G matrices."""
    n = m.shape[0] // G
    return m.as_strided((G, n, m.shape[1]), (n * m.stride(0), m.stride(0), 1), m.storage_offset())


def offsets_of(sizes, first=0):
    return torch.tensor([first] + [first + sum(sizes[:i + 1]) for i in range(len(sizes))], dtype=torch.int32)


def rows_of(sizes, first):
    return slice(first, first + sum(sizes))


def run_grouped(sizes, N, K, dtype, transB, out="f16", act=0, bias=True, pre=True, scales=False, pad=0, alpha=1.0, first=0, behind=0,
                policy=(1, 0), offset=0):
    G, rows = len(sizes), first + sum(sizes) + behind
    A = matrix(rows, K, dtype, 1, pad)
    W = groups_of(matrix(G * (N if transB else K), K if transB else N, dtype, 2, pad, scale=K ** -0.5), G)
    offs = offsets_of(sizes, first)
    C = matrix(rows, N, out, 3, pad, offset=offset)
    z = matrix(rows, N, out, 4, pad, offset=offset) if pre else None
    b = vector(G * N, 5).view(G, N) if bias else None
    sa = vector(rows, 6).abs() + 0.5 if scales else None
    sw = vector(G * N, 7).abs().view(G, N) + 0.5 if scales else None
    before = C.clone()
    c, zr, ez, ec = grouped64(A, W, sizes, first, transB, alpha, b, act, sa, sw)
    errs = emu.call(al.alcop_grouped_linear, A, W, offs, C, transB=transB, alpha=alpha, bias=b, act=act, pre=z, scale_a=sa,
                    scale_w=sw, reads=some(A, W, offs, b, sa, sw), writes=some(C, z), policy=policy)
    assert not errs, errs[:4]
    part = rows_of(sizes, first)
    if sum(sizes):
        check(C[part], c[part], ec[part], "C")
    if pre and sum(sizes):
        check(z[part], zr[part], ez[part], "pre")
    for rest in (slice(0, first), slice(part.stop, rows)):
        assert torch.equal(C[rest], before[rest])


@pytest.mark.parametrize("kernel", range(KERNELS))
@pytest.mark.parametrize("dtype,transB", [("f16", False), ("f16", True), ("bf16", False), ("bf16", True), ("e4m3", True)])
def test_every_kernel(kernel, dtype, transB, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    i = kernel + 10 * transB + 20 * (dtype == "bf16")
    # groups of none, one, a tile's and a few more rows; columns and depth that fill no tile
    sizes, N, K = ([0, 1, 17, 0, 16, 3], 72, 144) if kernel < 4 else ([3, 0, 70, 1, 65], 136, 80)
    run_grouped(sizes, N, K, dtype, transB, out=("f16", "bf16", "f32")[i % 3], act=i % 5, scales=dtype == "e4m3" or i % 2 == 0, pad=16,
                first=i % 3, behind=2, policy=emu.POLICIES[i % 4])


@pytest.mark.parametrize("kernel", range(KERNELS, KERNELS + F8_KERNELS))
@pytest.mark.parametrize("act", [0, 2, 4])
def test_every_kernel_that_multiplies_8_bits_as_they_are(kernel, act, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    run_grouped([5, 0, 67], 136, 272, "e4m3", True, out=("f16", "bf16")[kernel % 2], act=act, scales=True, pad=16)
    with pytest.raises(al.AlcopError):            # fp32 results get fp32 sums
        run_grouped([4], 16, 16, "e4m3", True, out="f32")


def test_whole_turns_of_the_large_tiles_and_quarters_behind_them(monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(KERNELS - 1))
    run_grouped([1] * 255 + [0, 130, 2], 16, 16, "f16", True, pre=False, first=2, behind=3)


@pytest.mark.parametrize("policy", emu.POLICIES)
def test_more_groups_than_lanes(policy):
    sizes = [(7 * g) % 5 for g in range(150)]
    run_grouped(sizes, 24, 16, "f16", True, pre=False, first=3, behind=4, policy=policy)


def test_all_rows_in_one_group_and_no_rows_at_all():
    run_grouped([0, 0, 40, 0], 40, 32, "bf16", True, act=3)
    run_grouped([0] * 3, 40, 32, "bf16", True, first=2, behind=3)
    run_grouped([1], 8, 8, "f16", False)
    run_grouped([0] * 64 + [9], 24, 16, "f16", True)
    run_grouped([0] * 128 + [9], 24, 16, "f16", True)


def test_an_odd_number_of_columns():
    for N in (43, 1, 40):
        run_grouped([5, 0, 18], N, 48, "f16", True, out="bf16", act=4, scales=True, pad=1 * 8, offset=1)


def test_groups_with_the_same_weights():
    A, W = matrix(30, 32, "f16", 1), matrix(40, 32, "f16", 2)
    offs, C = offsets_of([10, 5, 15]), matrix(30, 40, "f16", 3)
    errs = emu.call(al.alcop_grouped_linear, A, W.expand(3, 40, 32), offs, C, transB=True, reads=[A, W, offs], writes=[C])
    assert not errs, errs[:3]
    ref = torch.empty(30, 40, dtype=torch.float16)
    errs = emu.call(al.alcop_linear, A, W, ref, transB=True, reads=[A, W], writes=[ref])
    assert not errs
    torch.testing.assert_close(C, ref, rtol=2e-3, atol=2e-3)


@pytest.mark.parametrize("bad", [[-7, 3, 9, 20], [0, 15, 4, 20], [0, 5, 900, 2000], [20, 10, 5, 0], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 0]])
def test_offsets_out_of_order_or_range_stay_in_bounds(bad):
    A, W = matrix(20, 32, "f16", 1), groups_of(matrix(3 * 40, 32, "f16", 2), 3)
    offs, C, pre = torch.tensor(bad, dtype=torch.int32), matrix(20, 40, "f16", 3), matrix(20, 40, "f16", 4)
    assert not emu.call(al.alcop_grouped_linear, A, W, offs, C, transB=True, reads=[A, W, offs], writes=[C])
    dA, dW, db = torch.zeros(20, 32, dtype=torch.float16), torch.zeros(3, 40, 32, dtype=torch.float16), torch.zeros(3, 40)
    ws = torch.zeros(al.alcop_grouped_linear_backward_workspace_bytes(20, 3, 40, 32), dtype=torch.uint8)
    assert not emu.call(al.alcop_grouped_linear_backward, C, A, W, offs, dA=dA, dW=dW, dbias=db, pre=pre, act=3, transB=True,
                        workspace=ws, reads=[C, A, W, offs, pre], writes=[dA, dW, db, ws])


def run_backward(sizes, N, K, dtype, transB, out=None, act=0, bias=True, pad=0, alpha=1.0, first=0, behind=0, policy=(1, 0),
                 parts="AWb"):
    G, rows = len(sizes), first + sum(sizes) + behind
    dC, A = matrix(rows, N, dtype, 1, pad), matrix(rows, K, dtype, 2, pad)
    w_shape = (N, K) if transB else (K, N)
    W = groups_of(matrix(G * w_shape[0], w_shape[1], dtype, 3, pad, scale=K ** -0.5), G)
    pre = matrix(rows, N, dtype, 4, pad) if act else None
    offs = offsets_of(sizes, first)
    dA = matrix(rows, K, out or dtype, 5, pad) if "A" in parts else None
    dW = groups_of(matrix(G * w_shape[0], w_shape[1], out or dtype, 6, pad), G) if "W" in parts else None
    db = vector(G * N, 7).view(G, N) if "b" in parts else None
    ws = torch.zeros(al.alcop_grouped_linear_backward_workspace_bytes(rows, G, N, K), dtype=torch.uint8)
    before = None if dA is None else dA.clone()
    ra, rw, rb, ea, ew, eb = grouped_grad64(dC, A, W, sizes, first, transB, pre, act, alpha)
    errs = emu.call(al.alcop_grouped_linear_backward, dC, A, W, offs, dA=dA, dW=dW, dbias=db, pre=pre, act=act, alpha=alpha,
                    transB=transB, workspace=ws, reads=some(dC, A, W, offs, pre), writes=some(dA, dW, db, ws), policy=policy)
    assert not errs, errs[:4]
    part = rows_of(sizes, first)
    if dA is not None:
        if sum(sizes):
            check(dA[part], ra[part], ea[part], "dA")
        for rest in (slice(0, first), slice(part.stop, rows)):
            assert torch.equal(dA[rest], before[rest])
    if dW is not None:
        for g in range(G):
            check(dW[g], rw[g], ew[g], "dW of group %d" % g)
    if db is not None:
        check(db, rb, eb, "dbias")


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("dtype,transB", [("f16", False), ("bf16", True)])
def test_gradients(act, dtype, transB):
    run_backward([3, 0, 41, 1, 70], 72, 40, dtype, transB, act=act, pad=8, first=2, behind=3, policy=emu.POLICIES[act % 4])


@pytest.mark.parametrize("kernel", range(GRADIENT_KERNELS))
@pytest.mark.parametrize("dtype,transB", [("f16", True), ("bf16", False)])
def test_gradients_of_every_kernel(kernel, dtype, transB, monkeypatch):
    # the weights' gradients by their own kernels, the rows' by those of the product
    monkeypatch.setenv("ALCOP_GRADIENT_KERNEL", str(kernel))
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel + 4))
    run_backward([3, 0, 41, 1, 70], 72, 136, dtype, transB, act=4, pad=8, first=2, behind=3, policy=emu.POLICIES[kernel % 4])


def test_gradients_of_larger_tiles():
    run_backward([130, 0, 9], 136, 264, "bf16", True, act=4)


def test_gradients_left_out():
    for parts in ("A", "W", "b", "Ab", "Wb"):
        run_backward([3, 0, 12], 24, 40, "f16", True, act=2, parts=parts)
        run_backward([3, 0, 12], 24, 40, "f16", False, act=0, parts=parts, out="f32", alpha=-0.5)


def test_gradients_without_rows_are_zero():
    run_backward([0, 0], 24, 40, "f16", True, act=2, first=1, behind=2)
    run_backward([(3 * g) % 4 for g in range(140)], 16, 8, "bf16", True, act=4)
