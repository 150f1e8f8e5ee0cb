"""Linear layers, norms and 8-bit rows on the CPU model of the hardware (tests/emu): bounds of every access, waits
and barriers under every timing policy, and results against the plain forms in 64 bits."""
import ctypes

import numpy as np
import pytest
import torch

import emu_util as emu
import paper_2210_16691_amd as al
from layers_util import DT, HALF, ULP, check, check_e4m3, linear64, norm64, norm_grad64, slope64

F8_KERNELS = 6          # and on e4m3 operands with a 16-bit result (ALCOP_LINEAR_F8)
KERNELS = 11            # per operand type, layout and class of activation (ALCOP_LINEAR_CLASS)


def matrix(rows, cols, dtype, seed, pad=0, scale=1.0, offset=0):
    """Rows cols + pad apart, the first `offset` elements into their buffer; padding holds NaN."""
    g = torch.Generator().manual_seed(seed)
    flat = torch.full((offset + rows * (cols + pad),), float("nan"))
    v = flat[offset:].view(rows, cols + pad)[:, :cols]
    v.copy_(torch.randn(rows, cols, generator=g) * scale)
    return flat.to(DT[dtype])[offset:].view(rows, cols + pad)[:, :cols]


def vector(n, seed):
    return torch.randn(n, generator=torch.Generator().manual_seed(seed))


def some(*ts):
    return [t for t in ts if t is not None]


def run_linear(M, N, K, dtype, transB, out="f16", act=0, bias=True, residual=True, pre=True, scales=False, pad=0, alpha=1.0,
               policy=(1, 0), offset=0, in_place=False):
    A = matrix(M, K, dtype, 1, pad)
    W = matrix(*((N, K) if transB else (K, N)), dtype, 2, pad, scale=K ** -0.5)
    C = matrix(M, N, out, 3, pad, offset=offset)
    b = vector(N, 4) if bias else None
    r = (C if in_place else matrix(M, N, out, 5, pad, offset=offset)) if residual else None
    z = matrix(M, N, out, 6, pad, offset=offset) if pre else None
    sa, sw = (vector(M, 7).abs() + 0.5, vector(N, 8).abs() + 0.5) if scales else (None, None)
    ref, zref, ez, ec = linear64(A, W, transB, alpha, b, act, r, sa, sw)
    errs = emu.call(al.alcop_linear, A, W, C, transB=transB, alpha=alpha, bias=b, act=act, residual=r, pre=z, scale_a=sa,
                    scale_w=sw, reads=some(A, W, b, r, sa, sw), writes=some(C, z), policy=policy)
    assert not errs, errs[:4]
    check(C, ref, ec, "C")
    if pre:
        check(z, zref, ez, "pre")
    return C


def test_e4m3_conversions_of_the_model():
    L = emu.lib()
    L.emu_f32_to_e4m3.argtypes, L.emu_f32_to_e4m3.restype = [ctypes.c_float], ctypes.c_uint8
    L.emu_e4m3_to_f32.argtypes, L.emu_e4m3_to_f32.restype = [ctypes.c_uint8], ctypes.c_float
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    want = codes.view(torch.float8_e4m3fn).float().numpy()
    got = np.array([L.emu_e4m3_to_f32(int(c)) for c in codes], dtype=np.float32)
    assert np.array_equal(got, want, equal_nan=True)
    g = torch.Generator().manual_seed(0)
    vals = torch.cat([torch.randn(4000, generator=g) * 10.0 ** torch.randint(-4, 3, (4000,), generator=g),
                      codes.view(torch.float8_e4m3fn).float(), torch.tensor([0.0, -0.0, 2.0 ** -10, 3 * 2.0 ** -10, 17.0, 19.0])])
    vals = vals[(vals.abs() <= 448) | vals.isnan()]
    want = vals.to(torch.float8_e4m3fn).view(torch.uint8)
    for v, w in zip(vals.tolist(), want.tolist()):
        got = L.emu_f32_to_e4m3(v)
        assert got == w or (v != v and got & 0x7f == 0x7f), v


@pytest.mark.parametrize("kernel", range(KERNELS))
@pytest.mark.parametrize("dtype,transB", [("f16", False), ("f16", True), ("bf16", False), ("bf16", True), ("e4m3", True)])
def test_every_kernel_of_a_linear_layer(kernel, dtype, transB, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    i = kernel + 10 * transB + 20 * (dtype == "bf16")
    # two tiles of rows at most, a last tile that is not full in either direction, a partial last k-tile
    M, N, K = (37, 72, 144) if kernel < 4 else (140, 200, 80)
    run_linear(M, N, K, dtype, transB, out=("f16", "bf16", "f32")[i % 3], act=i % 5, scales=dtype == "e4m3" or i % 2 == 0, pad=16,
               policy=emu.POLICIES[i % 4])


def test_there_are_no_more_kernels(monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(KERNELS))
    with pytest.raises(al.AlcopError) as e:
        run_linear(8, 8, 16, "f16", True)
    assert e.value.code == al.ERR_SCHED


@pytest.mark.parametrize("kernel", range(KERNELS, KERNELS + F8_KERNELS))
@pytest.mark.parametrize("act", [0, 2, 4])
def test_every_kernel_that_multiplies_8_bits_as_they_are(kernel, act, monkeypatch):
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    run_linear(140, 200, 272, "e4m3", True, out=("f16", "bf16")[kernel % 2], act=act, scales=True, pad=16)
    run_linear(20, 43, 16, "e4m3", True, out="bf16", act=act, residual=False)
    with pytest.raises(al.AlcopError):            # fp32 results get fp32 sums
        run_linear(8, 16, 16, "e4m3", True, out="f32")


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("out", ["f16", "bf16", "f32"])
def test_activations_and_output_types(act, out):
    run_linear(5, 40, 32, "bf16" if out == "bf16" else "f16", True, out=out, act=act)


@pytest.mark.parametrize("kernel", [0, 3, 4, 8, 9])
@pytest.mark.parametrize("N,pad,offset", [(43, 16, 0), (40, 1, 0), (40, 16, 1), (1, 16, 0)])
def test_results_that_are_not_made_of_chunks(kernel, N, pad, offset, monkeypatch):
    # an odd number of columns, an odd pitch of C, an odd address: element by element, nothing beside them is written
    monkeypatch.setenv("ALCOP_LINEAR_KERNEL", str(kernel))
    dtype = "e4m3" if kernel % 2 else "f16"
    A, W = matrix(19, 48, dtype, 1, 16), matrix(N, 48, dtype, 2, 16, scale=0.2)
    for out in ("bf16", "f32"):
        C, r, z = (matrix(19, N, out, s, pad, offset=offset) for s in (3, 4, 5))
        whole = C.as_strided((19, N + pad), (N + pad, 1))[:18, N:].clone()
        b = vector(N, 6)
        ref, zref, ez, ec = linear64(A, W, True, 1.0, b, 4, r)
        errs = emu.call(al.alcop_linear, A, W, C, transB=True, bias=b, act=4, residual=r, pre=z, reads=[A, W, b, r], writes=[C, z])
        assert not errs, errs[:4]
        check(C, ref, ec, "C")
        check(z, zref, ez, "pre")
        assert whole.isnan().all() and C.as_strided((19, N + pad), (N + pad, 1))[:18, N:].isnan().all()


@pytest.mark.parametrize("M", [1, 2, 17])
def test_few_rows_and_the_residual_in_place(M):
    for dtype, K in (("f16", 8), ("bf16", 520), ("e4m3", 16), ("e4m3", 1040)):
        run_linear(M, 24, K, dtype, True, out="bf16", bias=False, pre=False, in_place=True)
        run_linear(M, 24, K, dtype, True, out="f32", residual=False, pre=False, alpha=-0.5)


@pytest.mark.parametrize("policy", emu.POLICIES)
def test_nothing_but_the_product(policy):
    run_linear(70, 136, 72, "bf16", False, out="bf16", bias=False, residual=False, pre=False, policy=policy)


def test_rows_of_a_linear_layer_keep_their_infinities_and_nan():
    A, W = matrix(6, 32, "f16", 1), matrix(16, 32, "f16", 2, scale=0.2)
    A[2, 5] = float("inf")
    A[4, 0] = float("nan")
    for act in range(5):
        C = torch.empty(6, 16, dtype=torch.float16)
        assert not emu.call(al.alcop_linear, A, W, C, transB=True, act=act, reads=[A, W], writes=[C])
        assert C[[0, 1, 3, 5]].isfinite().all() and C[4].isnan().all()
        z = A[2].double() @ W.double().t()
        # relu, GELU and SiLU of +infinity are infinite; of -infinity 0 for ReLU, else 0 * infinity
        assert torch.equal(C[2] == float("inf"), z == float("inf"))


# ---- gradients -------------------------------------------------------------------------------------------
def run_backward(M, N, K, dtype, transB, act, want="AWb", out=None, pad=0, alpha=1.0):
    out = out or dtype
    dC, pre = matrix(M, N, dtype, 1, pad), matrix(M, N, dtype, 2, pad, scale=1.5) if act else None
    A = matrix(M, K, dtype, 3, pad)
    W = matrix(*((N, K) if transB else (K, N)), dtype, 4, pad, scale=0.2)
    dA = matrix(M, K, out, 5, pad) if "A" in want else None
    dW = matrix(*W.shape, out, 6, pad) if "W" in want else None
    db = vector(N, 7) if "b" in want else None
    ws = torch.full((al.alcop_linear_backward_workspace_bytes(M, N, K),), 255, dtype=torch.uint8)
    errs = emu.call(al.alcop_linear_backward, dC, A, W, dA=dA, dW=dW, dbias=db, pre=pre, act=act, alpha=alpha, transB=transB,
                    workspace=ws, reads=some(dC, A, W, pre), writes=some(dA, dW, db, ws))
    assert not errs, errs[:4]
    # dZ: half a step of its type, and what the slope is off by
    d = dC.double()
    if act:
        z = pre.double()
        dz = d * slope64(z, act)
        edz = d.abs() * 16 * ULP * (1 + z.abs())
    else:
        dz, edz = d, 0 * d
    e = edz + HALF[DT[dtype]] * (dz.abs() + edz) * (act > 0) + 2.0 ** -25 * (act > 0)
    a, w = A.double(), W.double().t() if transB else W.double()
    if dA is not None:
        check(dA, alpha * dz @ w.t(), abs(alpha) * ((e + (N + 4) * ULP * dz.abs()) @ w.t().abs()), "dA")
    if dW is not None:
        ref, err = alpha * a.t() @ dz, abs(alpha) * (a.t().abs() @ (e + (M + 4) * ULP * dz.abs()))
        check(dW, ref.t() if transB else ref, err.t() if transB else err, "dW")
    if db is not None:
        check(db, dz.sum(0), (edz + (M + 4) * ULP * dz.abs()).sum(0), "dbias")


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("dtype,transB", [("f16", False), ("f16", True), ("bf16", False), ("bf16", True)])
def test_gradients_of_a_linear_layer(act, dtype, transB):
    run_backward(37, 72, 48, dtype, transB, act, pad=8, alpha=0.5)


@pytest.mark.parametrize("M", [1, 3, 8, 130])
def test_gradients_of_any_number_of_rows(M):
    # dW sums over the layer's rows: every remainder of 8
    run_backward(M, 40, 24, "f16", True, 3)
    run_backward(M, 40, 24, "bf16", False, 0, out="f32")


@pytest.mark.parametrize("want", ["A", "W", "b", "Ab", "AW"])
@pytest.mark.parametrize("act", [0, 4])
def test_gradients_one_by_one(want, act):
    run_backward(20, 16, 32, "bf16", True, act, want=want)


def test_the_bias_gradient_over_several_blocks():
    run_backward(1100, 520, 8, "f16", True, 1, want="b")


# ---- rows -----------------------------------------------------------------------------------------------
COLS = [1, 7, 8, 511, 520, 1023, 1032, 2048, 2056, 4101, 5000, 9000, 17000]


def run_norm(rows, cols, dtype, out, residual=True, gain=True, pad=0, offset=0, total=True):
    x, r = matrix(rows, cols, dtype, 1, pad, 2.0, offset), matrix(rows, cols, dtype, 2, pad, 1.0, offset) if residual else None
    h = matrix(rows, cols, dtype, 3, pad, offset=offset) if total else None
    g = vector(cols, 4) if gain else None
    y = matrix(rows, cols, out, 5, pad, offset=offset)
    s, d = vector(rows, 6) if out == "e4m3" else None, vector(rows, 7)
    yref, href, dref = norm64(x, r, g)
    errs = emu.call(al.alcop_rmsnorm, x, g, y, residual=r, total=h, scale=s, rstd=d, reads=some(x, r, g), writes=some(y, h, s, d))
    assert not errs, errs[:4]
    # half the sum's relative error, and a few roundings
    err = (cols / 2 + 8) * ULP
    check(d[:, None], dref[:, None], err * dref[:, None], "rstd")
    if total:
        check(h, href, ULP * href.abs(), "total")
    eh = ULP * href.abs() * dref[:, None] * (1 if g is None else g.double().abs())
    if out == "e4m3":
        check_e4m3(y, s, yref, err, "y")
    else:
        check(y, yref, err * yref.abs() + eh, "y")


@pytest.mark.parametrize("cols", COLS)
def test_norm_of_every_row_length(cols):
    k = COLS.index(cols)
    dtype = ("f16", "bf16", "f32")[k % 3]
    run_norm(3 if cols > 2000 else 6, cols, dtype, "e4m3" if k % 2 else dtype, pad=(0, 8, 3)[k % 3])
    run_norm(1, cols, ("bf16", "f32", "f16")[k % 3], ("e4m3", "f32")[k % 2], residual=k % 2 == 0, gain=k % 4 != 0, total=False)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("out", ["f16", "bf16", "f32", "e4m3"])
@pytest.mark.parametrize("offset", [0, 1])
def test_norm_of_every_type(dtype, out, offset):
    run_norm(5, 72, dtype, out, pad=8, offset=offset)


def test_rows_that_have_a_wave_each():
    # 1537 to 2048 columns are a block's row, but a wave's from 1536 rows on
    for rows, cols in ((1537, 1040), (1536, 1601)):
        x, y, s = matrix(rows, cols, "bf16", 1, 8), matrix(rows, cols, "e4m3", 2), vector(rows, 3)
        assert not emu.call(al.alcop_quantize_rows, x, y, s, reads=[x], writes=[y, s])
        check_e4m3(y, s, x.double(), 0.0)


def test_norm_in_place():
    for dtype in ("bf16", "f32"):
        x, r, g = matrix(5, 40, dtype, 1), matrix(5, 40, dtype, 2), vector(40, 3)
        yref, href, dref = norm64(x, r, g)
        errs = emu.call(al.alcop_rmsnorm, x, g, x, residual=r, total=r, reads=[g], writes=[x, r])
        assert not errs, errs[:4]
        check(r, href, ULP * href.abs(), "total")
        check(x, yref, 40 * ULP * yref.abs() + ULP * href.abs() * dref[:, None] * g.double().abs(), "y")


def test_rows_of_zeros_tiny_and_infinite_values():
    x = torch.zeros(6, 24)
    x[1] = 1e-42                                  # y is not zero, its sum of squares is
    x[2, 3] = 1e30
    x[3, 0] = float("inf")
    x[4, 7] = float("nan")
    x[5] = torch.arange(24) - 11.5
    y, s = torch.empty(6, 24, dtype=torch.float8_e4m3fn), torch.empty(6)
    assert not emu.call(al.alcop_quantize_rows, x, y, s, reads=[x], writes=[y, s])
    assert torch.equal(y[0].float(), torch.zeros(24)) and s[0] == 2.0 ** -126 and s[1] == 2.0 ** -126
    assert y[2, 3].float() == 448 and abs(float(s[2]) / (1e30 / 448) - 1) < 1e-6 and y[2].float().sum() == 448
    assert s[3] == float("inf") and y[3, 0].float().isnan() and y[3, 1:].float().eq(0).all()
    assert s[4].isnan() and y[4].float().isnan().all()
    assert y[5].float().isfinite().all()


@pytest.mark.parametrize("cols", COLS)
def test_quantize_every_row_length(cols):
    k = COLS.index(cols)
    x = matrix(4, cols, ("bf16", "f16", "f32")[k % 3], 1, (0, 3, 8)[k % 3], 3.0)
    y, s = matrix(4, cols, "e4m3", 2, (8, 5, 0)[k % 3]), vector(4, 3)
    assert not emu.call(al.alcop_quantize_rows, x, y, s, reads=[x], writes=[y, s])
    check_e4m3(y, s, x.double(), 0.0)


def run_norm_backward(rows, cols, dtype, gain=True, dtotal=True, dgain=True, pad=0, alias=None):
    dy, h = matrix(rows, cols, dtype, 1, pad), matrix(rows, cols, dtype, 2, pad, 2.0)
    g = vector(cols, 3) if gain else None
    rstd = (h.double().square().mean(1) + 1e-6).rsqrt().float()
    dt = matrix(rows, cols, dtype, 4, pad) if dtotal else None
    dx = {"dy": dy, "dtotal": dt}.get(alias)
    dx = matrix(rows, cols, dtype, 5, pad) if dx is None else dx
    dg = vector(cols, 6) if dgain else None
    ws = torch.full((al.alcop_rmsnorm_backward_workspace_bytes(rows, cols),), 255, dtype=torch.uint8) if dgain else None
    ref, gref, edx, edg = norm_grad64(dy, h, g, rstd, dt)
    errs = emu.call(al.alcop_rmsnorm_backward, dy, h, g, rstd, dx, dgain=dg, dtotal=dt, workspace=ws,
                    reads=some(dy, h, g, rstd, dt), writes=some(dx, dg, ws))
    assert not errs, errs[:4]
    check(dx, ref, edx, "dx")
    if dgain:
        check(dg[None], gref[None], edg[None], "dgain")


@pytest.mark.parametrize("cols", COLS)
def test_norm_gradient_of_every_row_length(cols):
    k = COLS.index(cols)
    run_norm_backward(3 if cols > 2000 else 9, cols, ("bf16", "f16", "f32")[k % 3], pad=(0, 3, 8)[k % 3])
    run_norm_backward(1, cols, ("f32", "bf16", "f16")[k % 3], gain=k % 2 == 0, dtotal=False, dgain=k % 3 == 0)


def test_norm_gradient_of_more_rows_than_groups():
    run_norm_backward(4099, 8, "f16")             # 1024 blocks of four rows: the first group takes two
    run_norm_backward(1027, 1040, "bf16", dtotal=False)


@pytest.mark.parametrize("alias", ["dy", "dtotal"])
def test_norm_gradient_in_place(alias):
    run_norm_backward(6, 520, "bf16", alias=alias)
    run_norm_backward(2, 17000, "f16", alias=alias)


@pytest.mark.parametrize("policy", emu.POLICIES)
def test_norm_waits_and_barriers(policy):
    x, g = matrix(2, 3000, "bf16", 1), vector(3000, 2)
    y, s = matrix(2, 3000, "e4m3", 3), vector(2, 4)
    assert not emu.call(al.alcop_rmsnorm, x, g, y, scale=s, reads=[x, g], writes=[y, s], policy=policy)
    check_e4m3(y, s, norm64(x, None, g)[0], 1508 * ULP)
    dx, dg = matrix(40, 3000, "bf16", 5), vector(3000, 6)
    dy, h = matrix(40, 3000, "bf16", 7), matrix(40, 3000, "bf16", 8)
    rstd = (h.double().square().mean(1) + 1e-6).rsqrt().float()
    ws = torch.empty(al.alcop_rmsnorm_backward_workspace_bytes(40, 3000), dtype=torch.uint8)
    assert not emu.call(al.alcop_rmsnorm_backward, dy, h, g, rstd, dx, dgain=dg, workspace=ws, reads=[dy, h, g, rstd],
                        writes=[dx, dg, ws], policy=policy)
    ref, gref, edx, edg = norm_grad64(dy, h, g, rstd)
    check(dx, ref, edx)
    check(dg[None], gref[None], edg[None])


# ---- a block: norm, 8-bit layer, 8-bit layer with the residual -----------------------------------------------
def test_a_feed_forward_block_in_8_bits():
    T, D, F = 11, 64, 96
    x, r, g = matrix(T, D, "bf16", 1), matrix(T, D, "bf16", 2), vector(D, 3)
    w1, w2, b1 = matrix(F, D, "bf16", 4, scale=D ** -0.5), matrix(D, F, "bf16", 5, scale=F ** -0.5), vector(F, 6)
    f8 = lambda rows, cols: torch.empty(rows, cols, dtype=torch.float8_e4m3fn)
    q1, s1, q2, s2, q3, s3, q4, s4 = f8(F, D), torch.empty(F), f8(D, F), torch.empty(D), f8(T, D), torch.empty(T), f8(T, F), torch.empty(T)
    h, u, out = torch.empty_like(x), torch.empty(T, F, dtype=torch.bfloat16), torch.empty_like(x)
    for fn, args, kw, reads, writes in [
            (al.alcop_quantize_rows, (w1, q1, s1), {}, [w1], [q1, s1]),
            (al.alcop_quantize_rows, (w2, q2, s2), {}, [w2], [q2, s2]),
            (al.alcop_rmsnorm, (x, g, q3), dict(residual=r, total=h, scale=s3), [x, r, g], [q3, h, s3]),
            (al.alcop_linear, (q3, q1, u), dict(transB=True, bias=b1, act=4, scale_a=s3, scale_w=s1), [q3, q1, b1, s3, s1], [u]),
            (al.alcop_quantize_rows, (u, q4, s4), {}, [u], [q4, s4]),
            (al.alcop_linear, (q4, q2, out), dict(transB=True, residual=h, scale_a=s4, scale_w=s2), [q4, q2, h, s4, s2], [out])]:
        assert not emu.call(fn, *args, reads=reads, writes=writes, **kw)
    # against the same steps on the 8-bit numbers as they are, in 64 bits
    val = lambda q, s: q.double() * s.double()[:, None]
    ref, _, _, ec = linear64(q3, q1, True, 1.0, b1, 4, None, s3, s1)
    check(u, ref, ec)
    ref, _, _, ec = linear64(q4, q2, True, 1.0, None, 0, h, s4, s2)
    check(out, ref, ec)
    y, href, _ = norm64(x, r, g)
    assert float((val(q3, s3) - y).abs().max() / y.abs().max()) <= 2.0 ** -4
