"""Operators of a transformer block around its matrix products, as timed cases.

Kinds of case:

linear           C = act(alpha * A.W + bias) + residual, optionally keeping the value in front of the
                 activation for training; W stored K x N or (as a layer's weights are) N x K
linear8          the same on e4m3 operands with one scale per row of A and one per column of the product
linear_backward  its gradients: with respect to A, W and the bias
norm             root-mean-square norm of x + residual, the sum kept as the next residual; the result in
                 the input's type, or in e4m3 with one scale per row, as linear8 takes it
norm_backward    its gradients: with respect to the sum (which is that of x and of the residual) and the gain
quantize         rows to e4m3 with one scale per row: weights when they are loaded, activations between
                 two 8-bit products

Activations: 0 none, 1 ReLU, 2 GELU (erf), 3 GELU (tanh approximation), 4 SiLU.
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
_SIZE = {"f16": 2, "bf16": 2, "f32": 4, "e4m3": 1}
_E4M3_MAX = 448.0
_TINY = 2.0 ** -126


def listed():
    return [
        # the smallest call: the output projection of one token, with the residual (launch latency)
        dict(name="linear_token", kind="linear", M=1, N=768, K=768, dtype="bf16", out="bf16", transB=True, act=0,
             bias=True, residual=True, pre=False, alpha=1.0, pad=0),
        # a layer at sizes that fill no tile, rows further apart than they are long, weights stored K x N
        dict(name="linear_ragged", kind="linear", M=507, N=2072, K=1000, dtype="f16", out="f16", transB=False, act=2,
             bias=True, residual=True, pre=False, alpha=1.0, pad=24),
        # the first layer of a feed-forward block in training: the value in front of the activation is kept
        dict(name="linear_train_8192", kind="linear", M=8192, N=8192, K=2048, dtype="bf16", out="bf16", transB=True,
             act=3, bias=True, residual=False, pre=True, alpha=1.0, pad=0),
        # the gradients of such a layer
        dict(name="linear_backward_4096", kind="linear_backward", M=4096, N=4096, K=1024, dtype="bf16", transB=True,
             act=3, bias=True, alpha=1.0, pad=0),
        # sixteen sequences decoding against 8-bit weights: the weights' bytes are what counts
        dict(name="linear8_step_16", kind="linear8", M=16, N=4096, K=4096, out="bf16", act=0, bias=False,
             residual=True, pre=False, alpha=1.0, pad=0),
        # a ragged prompt through an 8-bit layer
        dict(name="linear8_ragged", kind="linear8", M=1531, N=2050, K=1040, out="f16", act=4, bias=True,
             residual=False, pre=False, alpha=0.5, pad=16),
        # a long prompt through an 8-bit layer, the largest call
        dict(name="linear8_8192", kind="linear8", M=8192, N=8192, K=4096, out="bf16", act=0, bias=False,
             residual=True, pre=False, alpha=1.0, pad=0),
        # the norm in front of an 8-bit product, one token
        dict(name="norm8_token", kind="norm", rows=1, cols=4096, dtype="bf16", out="e4m3", residual=True, gain=True,
             pad=0),
        # the same for a training batch, in 16 bits
        dict(name="norm_16384", kind="norm", rows=16384, cols=4096, dtype="bf16", out="bf16", residual=True, gain=True,
             pad=0),
        # its gradients
        dict(name="norm_backward_8192", kind="norm_backward", rows=8192, cols=4096, dtype="bf16", gain=True, dtotal=True,
             pad=0),
        # a weight matrix to 8 bits, one scale per output channel
        dict(name="quantize_8192", kind="quantize", rows=8192, cols=4096, dtype="bf16", pad=0),
        # ragged activations to 8 bits
        dict(name="quantize_ragged", kind="quantize", rows=1531, cols=1111, dtype="f16", pad=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear8", "linear8", "linear_backward", "norm", "norm", "norm_backward",
                       "quantize"])
    if kind.startswith("linear"):
        unit = 16 if kind == "linear8" else 8
        while True:
            M = _log_int(rng, 1, 8192)
            N = max(64, _log_int(rng, 64, 8192) // 8 * 8)
            K = max(64, _log_int(rng, 64, 8192) // unit * unit)
            if M * N * K <= 2 ** 37:
                break
        alpha = rng.choice([1.0, 1.0, 0.5])
        pad = rng.choice([0, 0, unit, 3 * unit])
        act = rng.randrange(5)
        if kind == "linear_backward":
            return dict(kind=kind, M=M, N=N, K=K, dtype=rng.choice(["f16", "bf16"]), transB=rng.random() < 0.5, act=act,
                        bias=rng.random() < 0.7, alpha=alpha, pad=pad)
        case = dict(kind=kind, M=M, N=N, K=K)
        if kind == "linear":
            dtype = rng.choice(["f16", "bf16"])
            case.update(dtype=dtype, out=rng.choice([dtype, dtype, "f32"]), transB=rng.random() < 0.6)
        else:
            case.update(out=rng.choice(["f16", "bf16", "bf16", "f32"]))
        if case.get("transB", True) and rng.random() < 0.25:
            case["N"] = N - rng.randrange(1, 8)          # rows of weights need not be a multiple of anything
        case.update(act=act, bias=rng.random() < 0.6, residual=rng.random() < 0.5, pre=rng.random() < 0.3, alpha=alpha,
                    pad=pad)
        return case
    while True:
        rows, cols = _log_int(rng, 1, 16384), _log_int(rng, 64, 16384)
        if rows * cols <= 2 ** 26:
            break
    if rng.random() < 0.6:
        cols = max(64, cols // 8 * 8)
    case = dict(kind=kind, rows=rows, cols=cols, dtype=rng.choice(["f16", "bf16", "bf16", "f32"]),
                pad=rng.choice([0, 0, 8, 3]))
    if kind == "norm":
        case.update(out=rng.choice([case["dtype"], "e4m3"]), residual=rng.random() < 0.7, gain=rng.random() < 0.9)
    elif kind == "norm_backward":
        case.update(gain=rng.random() < 0.9, dtotal=rng.random() < 0.7)
    return case


# ---- inputs --------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 17)
    return g


def _matrix(g, rows, cols, pad, dtype, scale=1.0, outliers=False):
    """Normal values (with a few columns of larger ones, as activations have), rows cols + pad apart."""
    v = torch.randn(rows, cols + pad, generator=g, device="cuda") * scale
    if outliers:
        v[:, :: max(1, cols // 5)] *= 8.0
    return v.to(_DT[dtype])[:, :cols]


def _matrix8(g, rows, cols, pad, scale=1.0, outliers=False):
    v = _matrix(g, rows, cols, pad, "f32", scale, outliers)
    s = v.abs().amax(dim=1).clamp_min(1e-30) / _E4M3_MAX
    full = torch.zeros(rows, cols + pad, device="cuda", dtype=torch.float8_e4m3fn)
    full[:, :cols] = (v / s[:, None]).to(torch.float8_e4m3fn)
    return full[:, :cols], s


def _empty(rows, cols, pad, dtype):
    return torch.empty(rows, cols + pad, device="cuda", dtype=_DT[dtype])[:, :cols]


def prepare(case, seed):
    g = _generator(seed)
    kind, pad = case["kind"], case["pad"]
    st = {"case": case}
    if kind.startswith("linear"):
        M, N, K = case["M"], case["N"], case["K"]
        tb = case.get("transB", True)
        w_shape = (N, K) if tb else (K, N)
        if kind == "linear8":
            st["A"], st["sa"] = _matrix8(g, M, K, pad, outliers=True)
            st["W"], st["sw"] = _matrix8(g, N, K, pad, scale=K ** -0.5)
            out = case["out"]
        else:
            dtype = case["dtype"]
            st["A"] = _matrix(g, M, K, pad, dtype, outliers=True)
            st["W"] = _matrix(g, *w_shape, pad, dtype, scale=K ** -0.5)
            out = case.get("out", dtype)
        st["bias"] = torch.randn(N, generator=g, device="cuda") * 0.5 if case["bias"] else None
        if kind == "linear_backward":
            st["dC"] = _matrix(g, M, N, pad, case["dtype"], scale=0.5)
            st["pre"] = _matrix(g, M, N, pad, case["dtype"], scale=1.5) if case["act"] else None
            st["dA"] = _empty(M, K, pad, case["dtype"])
            st["dW"] = _empty(*w_shape, pad, case["dtype"])
            st["dbias"] = torch.empty(N, device="cuda") if case["bias"] else None
            if own:
                import paper_2210_16691_amd as al
                st["ws"] = torch.empty(al.alcop_linear_backward_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
        else:
            st["residual"] = _matrix(g, M, N, pad, out) if case["residual"] else None
            st["C"] = _empty(M, N, pad, out)
            st["pre"] = _empty(M, N, pad, out) if case["pre"] else None
        return st
    rows, cols, dtype = case["rows"], case["cols"], case["dtype"]
    if kind == "norm_backward":
        st["dy"] = _matrix(g, rows, cols, pad, dtype, scale=0.5)
        st["total"] = _matrix(g, rows, cols, pad, dtype, scale=2.0, outliers=True)
        st["rstd"] = (st["total"].double().square().mean(dim=1) + 1e-6).rsqrt().float()
        st["dtotal"] = _matrix(g, rows, cols, pad, dtype) if case["dtotal"] else None
        st["dx"] = _empty(rows, cols, pad, dtype)
        st["dgain"] = torch.empty(cols, device="cuda") if case["gain"] else None
        if own:
            import paper_2210_16691_amd as al
            st["ws"] = torch.empty(al.alcop_rmsnorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    else:
        st["x"] = _matrix(g, rows, cols, pad, dtype, outliers=True)
        out = case.get("out", "e4m3")
        st["y"] = _empty(rows, cols, pad, out)
        st["scale"] = torch.empty(rows, device="cuda") if out == "e4m3" else None
        if kind == "norm":
            st["residual"] = _matrix(g, rows, cols, pad, dtype, scale=2.0) if case["residual"] else None
            st["total"] = _empty(rows, cols, pad, dtype) if case["residual"] else None
            st["rstd"] = torch.empty(rows, device="cuda")
    if kind != "quantize":
        st["gain"] = 1.0 + 0.2 * torch.randn(cols, generator=g, device="cuda") if case["gain"] else None
    return st


# ---- the operators in their plain form -------------------------------------------------------------
def _act(z, act):
    if act == 1:
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == 2:
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == 3:
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == 4:
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == 1:
        return (z > 0).to(z.dtype)
    if act == 2:
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == 3:
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * z * z)
    if act == 4:
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _plain_linear(st):
    case = st["case"]
    w = st["W"].float()
    z = st["A"].float() @ (w.t() if case.get("transB", True) else w)
    if "sa" in st:
        z = z * st["sa"][:, None] * st["sw"][None, :]
    z = z * case["alpha"]
    if st["bias"] is not None:
        z = z + st["bias"]
    c = _act(z, case["act"])
    if st["residual"] is not None:
        c = c + st["residual"].float()
    dt = _DT[case["out"]]
    return [c.to(dt), z.to(dt)] if case["pre"] else [c.to(dt)]


def _plain_linear_backward(st):
    case = st["case"]
    dt = _DT[case["dtype"]]
    dz = st["dC"].float()
    if case["act"]:
        dz = dz * _act_slope(st["pre"].float(), case["act"])
    a, w = st["A"].float(), st["W"].float()
    if case["transB"]:
        da, dw = dz @ w, dz.t() @ a
    else:
        da, dw = dz @ w.t(), a.t() @ dz
    out = [(da * case["alpha"]).to(dt), (dw * case["alpha"]).to(dt)]
    return out + [dz.sum(dim=0)] if case["bias"] else out


def _to_8_bits(y):
    s = (y.abs().amax(dim=1) / _E4M3_MAX).clamp_min(_TINY)
    return [(y / s[:, None]).to(torch.float8_e4m3fn), s]


def _plain_norm(st):
    case = st["case"]
    h = st["x"].float()
    if st["residual"] is not None:
        h = h + st["residual"].float()
    rstd = 1.0 / torch.sqrt((h * h).mean(dim=1) + 1e-6)
    y = h * rstd[:, None]
    if st["gain"] is not None:
        y = y * st["gain"]
    out = _to_8_bits(y) if case["out"] == "e4m3" else [y.to(_DT[case["out"]])]
    out.append(rstd)
    if case["residual"]:
        out.append(h.to(_DT[case["dtype"]]))
    return out


def _plain_norm_backward(st):
    rstd = st["rstd"][:, None]
    xh = st["total"].float() * rstd
    dy = st["dy"].float()
    t = dy * st["gain"] if st["gain"] is not None else dy
    dx = rstd * (t - xh * (t * xh).mean(dim=1, keepdim=True))
    if st["dtotal"] is not None:
        dx = dx + st["dtotal"].float()
    out = [dx.to(st["dx"].dtype)]
    return out + [(dy * xh).sum(dim=0)] if st["gain"] is not None else out


def _plain(st):
    kind = st["case"]["kind"]
    if kind == "linear_backward":
        return _plain_linear_backward(st)
    if kind.startswith("linear"):
        return _plain_linear(st)
    if kind == "norm":
        return _plain_norm(st)
    if kind == "norm_backward":
        return _plain_norm_backward(st)
    return _to_8_bits(st["x"].float())


# ---- the framework's calls -------------------------------------------------------------------------
def _own(st):
    import paper_2210_16691_amd as al
    case = st["case"]
    kind = case["kind"]
    if kind == "linear_backward":
        al.alcop_linear_backward(st["dC"], st["A"], st["W"], dA=st["dA"], dW=st["dW"], dbias=st["dbias"], pre=st["pre"],
                                 act=case["act"], alpha=case["alpha"], transB=case["transB"], workspace=st["ws"])
        return [t for t in (st["dA"], st["dW"], st["dbias"]) if t is not None]
    if kind.startswith("linear"):
        al.alcop_linear(st["A"], st["W"], st["C"], transB=case.get("transB", True), alpha=case["alpha"], bias=st["bias"],
                        act=case["act"], residual=st["residual"], pre=st["pre"], scale_a=st.get("sa"),
                        scale_w=st.get("sw"))
        return [t for t in (st["C"], st["pre"]) if t is not None]
    if kind == "norm":
        al.alcop_rmsnorm(st["x"], st["gain"], st["y"], residual=st["residual"], total=st["total"], scale=st["scale"],
                         rstd=st["rstd"], eps=1e-6)
        return [t for t in (st["y"], st["scale"], st["rstd"], st["total"]) if t is not None]
    if kind == "norm_backward":
        al.alcop_rmsnorm_backward(st["dy"], st["total"], st["gain"], st["rstd"], st["dx"], dgain=st["dgain"],
                                  dtotal=st["dtotal"], workspace=st["ws"])
        return [t for t in (st["dx"], st["dgain"]) if t is not None]
    al.alcop_quantize_rows(st["x"], st["y"], st["scale"])
    return [st["y"], st["scale"]]


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without -----------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind.startswith("linear"):
        M, N, K = case["M"], case["N"], case["K"]
        if kind == "linear_backward":
            s = _SIZE[case["dtype"]]
            # dC and the value in front of the activation, A, W; dA, dW, the bias's gradient
            return {"bytes": s * (M * N * (2 if case["act"] else 1) + 2 * M * K + 2 * N * K) + (4 * N if case["bias"] else 0),
                    "flops": 4 * M * N * K}
        s, o = (1 if kind == "linear8" else _SIZE[case["dtype"]]), _SIZE[case["out"]]
        b = s * (M * K + N * K) + o * M * N * (1 + case["residual"] + case["pre"]) + (4 * N if case["bias"] else 0)
        return {"bytes": b + (4 * (M + N) if kind == "linear8" else 0), "flops": 2 * M * N * K}
    rows, cols, s = case["rows"], case["cols"], _SIZE[case["dtype"]]
    n = rows * cols
    if kind == "quantize":
        return {"bytes": n * (s + 1) + 4 * rows, "flops": 2 * n}
    g = 4 * cols if case["gain"] else 0
    if kind == "norm_backward":
        return {"bytes": n * s * (4 if case["dtotal"] else 3) + 4 * rows + 2 * g, "flops": 9 * n}
    o = _SIZE[case["out"]]
    return {"bytes": n * (s * (3 if case["residual"] else 1) + o) + g + 4 * rows * (2 if o == 1 else 1), "flops": 6 * n}


# ---- the definitions in 64 bits --------------------------------------------------------------------
_ACT64 = {0: lambda z: z, 1: torch.nn.functional.relu, 2: torch.nn.functional.gelu,
          3: lambda z: torch.nn.functional.gelu(z, approximate="tanh"), 4: torch.nn.functional.silu}


def exact(case, seed):
    st = prepare(case, seed)
    d = {k: v.double() if isinstance(v, torch.Tensor) and v.dtype != torch.uint8 else v for k, v in st.items()}
    kind = case["kind"]
    if kind.startswith("linear"):
        w = d["W"].t() if case.get("transB", True) else d["W"]
        if kind == "linear_backward":
            dz = d["dC"]
            if case["act"]:
                z = d["pre"].detach().clone().requires_grad_(True)
                dz, = torch.autograd.grad(_ACT64[case["act"]](z), z, d["dC"])
            dw = case["alpha"] * torch.matmul(d["A"].t(), dz)
            res = [case["alpha"] * torch.matmul(dz, w.t()), dw.t() if case["transB"] else dw]
            return res + [dz.sum(0)] if case["bias"] else res
        a = d["A"]
        if kind == "linear8":
            a, w = a * d["sa"].unsqueeze(1), w * d["sw"]
        z = torch.matmul(a, w) * case["alpha"]
        if case["bias"]:
            z += d["bias"]
        c = _ACT64[case["act"]](z)
        if case["residual"]:
            c = c + d["residual"]
        return [c, z] if case["pre"] else [c]
    if kind == "norm_backward":
        n = case["cols"]
        xh = d["total"] * d["rstd"].unsqueeze(1)
        t = d["dy"] * d["gain"] if case["gain"] else d["dy"]
        dx = (t - xh * ((t * xh).sum(1, keepdim=True) / n)) * d["rstd"].unsqueeze(1)
        if case["dtotal"]:
            dx = dx + d["dtotal"]
        return [dx, torch.einsum("ij,ij->j", d["dy"], xh)] if case["gain"] else [dx]
    y, tail = d["x"], []
    if kind == "norm":
        h = y + d["residual"] if case["residual"] else y
        rstd = (h.pow(2).sum(1) / case["cols"] + 1e-6).pow(-0.5)
        y = h * rstd.unsqueeze(1)
        if case["gain"]:
            y = y * d["gain"]
        tail = [rstd] + ([h] if case["residual"] else [])
        if case["out"] != "e4m3":
            return [y] + tail
    s = torch.clamp(y.abs().max(dim=1).values / _E4M3_MAX, min=_TINY)
    return [y / s.unsqueeze(1), s] + tail
