"""More operators of a transformer in training and serving, beside the linear layers and norms, as timed cases.

Kinds of case:

layernorm           norm of x + residual with its mean taken away, gain and shift; the sum kept as the next residual;
                    the result in the input's type, or in e4m3 with one scale per row
layernorm_backward  its gradients: with respect to the sum (which is that of x and of the residual), gain and shift
grouped             rows sorted by expert, each expert's rows times its own weights (stored N x K or K x N), bias and
                    activation, optionally keeping the value in front of the activation; how many rows an expert
                    has is known on the device only
grouped8            the same on e4m3 operands with a scale per row and one per expert and column
grouped_backward    its gradients: with respect to the rows, each expert's weights and bias
loss                cross entropy of rows against the product with a vocabulary's vectors, logits not kept
loss_backward       its gradients: with respect to the rows and the vocabulary's vectors

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
_EPS = 1e-5


def listed():
    return [
        # the norm in front of one token's product (launch latency)
        dict(name="layernorm_token", kind="layernorm", rows=1, cols=768, dtype="bf16", out="bf16", residual=True, pad=0),
        # the norm of a training batch
        dict(name="layernorm_16384", kind="layernorm", rows=16384, cols=4096, dtype="bf16", out="bf16", residual=True, pad=0),
        # its gradients
        dict(name="layernorm_backward_8192", kind="layernorm_backward", rows=8192, cols=4096, dtype="bf16", dtotal=True, pad=0),
        # gradients at sizes that no chunk divides, rows further apart than they are long
        dict(name="layernorm_backward_ragged", kind="layernorm_backward", rows=1531, cols=1111, dtype="f16", dtotal=False, pad=3),
        # sixteen tokens decoding, two of 32 experts each: the weights of the experts that have a row count
        dict(name="grouped_step_32", kind="grouped", rows=32, groups=32, N=2048, K=1024, dtype="bf16", out="bf16", transB=True,
             act=4, bias=False, pre=False, spread="skewed", behind=0, pad=0),
        # a ragged prompt, a few experts without a row, rows behind the last one (a padded batch)
        dict(name="grouped_ragged", kind="grouped", rows=1531, groups=12, N=1048, K=520, dtype="f16", out="f16", transB=False,
             act=2, bias=True, pre=False, spread="skewed", behind=37, pad=8),
        # the first layer of the experts in training
        dict(name="grouped_train_16384", kind="grouped", rows=16384, groups=16, N=4096, K=2048, dtype="bf16", out="bf16",
             transB=True, act=4, bias=True, pre=True, spread="uneven", behind=0, pad=0),
        # a prompt through 8-bit experts
        dict(name="grouped8_4096", kind="grouped8", rows=4096, groups=8, N=2048, K=4096, out="bf16", act=0, bias=False,
             pre=False, spread="uneven", behind=0, pad=0),
        # the gradients of such a layer
        dict(name="grouped_backward_8192", kind="grouped_backward", rows=8192, groups=16, N=2048, K=2048, dtype="bf16",
             transB=True, act=4, bias=True, spread="uneven", behind=0, pad=0),
        # the loss of a short text against an odd vocabulary
        dict(name="loss_ragged", kind="loss", rows=509, vocab=30011, K=768, dtype="f16", ignored=True, alpha=1.0, pad=8),
        # the loss of a training batch against a large vocabulary
        dict(name="loss_8192", kind="loss", rows=8192, vocab=65536, K=2048, dtype="bf16", ignored=False, alpha=1.0, pad=0),
        # its gradients, the largest call
        dict(name="loss_backward_4096", kind="loss_backward", rows=4096, vocab=65536, K=2048, dtype="bf16", ignored=True,
             alpha=1.0, pad=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["layernorm", "layernorm", "layernorm_backward", "grouped", "grouped", "grouped8", "grouped_backward",
                       "loss", "loss_backward"])
    if kind.startswith("layernorm"):
        while True:
            rows, cols = _log_int(rng, 1, 16384), _log_int(rng, 64, 16384)
            if rows * cols <= 2 ** 26:
                break
        if rng.random() < 0.6:
            cols = max(64, cols // 8 * 8)
        case = dict(kind=kind, rows=rows, cols=cols, dtype=rng.choice(["f16", "bf16", "bf16", "f32"]), pad=rng.choice([0, 0, 8, 3]))
        if kind == "layernorm":
            case.update(out=rng.choice([case["dtype"], case["dtype"], "e4m3"]), residual=rng.random() < 0.7)
        else:
            case.update(dtotal=rng.random() < 0.7)
        return case
    if kind.startswith("grouped"):
        unit = 16 if kind == "grouped8" else 8
        while True:
            rows, groups = _log_int(rng, 1, 16384), _log_int(rng, 1, 64)
            N = max(64, _log_int(rng, 64, 4096) // 8 * 8)
            K = max(64, _log_int(rng, 64, 4096) // unit * unit)
            if rows * N * K <= 2 ** 36 and groups * N * K <= 2 ** 28:
                break
        case = dict(kind=kind, rows=rows, groups=groups, N=N, K=K, act=rng.randrange(5), bias=rng.random() < 0.5,
                    spread=rng.choice(["uneven", "skewed", "one"]), behind=rng.choice([0, 0, rows // 7]),
                    pad=rng.choice([0, 0, unit, 3 * unit]))
        if kind == "grouped8":
            case.update(out=rng.choice(["f16", "bf16", "bf16", "f32"]), pre=rng.random() < 0.3)
        else:
            case.update(dtype=rng.choice(["f16", "bf16"]), transB=rng.random() < 0.6)
        if kind == "grouped":
            case.update(out=rng.choice([case["dtype"], case["dtype"], "f32"]), pre=rng.random() < 0.3)
        if kind != "grouped_backward" and case.get("transB", True) and rng.random() < 0.25:
            case["N"] = N - rng.randrange(1, 8)          # rows of weights need not be a multiple of anything
        return case
    while True:
        rows, vocab = _log_int(rng, 1, 8192), _log_int(rng, 100, 131072)
        K = max(64, _log_int(rng, 64, 4096) // 8 * 8)
        if rows * vocab * K <= 2 ** 38 and vocab * K <= 2 ** 28:
            break
    return dict(kind=kind, rows=rows, vocab=vocab, K=K, dtype=rng.choice(["f16", "bf16"]), ignored=rng.random() < 0.5,
                alpha=rng.choice([1.0, 1.0, 0.5]), pad=rng.choice([0, 0, 8, 24]))


# ---- inputs --------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 6971 + 29)
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


def _zeros(rows, cols, pad, dtype):
    return torch.zeros(rows, cols + pad, device="cuda", dtype=_DT[dtype])[:, :cols]


def _by_group(m, groups):
    """A matrix of groups * n rows as groups of n rows."""
    return m.as_strided((groups, m.shape[0] // groups, m.shape[1]), (m.shape[0] // groups * m.stride(0), m.stride(0), 1))


def _sizes(case, seed):
    """Rows of each expert: near even, a few experts with most of the rows and some with none, or one with all."""
    g = torch.Generator().manual_seed(seed * 271 + 5)
    n, rows = case["groups"], case["rows"] - case["behind"]
    if case["spread"] == "one":
        sizes = [0] * n
        sizes[int(torch.randint(n, (1,), generator=g))] = rows
        return sizes
    weight = torch.rand(n, generator=g) + 0.5 if case["spread"] == "uneven" else torch.rand(n, generator=g) ** 3 + 1e-6
    pick = torch.multinomial(weight, rows, replacement=True, generator=g)
    return torch.bincount(pick, minlength=n).tolist()


def prepare(case, seed):
    g = _generator(seed)
    kind, pad = case["kind"], case["pad"]
    st = {"case": case}
    if kind.startswith("layernorm"):
        rows, cols, dtype = case["rows"], case["cols"], case["dtype"]
        if kind == "layernorm_backward":
            st["dy"] = _matrix(g, rows, cols, pad, dtype, scale=0.5)
            st["total"] = _matrix(g, rows, cols, pad, dtype, scale=2.0, outliers=True)
            d = st["total"].double()
            st["mean"] = d.mean(dim=1).float()
            st["rstd"] = (d.var(dim=1, unbiased=False) + _EPS).rsqrt().float()
            st["dtotal"] = _matrix(g, rows, cols, pad, dtype) if case["dtotal"] else None
            st["dx"] = _zeros(rows, cols, pad, dtype)
            st["dgain"], st["dshift"] = torch.zeros(cols, device="cuda"), torch.zeros(cols, device="cuda")
            if own:
                import paper_2210_16691_amd as al
                st["ws"] = torch.empty(al.alcop_layernorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
        else:
            st["x"] = _matrix(g, rows, cols, pad, dtype, outliers=True)
            st["residual"] = _matrix(g, rows, cols, pad, dtype, scale=2.0) if case["residual"] else None
            st["total"] = _zeros(rows, cols, pad, dtype) if case["residual"] else None
            st["y"] = _zeros(rows, cols, pad, case["out"])
            st["scale"] = torch.zeros(rows, device="cuda") if case["out"] == "e4m3" else None
            st["mean"], st["rstd"] = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
            st["shift"] = 0.1 * torch.randn(cols, generator=g, device="cuda")
        st["gain"] = 1.0 + 0.2 * torch.randn(cols, generator=g, device="cuda")
        return st
    if kind.startswith("grouped"):
        rows, G, N, K = case["rows"], case["groups"], case["N"], case["K"]
        tb = case.get("transB", True)
        w_rows, w_cols = (N, K) if tb else (K, N)
        st["sizes"] = _sizes(case, seed)
        ends = torch.tensor([0] + st["sizes"]).cumsum(0)
        st["ends"] = ends.tolist()
        st["offsets"] = ends.to(torch.int32).cuda()
        if kind == "grouped8":
            st["A"], st["sa"] = _matrix8(g, rows, K, pad, outliers=True)
            w, sw = _matrix8(g, G * N, K, pad, scale=K ** -0.5)
            st["sw"] = sw.view(G, N)
            out = case["out"]
        else:
            st["A"] = _matrix(g, rows, K, pad, case["dtype"], outliers=True)
            w = _matrix(g, G * w_rows, w_cols, pad, case["dtype"], scale=K ** -0.5)
            out = case.get("out", case["dtype"])
        st["W"] = _by_group(w, G)
        st["bias"] = torch.randn(G, N, generator=g, device="cuda") * 0.5 if case["bias"] else None
        if kind == "grouped_backward":
            st["dC"] = _matrix(g, rows, N, pad, case["dtype"], scale=0.5)
            st["pre"] = _matrix(g, rows, N, pad, case["dtype"], scale=1.5) if case["act"] else None
            st["dA"] = _zeros(rows, K, pad, case["dtype"])
            st["dW"] = _by_group(_zeros(G * w_rows, w_cols, pad, case["dtype"]), G)
            st["dbias"] = torch.zeros(G, N, device="cuda") if case["bias"] else None
            if own:
                import paper_2210_16691_amd as al
                st["ws"] = torch.empty(al.alcop_grouped_linear_backward_workspace_bytes(rows, G, N, K), dtype=torch.uint8,
                                       device="cuda")
        else:
            st["C"] = _zeros(rows, N, pad, out)
            st["pre"] = _zeros(rows, N, pad, out) if case["pre"] else None
        return st
    rows, V, K = case["rows"], case["vocab"], case["K"]
    st["X"] = _matrix(g, rows, K, pad, case["dtype"])
    st["W"] = _matrix(g, V, K, pad, case["dtype"], scale=2.0 * K ** -0.5)
    labels = torch.randint(0, V, (rows,), generator=g, device="cuda")
    if case["ignored"]:
        labels[torch.rand(rows, generator=g, device="cuda") < 0.1] = -100
    st["labels"] = labels
    if kind == "loss_backward":
        st["dloss"] = (1.0 + torch.rand(rows, generator=g, device="cuda")) / rows
        st["lse"] = torch.cat([torch.logsumexp((x.float() @ st["W"].float().t()) * case["alpha"], dim=1)
                               for x in st["X"].split(2048)])
        st["dX"] = _zeros(rows, K, pad, case["dtype"])
        st["dW"] = _zeros(V, K, pad, case["dtype"])
        if own:
            import paper_2210_16691_amd as al
            st["ws"] = torch.empty(al.alcop_linear_cross_entropy_backward_workspace_bytes(rows, V, K), dtype=torch.uint8,
                                   device="cuda")
    else:
        st["loss"], st["lse"] = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
        if own:
            import paper_2210_16691_amd as al
            st["ws"] = torch.empty(al.alcop_linear_cross_entropy_workspace_bytes(rows, V, K), dtype=torch.uint8, device="cuda")
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


def _plain_layernorm(st):
    case = st["case"]
    h = st["x"].float()
    if case["residual"]:
        h = h + st["residual"].float()
    mean = h.mean(dim=1)
    d = h - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).mean(dim=1) + _EPS)
    y = d * rstd[:, None] * st["gain"] + st["shift"]
    if case["out"] == "e4m3":
        s = (y.abs().amax(dim=1) / _E4M3_MAX).clamp_min(_TINY)
        q = (y / s[:, None]).to(torch.float8_e4m3fn)
        out = [q.float() * s[:, None], s]
    else:
        out = [y.to(_DT[case["out"]])]
    out += [mean, rstd]
    return out + [h.to(_DT[case["dtype"]])] if case["residual"] else out


def _plain_layernorm_backward(st):
    rstd = st["rstd"][:, None]
    xh = (st["total"].float() - st["mean"][:, None]) * rstd
    dy = st["dy"].float()
    t = dy * st["gain"]
    dx = rstd * (t - t.mean(dim=1, keepdim=True) - xh * (t * xh).mean(dim=1, keepdim=True))
    if st["dtotal"] is not None:
        dx = dx + st["dtotal"].float()
    return [dx.to(st["dx"].dtype), (dy * xh).sum(dim=0), dy.sum(dim=0)]


def _plain_grouped(st):
    case = st["case"]
    tb = case.get("transB", True)
    dt = _DT[case["out"]]
    z = torch.zeros(case["rows"], case["N"], device="cuda")
    c = torch.zeros_like(z)
    for e, size in enumerate(st["sizes"]):
        if not size:
            continue
        lo, hi = st["ends"][e], st["ends"][e + 1]
        w = st["W"][e].float()
        p = st["A"][lo:hi].float() @ (w.t() if tb else w)
        if "sa" in st:
            p = p * st["sa"][lo:hi, None] * st["sw"][e]
        if st["bias"] is not None:
            p = p + st["bias"][e]
        z[lo:hi] = p
        c[lo:hi] = _act(p, case["act"])
    return [c.to(dt), z.to(dt)] if case["pre"] else [c.to(dt)]


def _plain_grouped_backward(st):
    case = st["case"]
    dt = _DT[case["dtype"]]
    da = torch.zeros(case["rows"], case["K"], device="cuda")
    dw = torch.zeros(st["W"].shape, device="cuda")
    db = torch.zeros(case["groups"], case["N"], device="cuda")
    for e, size in enumerate(st["sizes"]):
        if not size:
            continue
        lo, hi = st["ends"][e], st["ends"][e + 1]
        dz = st["dC"][lo:hi].float()
        if case["act"]:
            dz = dz * _act_slope(st["pre"][lo:hi].float(), case["act"])
        a, w = st["A"][lo:hi].float(), st["W"][e].float()
        if case["transB"]:
            da[lo:hi], dw[e] = dz @ w, dz.t() @ a
        else:
            da[lo:hi], dw[e] = dz @ w.t(), a.t() @ dz
        db[e] = dz.sum(dim=0)
    out = [da.to(dt), dw.to(dt)]
    return out + [db] if case["bias"] else out


def _plain_loss(st):
    z = (st["X"].float() @ st["W"].float().t()) * st["case"]["alpha"]
    top = z.amax(dim=1, keepdim=True)
    lse = torch.log(torch.exp(z - top).sum(dim=1)) + top[:, 0]
    y = st["labels"]
    there = y >= 0
    hit = z.gather(1, torch.where(there, y, torch.zeros_like(y))[:, None])[:, 0]
    return [torch.where(there, lse - hit, torch.zeros_like(lse)), lse]


def _plain_loss_backward(st):
    case = st["case"]
    x, w = st["X"].float(), st["W"].float()
    y = st["labels"]
    there = (y >= 0).float()
    p = torch.exp((x @ w.t()) * case["alpha"] - st["lse"][:, None])
    p.scatter_add_(1, torch.where(y >= 0, y, torch.zeros_like(y))[:, None], -there[:, None])
    p *= (st["dloss"] * there * case["alpha"])[:, None]
    dt = _DT[case["dtype"]]
    return [(p @ w).to(dt), (p.t() @ x).to(dt)]


_PLAIN = {"layernorm": _plain_layernorm, "layernorm_backward": _plain_layernorm_backward, "grouped": _plain_grouped,
          "grouped8": _plain_grouped, "grouped_backward": _plain_grouped_backward, "loss": _plain_loss,
          "loss_backward": _plain_loss_backward}


# ---- the framework's calls -------------------------------------------------------------------------
def _own(st):
    import paper_2210_16691_amd as al
    case = st["case"]
    kind = case["kind"]
    if kind == "layernorm":
        al.alcop_layernorm(st["x"], st["gain"], st["shift"], st["y"], residual=st["residual"], total=st["total"],
                           scale=st["scale"], mean=st["mean"], rstd=st["rstd"], eps=_EPS)
        if case["out"] == "e4m3":
            out = [st["y"].float() * st["scale"][:, None], st["scale"]]
        else:
            out = [st["y"]]
        out += [st["mean"], st["rstd"]]
        return out + [st["total"]] if case["residual"] else out
    if kind == "layernorm_backward":
        al.alcop_layernorm_backward(st["dy"], st["total"], st["gain"], st["mean"], st["rstd"], st["dx"], dgain=st["dgain"],
                                    dshift=st["dshift"], dtotal=st["dtotal"], workspace=st["ws"])
        return [st["dx"], st["dgain"], st["dshift"]]
    if kind == "grouped_backward":
        al.alcop_grouped_linear_backward(st["dC"], st["A"], st["W"], st["offsets"], dA=st["dA"], dW=st["dW"], dbias=st["dbias"],
                                         pre=st["pre"], act=case["act"], transB=case["transB"], workspace=st["ws"])
        return [t for t in (st["dA"], st["dW"], st["dbias"]) if t is not None]
    if kind.startswith("grouped"):
        al.alcop_grouped_linear(st["A"], st["W"], st["offsets"], st["C"], transB=case.get("transB", True), bias=st["bias"],
                                act=case["act"], pre=st["pre"], scale_a=st.get("sa"), scale_w=st.get("sw"))
        return [t for t in (st["C"], st["pre"]) if t is not None]
    if kind == "loss":
        al.alcop_linear_cross_entropy(st["X"], st["W"], st["labels"], st["loss"], st["lse"], st["ws"], alpha=case["alpha"])
        return [st["loss"], st["lse"]]
    al.alcop_linear_cross_entropy_backward(st["X"], st["W"], st["labels"], st["lse"], st["ws"], dX=st["dX"], dW=st["dW"],
                                           dloss=st["dloss"], alpha=case["alpha"])
    return [st["dX"], st["dW"]]


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["kind"]](state)


# ---- what a pass cannot do without -----------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind.startswith("layernorm"):
        rows, cols, s = case["rows"], case["cols"], _SIZE[case["dtype"]]
        n = rows * cols
        if kind == "layernorm_backward":
            # dy, the sum, dtotal, dx; mean and rstd; gain, its gradient, the shift's
            return {"bytes": n * s * (4 if case["dtotal"] else 3) + 8 * rows + 12 * cols, "flops": 12 * n}
        o = _SIZE[case["out"]]
        return {"bytes": n * (s * (3 if case["residual"] else 1) + o) + 8 * cols + 4 * rows * (3 if o == 1 else 2), "flops": 8 * n}
    if kind.startswith("grouped"):
        rows, G, N, K = case["rows"] - case["behind"], case["groups"], case["N"], case["K"]
        # experts that may have a row, weights of the others are not read
        live = 1 if case["spread"] == "one" else min(G, rows)
        if kind == "grouped_backward":
            s = _SIZE[case["dtype"]]
            b = s * (rows * N * (2 if case["act"] else 1) + 2 * rows * K + live * N * K + G * N * K)
            return {"bytes": b + (4 * G * N if case["bias"] else 0), "flops": 4 * rows * N * K}
        s, o = (1 if kind == "grouped8" else _SIZE[case["dtype"]]), _SIZE[case["out"]]
        b = s * (rows * K + live * N * K) + o * rows * N * (1 + case["pre"]) + (4 * live * N if case["bias"] else 0)
        return {"bytes": b + (4 * (rows + live * N) if kind == "grouped8" else 0), "flops": 2 * rows * N * K}
    rows, V, K = case["rows"], case["vocab"], case["K"]
    if kind == "loss":
        return {"bytes": 2 * (rows * K + V * K) + 16 * rows, "flops": 2 * rows * V * K}
    return {"bytes": 4 * (rows * K + V * K) + 16 * rows, "flops": 6 * rows * V * K}


# ---- the definitions in 64 bits --------------------------------------------------------------------
_ACT64 = {0: lambda z: z, 1: torch.nn.functional.relu, 2: torch.nn.functional.gelu,
          3: lambda z: torch.nn.functional.gelu(z, approximate="tanh"), 4: torch.nn.functional.silu}


def _exact_layernorm(st, case):
    h = st["x"].double()
    if case["residual"]:
        h = h + st["residual"].double()
    var, mean = torch.var_mean(h, dim=1, unbiased=False)
    rstd = (var + _EPS).pow(-0.5)
    y = torch.addcmul(st["shift"].double(), (h - mean.unsqueeze(1)) * rstd.unsqueeze(1), st["gain"].double())
    if case["out"] == "e4m3":
        y = [None, torch.clamp(y.abs().max(dim=1).values / _E4M3_MAX, min=_TINY)]    # 8 bits have no value between their steps
    else:
        y = [y]
    return y + [mean, rstd] + ([h] if case["residual"] else [])


def _exact_layernorm_backward(st, case):
    n = case["cols"]
    dy, r = st["dy"].double(), st["rstd"].double().unsqueeze(1)
    xh = (st["total"].double() - st["mean"].double().unsqueeze(1)) * r
    t = dy * st["gain"].double()
    dx = (t - (t.sum(1, keepdim=True) + xh * (t * xh).sum(1, keepdim=True)) / n) * r
    if case["dtotal"]:
        dx = dx + st["dtotal"].double()
    return [dx, torch.einsum("ij,ij->j", dy, xh), dy.sum(0)]


def _exact_grouped(st, case):
    tb, backward = case.get("transB", True), case["kind"] == "grouped_backward"
    left = torch.zeros(case["rows"], case["K"] if backward else case["N"], dtype=torch.float64, device="cuda")
    pre = torch.zeros_like(left)
    dws, dbs = [], []
    first = 0
    for e, size in enumerate(st["sizes"]):
        part = slice(first, first + size)
        first += size
        w = st["W"][e].double()
        w = w.t() if tb else w                       # K x N
        a = st["A"][part].double()
        if backward:
            dz = st["dC"][part].double()
            if case["act"]:
                z = st["pre"][part].double().requires_grad_(True)
                dz, = torch.autograd.grad(_ACT64[case["act"]](z), z, dz)
            left[part] = torch.matmul(dz, w.t())
            dw = torch.matmul(a.t(), dz)
            dws.append(dw.t() if tb else dw)
            dbs.append(dz.sum(0))
            continue
        if case["kind"] == "grouped8":
            a, w = a * st["sa"][part].double().unsqueeze(1), w * st["sw"][e].double()
        z = torch.matmul(a, w)
        if case["bias"]:
            z = z + st["bias"][e].double()
        pre[part] = z
        left[part] = _ACT64[case["act"]](z)
    if backward:
        return [left, torch.stack(dws)] + ([torch.stack(dbs)] if case["bias"] else [])
    return [left, pre] if case["pre"] else [left]


def _exact_loss(st, case):
    w, losses, lses = st["W"].double(), [], []
    for x, y in zip(st["X"].split(1024), st["labels"].split(1024)):
        z = torch.matmul(x.double(), w.t()) * case["alpha"]
        losses.append(torch.nn.functional.cross_entropy(z, y, reduction="none", ignore_index=-100))
        lses.append(torch.logsumexp(z, dim=1))
    return [torch.cat(losses), torch.cat(lses)]


def _exact_loss_backward(st, case):
    w, dxs = st["W"].double(), []
    dw = torch.zeros_like(w)
    for x, y, lse, d in zip(*(st[k].split(1024) for k in ("X", "labels", "lse", "dloss"))):
        x = x.double()
        q = torch.exp(torch.matmul(x, w.t()) * case["alpha"] - lse.double().unsqueeze(1))
        at = torch.nonzero(y != -100)[:, 0]
        q[at, y[at]] -= 1.0
        q *= torch.where(y != -100, d.double(), 0.0).unsqueeze(1) * case["alpha"]
        dxs.append(torch.matmul(q, w))
        dw += torch.matmul(q.t(), x)
    return [torch.cat(dxs), dw]


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "layernorm":
        return _exact_layernorm(st, case)
    if kind == "layernorm_backward":
        return _exact_layernorm_backward(st, case)
    if kind == "loss":
        return _exact_loss(st, case)
    if kind == "loss_backward":
        return _exact_loss_backward(st, case)
    return _exact_grouped(st, case)
