"""A transformer's experts between two norms, and the loss behind them, forward and backward out of the operators, every result checked
against its formula in 64 bits on the inputs that it was given."""
import torch

import paper_2210_16691_amd as al
from layers_util import HALF, ULP, check
from more_util import grouped64, grouped_grad64, layernorm64, layernorm_grad64, loss64, loss_grad64


def run_block(call, dev, dtype, rows, dim, hidden, sizes, vocab, seed=0, behind=0):
    """call(fn, *args, **kw): runs fn so that its results are there on return."""
    g = torch.Generator().manual_seed(seed)
    t = lambda *s, scale=1.0, to=dtype: (torch.randn(*s, generator=g) * scale).to(to).to(dev)
    f32 = torch.float32
    G, n = len(sizes), rows - behind
    assert sum(sizes) == n
    offs = torch.tensor([0] + sizes).cumsum(0).to(torch.int32).to(dev)
    x, r = t(rows, dim), t(rows, dim)
    g1, b1, g2, b2 = t(dim, to=f32), t(dim, to=f32), t(dim, to=f32), t(dim, to=f32)
    W1, W2 = t(G, hidden, dim, scale=dim ** -0.5), t(G, dim, hidden, scale=hidden ** -0.5)
    bias1, route = t(G, hidden, to=f32), t(rows, to=f32).abs()
    voc = t(vocab, dim, scale=dim ** -0.5)
    labels = torch.randint(0, vocab, (rows,), generator=g)
    labels[::7] = -100
    labels = labels.to(dev)
    new = lambda *s, to=dtype: torch.zeros(*s, dtype=to, device=dev)
    byte = lambda k: torch.zeros(k, dtype=torch.uint8, device=dev)
    part = slice(0, n)

    # forward: norm(x + r) -> experts (up, SiLU; down, weighted by the router) -> norm(their sum with the residual) -> loss
    s1, y1, m1, d1 = new(rows, dim), new(rows, dim), new(rows, to=f32), new(rows, to=f32)
    call(al.alcop_layernorm, x, g1, b1, y1, residual=r, total=s1, mean=m1, rstd=d1)
    ref = layernorm64(x, r, g1, b1)
    check(y1, ref[0], ref[4], "norm")
    check(s1, ref[1], ULP * ref[1].abs(), "sum")
    up, pre = new(rows, hidden), new(rows, hidden)
    call(al.alcop_grouped_linear, y1, W1, offs, up, transB=True, bias=bias1, act=4, pre=pre)
    c, z, ez, ec = grouped64(y1, W1, sizes, 0, True, 1.0, bias1, 4)
    check(up[part], c[part], ec[part], "up")
    check(pre[part], z[part], ez[part], "pre")
    down = new(rows, dim)
    call(al.alcop_grouped_linear, up, W2, offs, down, transB=True, scale_a=route)
    c, _, _, ec = grouped64(up, W2, sizes, 0, True, sa=route)
    check(down[part], c[part], ec[part], "down")
    assert not down[n:].any()
    s2, y2, m2, d2 = new(rows, dim), new(rows, dim), new(rows, to=f32), new(rows, to=f32)
    call(al.alcop_layernorm, down, g2, b2, y2, residual=s1, total=s2, mean=m2, rstd=d2)
    ref = layernorm64(down, s1, g2, b2)
    check(y2, ref[0], ref[4], "second norm")
    loss, lse = new(rows, to=f32), new(rows, to=f32)
    call(al.alcop_linear_cross_entropy, y2, voc, labels, loss, lse, byte(al.alcop_linear_cross_entropy_workspace_bytes(rows, vocab, dim)))
    ref = loss64(y2, voc, labels)
    check(loss[None], ref[0][None], ref[2][None], "loss")

    # backward
    dloss = new(rows, to=f32) + 1.0 / rows
    dy2, dvoc = new(rows, dim), new(vocab, dim)
    call(al.alcop_linear_cross_entropy_backward, y2, voc, labels, lse, byte(al.alcop_linear_cross_entropy_backward_workspace_bytes(rows, vocab, dim)),
         dX=dy2, dW=dvoc, dloss=dloss)
    rx, rw, ex, ew = loss_grad64(y2, voc, labels, lse, dloss)
    check(dy2, rx, ex, "gradient of the loss")
    check(dvoc, rw, ew, "gradient of the vocabulary")
    ds2, dg2, db2 = new(rows, dim), new(dim, to=f32), new(dim, to=f32)
    wn = byte(al.alcop_layernorm_backward_workspace_bytes(rows, dim))
    call(al.alcop_layernorm_backward, dy2, s2, g2, m2, d2, ds2, dgain=dg2, dshift=db2, workspace=wn)
    rx, rg, rb, ex, eg, eb = layernorm_grad64(dy2, s2, g2, m2, d2)
    check(ds2, rx, ex, "gradient of the second norm")
    check(dg2[None], rg[None], eg[None], "dgain")
    check(db2[None], rb[None], eb[None], "dshift")
    # what the router weighs a row's result with, it weighs its gradient with
    ddown = (ds2.float() * route[:, None]).to(dtype)
    dup, dW2 = new(rows, hidden), new(G, dim, hidden)
    call(al.alcop_grouped_linear_backward, ddown, up, W2, offs, dA=dup, dW=dW2, transB=True)
    ra, rw, _, ea, ew, _ = grouped_grad64(ddown, up, W2, sizes, 0, True)
    check(dup[part], ra[part], ea[part], "gradient of up")
    for e in range(G):
        check(dW2[e], rw[e], ew[e], "gradient of the experts' second weights")
    dy1, dW1, dbias1 = new(rows, dim), new(G, hidden, dim), new(G, hidden, to=f32)
    call(al.alcop_grouped_linear_backward, dup, y1, W1, offs, dA=dy1, dW=dW1, dbias=dbias1, pre=pre, act=4, transB=True,
         workspace=byte(al.alcop_grouped_linear_backward_workspace_bytes(rows, G, hidden, dim)))
    ra, rw, rb, ea, ew, eb = grouped_grad64(dup, y1, W1, sizes, 0, True, pre, 4)
    check(dy1[part], ra[part], ea[part], "gradient of the first norm's result")
    for e in range(G):
        check(dW1[e], rw[e], ew[e], "gradient of the experts' first weights")
    check(dbias1, rb, eb, "gradient of the biases")
    assert not dy1[n:].any()
    dx, dg1, db1 = new(rows, dim), new(dim, to=f32), new(dim, to=f32)
    call(al.alcop_layernorm_backward, dy1, s1, g1, m1, d1, dx, dgain=dg1, dshift=db1, dtotal=ds2, workspace=wn)
    rx, rg, rb, ex, eg, eb = layernorm_grad64(dy1, s1, g1, m1, d1, ds2)
    check(dx, rx, ex, "gradient of x")
    check(dg1[None], rg[None], eg[None], "dgain")
    check(db1[None], rb[None], eb[None], "dshift")
    return [x, y1, up, down, y2, loss, dy2, dvoc, ds2, dup, dW2, dy1, dW1, dbias1, dx, dg1, db1]
