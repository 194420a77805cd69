"""A training step of clients' blocks with the normalisation, the layer of 4-bit values, the orthogonalised update and the message, as they
follow one another, against the same step in 64 bits: x + r, its normalised rows, quantised, through W (held in 4 bits) and GELU, the gradient
back to x and r, the update of the weights that W was quantised from, and the message of what it moved by."""
import pytest
import torch

import mx4_oracle as M
import ops_oracle as O
from test_gpu_ops_linear import TYPES, d64, ops, rand  # noqa: F401
from test_gpu_ops_layer_norm import backward as norm_backward, forward as norm_forward
from test_gpu_ops_orthogonal import MUON, definition

pytestmark = pytest.mark.gpu


def step(ops, x, r, gamma, beta, w, dy, rate):   # noqa: F811
    """One step; everything that it makes."""
    y, h, mean, rstd = ops.aet_layer_norm_forward(x, gamma, beta, residual=r)
    q, qs = ops.aet_mx4_quantise(y)
    held, held_s = ops.aet_mx4_quantise(w)
    cols = x.shape[-1]
    z, pre = ops.aet_mx4_linear_forward(q, qs, held, held_s, cols=cols, act="gelu", keep_pre=True, dtype=x.dtype)
    dq, dw, _ = ops.aet_mx4_linear_backward(dy, q, qs, held, held_s, pre, cols=cols, act="gelu")
    dx, dgamma, dbeta = ops.aet_layer_norm_backward(dq, h, mean, rstd, gamma, dh=x)   # (x stands for what comes along the stream)
    new = ops.aet_orthogonalise(dw, w=w, keep=0.99, scale=-rate)
    c, s = ops.aet_mx4_quantise(new - w)
    moved = ops.aet_mx4_dequantise(c, s, cols=cols, dtype=x.dtype)
    return dict(y=y, h=h, mean=mean, rstd=rstd, q=q, qs=qs, held=held, held_s=held_s, z=z, pre=pre, dq=dq, dw=dw, dx=dx, dgamma=dgamma, dbeta=dbeta, new=new,
                c=c, s=s, moved=moved)


def inputs(dtype, size):
    n, rows, cols, out = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(out)
    return (rand(g, (n, rows, cols), dt), rand(g, (n, rows, cols), dt), rand(g, (n, cols), dt), rand(g, (n, cols), dt), rand(g, (n, out, cols), dt, cols ** -0.5),
            rand(g, (n, rows, out), dt, 0.1))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(3, 40, 72, 130), (1, 300, 515, 96), (4, 16, 784, 128)], ids=str)
def test_a_step(ops, size, dtype):   # noqa: F811
    """Each operator against 64 bits on what the one before it made (a rounding to 4 bits on its way would hide the others')."""
    n, rows, cols, out = size
    dt = TYPES[dtype]
    x, r, gamma, beta, w, dy = inputs(dtype, size)
    t = step(ops, x, r, gamma, beta, w, dy, 0.02)
    wy, wh, _, _ = norm_forward(d64(x), d64(r), d64(gamma), d64(beta), 1e-5, dt)
    O.near(t["y"], wy, "y")
    O.near(t["h"], wh, "h")
    for codes, scales, v in ((t["q"], t["qs"], t["y"]), (t["held"], t["held_s"], w), (t["c"], t["s"], t["new"] - w)):
        wc, ws = M.quantise(d64(v).reshape(-1, cols))
        assert torch.equal(codes.cpu().reshape(wc.shape), wc) and torch.equal(scales.cpu().reshape(ws.shape), ws)
    vx, vw = M.values(t["q"], t["qs"], cols), M.values(t["held"], t["held_s"], cols)
    wz, wp = O.linear_forward(vx, vw, None, None, "gelu", 0.0, 0, 0, dt)
    O.near(t["z"], wz, "z")
    O.near(t["pre"], wp, "pre")
    dq, dw, _ = O.linear_backward(d64(dy), vx, vw, d64(t["pre"]), "gelu", 0.0, 0, 0, dt)
    O.near(t["dq"], dq, "dq")
    O.near(t["dw"], dw, "dw")
    for got, want, what in zip((t["dx"], t["dgamma"], t["dbeta"]),
                               norm_backward(d64(t["dq"]), d64(t["h"]), d64(t["mean"]), d64(t["rstd"]), d64(gamma), d64(x), dt), ("dx", "dgamma", "dbeta")):
        O.near(got, want, what)
    want = 0.99 * d64(w) - 0.02 * definition(d64(t["dw"]), 5, MUON)
    # the update is within 1e-4 of its norm (see the operator's own test), and the sum is rounded once
    assert float((d64(t["new"]) - want).norm()) <= 1e-4 * 0.02 * float(definition(d64(t["dw"]), 5, MUON).norm()) + O.ROUND[dt] * float(want.norm())
    assert torch.equal(d64(t["moved"]), M.values(t["c"], t["s"], cols))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_step_captured(ops, dtype):   # noqa: F811
    """Two graphs of it over the same tensors, replayed in turn with eager steps between: every replay is the eager step."""
    args = inputs(dtype, (2, 130, 264, 200))
    step(ops, *args, 0.02)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(step(ops, *args, 0.02))
    g = torch.Generator().manual_seed(1)
    for k in range(3):
        args[0].copy_(rand(g, args[0].shape, args[0].dtype))
        args[5].copy_(rand(g, args[5].shape, args[5].dtype))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = step(ops, *args, 0.02)
        for out in outs:
            for name in want:
                assert torch.equal(out[name], want[name]), (k, name)


def test_two_streams_at_once(ops):   # noqa: F811
    """Steps of two sets of clients side by side, each with workspaces of its own."""
    sets = [inputs("bf16", (2, 130, 264, 200)), inputs("bf16", (1, 300, 515, 96))]
    want = [step(ops, *a, 0.02) for a in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        got = []
        for a, s in zip(sets, streams):
            with torch.cuda.stream(s):
                got.append(step(ops, *a, 0.02))
    torch.cuda.synchronize()
    for w, o in zip(want, got):
        for name in w:
            assert torch.equal(w[name], o[name]), name
