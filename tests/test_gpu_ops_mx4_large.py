"""The linear layer of 4-bit values and its gradient at sizes that take the larger tiles and split sums, ragged each way, against 64 bits."""
import pytest
import torch

import mx4_oracle as M
import ops_oracle as O
from test_gpu_ops_linear import DEV, TYPES, d64, ops, rand  # noqa: F401
from test_gpu_ops_mx4 import held

pytestmark = pytest.mark.gpu


def products(a, b):
    """a b^T, and the same of the magnitudes; on the GPU, for the time that it takes."""
    a, b = a.to(DEV), b.to(DEV).transpose(-1, -2).contiguous()
    return torch.matmul(a, b), torch.matmul(a.abs(), b.abs())


def forward(vx, vw, bias, residual, name, p, seed, first_row, dt):
    """(y, bound), (pre, bound), as the oracle has them."""
    z, S = (t.cpu() for t in products(vx, vw))
    z, S = z + bias[:, None], S + bias.abs()[:, None]
    off = (vx.shape[-1] + 4) * O.U32 * S
    m, r = O.mask3(z.shape, seed, first_row, p), O.ROUND[dt]
    y = O.act(z, name) * m
    yoff = (1.13 * off + (8 * O.U32 * (z.abs() + 1) if name in ("silu", "gelu") else 0) + 2 * O.U32 * z.abs()) * m
    y = y + residual
    yoff = yoff + 2 * O.U32 * (y.abs() + residual.abs())
    return (y, yoff + r * (y.abs() + yoff)), (z, off + r * (z.abs() + off))


# n, rows, in, out.  Tiles of 256: in one piece, the scales' places used a second time, two parts of 15 and four of 10 units of 512 k; of 128: in
# one piece, 2, 4 and 16 parts; of 64: parts of 2, 3, 4 and 7 units.  Sums of whole units lie as the tiles read them, others are copied.
FORWARD = [(1, 3000, 1000, 4100), (1, 3000, 1024, 4100), (1, 2999, 2600, 4100), (3, 342, 15019, 3628), (3, 144, 19169, 2774),
           (1, 1500, 600, 2000), (2, 1500, 2900, 1001), (3, 2810, 5737, 66), (1, 65, 6780, 4184), (3, 69, 17146, 322),
           (1, 64, 8192, 64), (1, 130, 10240, 500), (1, 500, 16384, 500), (3, 324, 6204, 431)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", FORWARD, ids=str)
def test_forward(ops, size, dtype):   # noqa: F811
    n, rows, inp, out = size
    dt = TYPES[dtype]
    for k, (name, p, pad, skip) in enumerate((("gelu", 0.0, 0, 0), ("silu", 0.2, 16, 0))[:1 if rows * out > 4e6 else 2]):
        g = torch.Generator().manual_seed(rows + k)
        (x, xs), (w, ws) = held(g, (n, rows, inp), pad, skip), held(g, (n, out, inp), pad, skip)
        b, res = rand(g, (n, out), dt), rand(g, (n, rows, out), dt, pad=pad, skip=skip)
        y, pre = ops.aet_mx4_linear_forward(x, xs, w, ws, b, cols=inp, residual=res, act=name, p=p, seed=k, first_row=5, keep_pre=True, dtype=dt)
        wy, wz = forward(M.values(x, xs, inp), M.values(w, ws, inp), d64(b), d64(res), name, p, k, 5, dt)
        O.near(pre, wz, f"pre {size} {dtype} {name}")
        O.near(y, wy, f"y {size} {dtype} {name}")


@pytest.mark.parametrize("size", [(1, 3000, 1000, 4100), (1, 1500, 2900, 1001), (3, 144, 19169, 2774), (1, 130, 10240, 500)], ids=str)
def test_blocks_that_are_nan(ops, size):   # noqa: F811
    """They make their rows and outputs NaN, and nothing else."""
    n, rows, inp, out = size
    g = torch.Generator().manual_seed(8)
    (x, xs), (w, ws) = held(g, (n, rows, inp)), held(g, (n, out, inp))
    y, _ = ops.aet_mx4_linear_forward(x, xs, w, ws, cols=inp)
    last = (inp + 31) // 32 - 1
    xs[0, rows - 1, last], xs[0, 7, 0], ws[0, out - 1, last], ws[0, 3, 5] = 255, 255, 255, 255
    x[0, 7, :16] = 0
    bad, _ = ops.aet_mx4_linear_forward(x, xs, w, ws, cols=inp)
    fine = torch.ones(n, rows, out, dtype=torch.bool, device=DEV)
    fine[0, [7, rows - 1]], fine[0, :, [3, out - 1]] = False, False
    assert bool(bad[~fine].isnan().all()) and torch.equal(bad[fine], y[fine])


# Tiles of 256, of 128 (whole and in parts), of 64 x 128, and both products in one launch; ragged each way
GRADIENT = [(1, 4100, 2050, 4090), (1, 3000, 4090, 3100), (1, 8000, 1000, 1000), (16, 257, 512, 1000), (1, 1300, 2000, 1290)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("size", GRADIENT, ids=str)
def test_gradient(ops, size, act, dtype):   # noqa: F811
    n, rows, inp, out = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(rows)
    (x, xs), (w, ws) = held(g, (n, rows, inp)), held(g, (n, out, inp))
    dy, pre = rand(g, (n, rows, out), dt), rand(g, (n, rows, out), dt)
    got = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, cols=inp, act=act)
    d, z = dy.double(), pre.double()
    dz, off = d, torch.zeros_like(d)
    if act != "none":   # the slope is off by up to 10 U32 (|z| + 1)
        dz = d * O.slope(z, act)
        off = d.abs() * (4 * 1.13 + 10 * (z.abs() + 1)) * O.U32 + (dz.abs() * 2.0 ** -16 if dt == torch.bfloat16 else 0)
    vx, vw = M.values(x, xs, inp).to(DEV), M.values(w, ws, inp).to(DEV)
    t = lambda v: v.transpose(1, 2).contiguous()   # noqa: E731
    r = O.ROUND[dt]
    for q, a, o, b, what in ((got[0], dz, off, vw, "dx"), (got[1], t(dz), t(off), vx, "dw")):
        v, S = torch.matmul(a, b), torch.matmul(a.abs(), b.abs())
        # sums of up to three parts of each term
        o = torch.matmul(o, b.abs()) + (3 * a.shape[-1] + 4) * O.U32 * S
        fine = (q.double() - v).abs() <= o + r * (v.abs() + o)
        assert bool(fine.all()), f"{what}: {int((~fine).sum())} of {fine.numel()} are off"
        # and on the whole as near as sums in fp32 are: they round some K times by U32 of a part of S, at random
        whole = float((q.double() - v).norm()) / float(S.norm())
        assert whole <= 4 * O.U32 + (2.0 ** -16 + r if dt == torch.bfloat16 else 0), f"{what}: {whole:.3g} of the sum of magnitudes"
    v, o = dz.sum(1), off.sum(1) + (rows + 4) * O.U32 * dz.abs().sum(1)
    assert bool(((got[2].double() - v).abs() <= o + r * (v.abs() + o)).all()), "db"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(3000, 4090, 3100), (1300, 2000, 1290)], ids=str)
def test_captured_and_replayed(ops, size, dtype):   # noqa: F811
    """Two graphs of the layer and its gradient, replayed in turn with eager calls between."""
    rows, inp, out = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(6)
    x, dy = rand(g, (rows, inp), dt), rand(g, (rows, out), dt)
    w, ws = held(g, (out, inp))

    def step():
        c, s = ops.aet_mx4_quantise(x)
        y, pre = ops.aet_mx4_linear_forward(c, s, w, ws, act="gelu", keep_pre=True, dtype=dt)
        return (y, *ops.aet_mx4_linear_backward(dy, c, s, w, ws, pre, act="gelu"))

    step()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(step())
    for k in range(3):
        x.copy_(rand(g, (rows, inp), dt))
        dy.copy_(rand(g, (rows, out), dt, 10.0 ** -k))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = step()
        for got in outs:
            assert all(torch.equal(p, q) for p, q in zip(got, want)), k
