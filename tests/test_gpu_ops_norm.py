"""Group normalisation and dropout and their gradients against their definitions in 64 bits."""
import pytest
import torch

import ops_oracle as O
from test_gpu_ops_linear import DEV, TYPES, d64, ops, rand  # noqa: F401

pytestmark = pytest.mark.gpu

# n, batch, positions, groups, width: one value a group; one position; a channel a group; odd everything; a sample that
# fits one compute unit and ones that do not; few samples with many positions; many small samples
SIZES = [(1, 1, 20, 1, 1), (2, 3, 1, 4, 8), (1, 2, 50, 16, 1), (2, 2, 35, 3, 5), (1, 1, 784, 4, 4), (3, 4, 64, 8, 4),
         (2, 2, 256, 2, 24), (1, 3, 100, 1, 33), (1, 1, 4096, 8, 40), (1, 2, 3001, 5, 7), (1, 1, 20000, 2, 16), (4, 30, 9, 2, 6),
         (1, 2, 17, 32, 40), (1, 1, 1, 1, 2000), (1, 1, 900, 3, 96)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_group_norm(ops, size, dtype):   # noqa: F811
    n, b, P, G, width = size
    dt, ch = TYPES[dtype], G * width
    for k, (name, pad, skip) in enumerate((("none", 0, 0), ("silu", 0, 0), ("gelu", 3, 1), ("relu", 8, 0))):
        g = torch.Generator().manual_seed(P + k)
        x = rand(g, (n, b, P, ch), dt, pad=pad, skip=skip) + 0.5 if not pad else rand(g, (n, b, P, ch), dt, 2.0, pad, skip)
        dy = rand(g, (n, b, P, ch), dt, pad=pad, skip=skip)
        gamma, beta = rand(g, (n, ch), dt, pad=pad, skip=skip), rand(g, (n, ch), dt, pad=pad, skip=skip)
        y, mean, rstd = ops.aet_group_norm_forward(x, G, gamma, beta, eps=1e-3, act=name)
        wy, wm, wr = O.group_norm_forward(d64(x), G, d64(gamma), d64(beta), 1e-3, name, dt)
        O.near(y, wy, f"y {size} {dtype} {name}")
        spread = 1 / wr
        O.near(mean, (wm, 64 * O.U32 * (wm.abs() + spread)), "mean")
        # the variance is off by less than 64 units of itself and of the mean's error squared
        O.near(rstd, (wr, 64 * O.U32 * wr * (1 + O.U32 * (wm * wr).square())), "rstd")
        got = ops.aet_group_norm_backward(dy, x, mean, rstd, gamma, beta, act=name)
        want = O.group_norm_backward(d64(dy), d64(x), d64(mean), d64(rstd), d64(gamma), d64(beta), name, dt)
        if name == "relu":   # a value next to the kink may fall on its other side: then so does the slope
            t = (d64(x).view(n, b, P, G, width) - d64(mean)[:, :, None, :, None]) * d64(rstd)[:, :, None, :, None]
            t = t.reshape(n, b, P, ch) * d64(gamma)[:, None, None] + d64(beta)[:, None, None]
            if bool((t.abs() < 1e-5 * (t.abs().amax() + 1)).any()):
                continue
        for what, a, w in zip(("dx", "dgamma", "dbeta"), got, want):
            O.near(a, w, f"{what} {size} {dtype} {name}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_group_norm_parameters(ops, dtype):   # noqa: F811
    """No gamma or beta, the same ones for all clients (their gradients are sums over the clients), no dx, no clients."""
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(1)
    n, b, P, G, width = 3, 2, 30, 4, 6
    ch = G * width
    x, dy = rand(g, (n, b, P, ch), dt), rand(g, (n, b, P, ch), dt)
    gamma, beta = rand(g, (ch,), dt), rand(g, (ch,), dt)
    y, mean, rstd = ops.aet_group_norm_forward(x, G, gamma, beta, act="gelu")
    fold = x.view(1, n * b, P, ch)
    y1, m1, r1 = ops.aet_group_norm_forward(fold, G, gamma[None], beta[None], act="gelu")
    assert torch.equal(y.view_as(y1), y1) and torch.equal(mean.view_as(m1), m1) and torch.equal(rstd.view_as(r1), r1)
    dx, dgamma, dbeta = ops.aet_group_norm_backward(dy, x, mean, rstd, gamma, beta, act="gelu")
    fx, fg, fb = ops.aet_group_norm_backward(dy.view_as(fold), fold, m1, r1, gamma[None], beta[None], act="gelu")
    assert torch.equal(dx.view_as(fx), fx) and torch.equal(dgamma, fg[0]) and torch.equal(dbeta, fb[0])
    none, dgamma2, dbeta2 = ops.aet_group_norm_backward(dy, x, mean, rstd, gamma, beta, act="gelu", need=(False, True))
    assert none is None and torch.equal(dgamma2, dgamma) and torch.equal(dbeta2, dbeta)
    only, n1, n2 = ops.aet_group_norm_backward(dy, x, mean, rstd, gamma, beta, act="gelu", need=(True, False))
    assert torch.equal(only, dx) and n1 is None and n2 is None
    ones, zeros = torch.ones(n, ch, dtype=dt, device=DEV), torch.zeros(n, ch, dtype=dt, device=DEV)
    a = ops.aet_group_norm_forward(x, G, act="silu")
    assert torch.equal(a[0], ops.aet_group_norm_forward(x, G, ones, zeros, act="silu")[0])
    dx, dgamma, dbeta = ops.aet_group_norm_backward(dy, x, a[1], a[2], act="silu")
    assert dgamma is None and dbeta is None
    assert torch.equal(dx, ops.aet_group_norm_backward(dy, x, a[1], a[2], ones, zeros, act="silu")[0])
    one = ops.aet_group_norm_forward(x[1], G, gamma, beta, act="gelu")
    assert torch.equal(one[0], y[1]) and torch.equal(one[1], mean[1])
    # in place, and dx onto dy is the C call's; the maps' places between rows stay
    whole = torch.full((n, b, P, ch + 5), 3.0, dtype=dt, device=DEV)
    whole[..., 2:2 + ch] = x
    ops.aet_group_norm_forward(whole[..., 2:2 + ch], G, gamma, beta, act="gelu", out=whole[..., 2:2 + ch])
    # dx in dy's place, dgamma and dbeta as parts of one row of parameters a client
    onto, flat = dy.clone(), torch.full((n, 2 * ch + 3), 5.0, dtype=dt, device=DEV)
    pg, pb = gamma.expand(n, ch).contiguous(), beta.expand(n, ch).contiguous()
    want = ops.aet_group_norm_backward(dy, x, mean, rstd, pg, pb, act="gelu")
    got = ops.aet_group_norm_backward(onto, x, mean, rstd, pg, pb, act="gelu", out=(onto, flat[:, 1:1 + ch], flat[:, 2 + ch:2 + 2 * ch]))
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(onto, want[0]) and bool((flat[:, 0] == 5).all())
    assert torch.equal(whole[..., 2:2 + ch], y) and bool((whole[..., :2] == 3).all()) and bool((whole[..., 2 + ch:] == 3).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_group_norm_edges(ops, dtype):   # noqa: F811
    dt = TYPES[dtype]
    z = lambda *s: torch.ones(*s, dtype=dt, device=DEV)   # noqa: E731
    y, mean, rstd = ops.aet_group_norm_forward(z(2, 3, 0, 8), 2, eps=0.25)
    assert y.numel() == 0 and bool((mean == 0).all()) and bool((rstd == 2).all())
    dx, dgamma, dbeta = ops.aet_group_norm_backward(z(2, 3, 0, 8), z(2, 3, 0, 8), mean, rstd, z(2, 8), z(2, 8))
    assert dx.numel() == 0 and torch.equal(dgamma, z(2, 8) * 0) and torch.equal(dbeta, z(2, 8) * 0)
    dx, dgamma, dbeta = ops.aet_group_norm_backward(z(2, 0, 4, 8), z(2, 0, 4, 8), z(2, 0, 2).float(), z(2, 0, 2).float(), z(2, 8), z(2, 8))
    assert torch.equal(dgamma, z(2, 8) * 0) and torch.equal(dbeta, z(2, 8) * 0)
    assert ops.aet_group_norm_forward(z(0, 3, 4, 8), 2)[0].numel() == 0
    # the same value everywhere: what is normalised is 0 exactly, and so is its gradient
    y, mean, rstd = ops.aet_group_norm_forward(z(1, 2, 40, 16) * 3, 2, z(1, 16), z(1, 16) * 0.5)
    assert torch.equal(y, z(1, 2, 40, 16) * 0.5) and bool((mean == 3).all())
    # far from 0: the variance is that of the values, not lost in their square
    x = (torch.arange(64, device=DEV).view(1, 1, 64, 1) % 2).expand(1, 1, 64, 4).to(dt).contiguous() * 2 + 200
    y, mean, rstd = ops.aet_group_norm_forward(x, 1, eps=0.0)
    assert torch.equal(y, (x - 201)) and bool((mean == 201).all()) and bool((rstd == 1).all())
    # an infinity makes its own group NaN and no other
    x = torch.randn(1, 2, 50, 12, device=DEV).to(dt)
    x[0, 1, 7, 5] = float("inf")
    y, mean, rstd = ops.aet_group_norm_forward(x, 3, act="silu")
    assert torch.isnan(y[0, 1, :, 4:8]).all() and torch.isfinite(y[0, 0]).all()
    assert torch.isfinite(y[0, 1, :, :4]).all() and torch.isfinite(y[0, 1, :, 8:]).all()


def test_group_norm_differences(ops):   # noqa: F811
    """Central differences in fp32 along random directions; steps of 1/64, values of order one."""
    g = torch.Generator().manual_seed(5)
    n, b, P, G, width = 2, 2, 12, 2, 4
    f32 = torch.float32
    x, gamma, beta, cst = (rand(g, s, f32) for s in ((n, b, P, 8), (n, 8), (n, 8), (n, b, P, 8)))
    for name in ("none", "silu", "gelu"):
        _, mean, rstd = ops.aet_group_norm_forward(x, G, gamma, beta, act=name)
        grads = ops.aet_group_norm_backward(cst, x, mean, rstd, gamma, beta, act=name)
        for k in range(3):
            t = [x, gamma, beta]
            v = rand(g, t[k].shape, f32)
            f = []
            for s in (2.0 ** -6, -2.0 ** -6):
                u = list(t)
                u[k] = t[k] + s * v
                f.append((ops.aet_group_norm_forward(u[0], G, u[1], u[2], act=name)[0].double() * cst.double()).sum())
            want = float((f[0] - f[1]) * 2.0 ** 5)
            got = float((grads[k].double() * v.double()).sum())
            scale = float((grads[k].double().square().sum() * v.double().square().sum()).sqrt())
            assert abs(got - want) <= 5e-3 * scale, (name, k, got, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,skip", [(0, 0), (1, 0), (8, 0), (0, 1), (3, 5)])
@pytest.mark.parametrize("size", [(1, 1, 1), (1, 1, 784), (2, 3, 7), (1, 33, 128), (3, 5, 1000), (1, 70, 2049), (1, 1000, 3), (1, 3, 8192)], ids=str)
def test_dropout(ops, size, pad, skip, dtype):   # noqa: F811
    n, rows, cols = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(rows + cols)
    x, res = rand(g, size, dt, pad=pad, skip=skip), rand(g, size, dt, pad=pad, skip=skip)
    for p, seed, first in ((0.1, 0, 0), (0.5, 2 ** 64 - 1, 2 ** 40 + 1), (0.0, 3, 5), (0.999, 7, 1)):
        m = O.mask3(size, seed, first, p)
        y = ops.aet_dropout_forward(x, p=p, seed=seed, first_row=first)
        want = d64(x) * m
        O.near(y, (want, (O.ROUND[dt] + 3 * O.U32) * want.abs()), "y")
        assert torch.equal(y.cpu() == 0, (m == 0) | (d64(x) == 0))
        assert torch.equal(ops.aet_dropout_backward(x, p=p, seed=seed, first_row=first), y)
        y = ops.aet_dropout_forward(x, p=p, seed=seed, first_row=first, residual=res)
        total = want + d64(res)
        O.near(y, (total, O.ROUND[dt] * total.abs() * 1.01 + 4 * O.U32 * (want.abs() + d64(res).abs())), "y with residual")
        inplace = x.clone()
        ops.aet_dropout_forward(inplace, p=p, seed=seed, first_row=first, residual=res, out=inplace)
        assert torch.equal(inplace, y)
    # rows of a larger tensor, called by parts
    if rows > 2 and n == 1:
        whole = ops.aet_dropout_forward(x, p=0.3, seed=8)
        part = ops.aet_dropout_forward(x[:, 2:], p=0.3, seed=8, first_row=2)
        assert torch.equal(whole[:, 2:], part)


def test_dropout_takes_out_what_is_not_finite(ops):   # noqa: F811
    x = torch.full((64, 64), float("nan"), device=DEV)
    y = ops.aet_dropout_forward(x, p=0.5, seed=1)
    m = O.kept(1, 0, 64, 64, 0.5)
    assert torch.equal(torch.isnan(y).cpu(), m > 0) and bool((y.cpu()[m == 0] == 0).all())
    assert ops.aet_dropout_forward(torch.empty(0, 5, device=DEV), p=0.5, seed=1).shape == (0, 5)


def test_other_streams_and_graphs(ops):   # noqa: F811
    g = torch.Generator().manual_seed(4)
    for dt, (n, b, P, G, width) in ((torch.float32, (2, 3, 64, 4, 8)), (torch.bfloat16, (1, 1, 5000, 8, 16))):
        x, dy = rand(g, (n, b, P, G * width), dt), rand(g, (n, b, P, G * width), dt)
        gamma, beta = rand(g, (n, G * width), dt), rand(g, (n, G * width), dt)

        def calls(stream=None):
            y, mean, rstd = ops.aet_group_norm_forward(x, G, gamma, beta, act="silu", stream=stream)
            more = ops.aet_group_norm_backward(dy, x, mean, rstd, gamma, beta, act="silu", stream=stream)
            flat = y.view(n, b * P, G * width)
            d = ops.aet_dropout_forward(flat, p=0.2, seed=6, residual=dy.view_as(flat), stream=stream)
            return y, mean, rstd, *more, d

        want = calls()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        got = calls(s)
        s.synchronize()
        assert all(torch.equal(a, w) for a, w in zip(got, want))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = calls()
        for _ in range(3):
            for t in got:
                t.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, w) for a, w in zip(got, want))
            x.float().sum().item()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_clients_of_shared_parameters(ops, dtype):   # noqa: F811
    """gamma and beta of all clients, of whom there are none: the gradients are sums of nothing."""
    dt = TYPES[dtype]
    z = lambda *s: torch.ones(*s, dtype=dt, device=DEV)   # noqa: E731
    out = (None, torch.full((8,), 5.0, dtype=dt, device=DEV), torch.full((8,), 5.0, dtype=dt, device=DEV))
    dx, dgamma, dbeta = ops.aet_group_norm_backward(z(0, 3, 4, 8), z(0, 3, 4, 8), z(0, 3, 2).float(), z(0, 3, 2).float(), z(8), z(8), out=out)
    assert dx.shape == (0, 3, 4, 8) and torch.equal(dgamma, z(8) * 0) and torch.equal(dbeta, z(8) * 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_group_norm_of_many_groups(ops, dtype):   # noqa: F811
    """Thousands of groups of a channel or two: what a workgroup keeps of each has to fit."""
    dt = TYPES[dtype]
    for n, b, P, G, width in ((1, 600, 3, 2048, 1), (2, 130, 16, 2500, 1), (1, 300, 5, 1030, 2)):
        ch = G * width
        g = torch.Generator().manual_seed(G)
        x, dy, gamma, beta = (rand(g, s, dt) for s in ((n, b, P, ch), (n, b, P, ch), (n, ch), (n, ch)))
        y, mean, rstd = ops.aet_group_norm_forward(x, G, gamma, beta, eps=1e-2, act="silu")
        wy, _, _ = O.group_norm_forward(d64(x), G, d64(gamma), d64(beta), 1e-2, "silu", dt)
        O.near(y, wy, f"y {dtype} {G}")
        got = ops.aet_group_norm_backward(dy, x, mean, rstd, gamma, beta, act="silu")
        want = O.group_norm_backward(d64(dy), d64(x), d64(mean), d64(rstd), d64(gamma), d64(beta), "silu", dt)
        for what, a, w in zip(("dx", "dgamma", "dbeta"), got, want):
            O.near(a, w, f"{what} {dtype} {G}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(2, 3, 50, 3, 5), (1, 2, 4096, 8, 3), (1, 40, 300, 6, 7), (1, 3, 20000, 3, 11), (1, 2, 9000, 1, 3), (2, 64, 1024, 9, 10),
                                  (1, 700, 20, 300, 5)], ids=str)
def test_pieces_in_place(ops, size, dtype):   # noqa: F811
    """Channels that are not whole pieces of 16 bytes, results in the inputs' places, NaN between the rows: the same bits, and
    nothing beside them is written."""
    n, b, P, G, width = size
    dt, ch = TYPES[dtype], G * width
    g = torch.Generator().manual_seed(ch + P)
    gamma, beta = rand(g, (n, ch), dt), rand(g, (n, ch), dt)
    x, dy = rand(g, (n, b, P, ch), dt), rand(g, (n, b, P, ch), dt)
    y, mean, rstd = ops.aet_group_norm_forward(x, G, gamma, beta, act="silu")
    O.near(y, O.group_norm_forward(d64(x), G, d64(gamma), d64(beta), 1e-5, "silu", dt)[0], f"y {size} {dtype}")
    want = ops.aet_group_norm_backward(dy, x, mean, rstd, gamma, beta, act="silu")
    for what, a, w in zip(("dx", "dgamma", "dbeta"), want, O.group_norm_backward(d64(dy), d64(x), d64(mean), d64(rstd), d64(gamma), d64(beta), "silu", dt)):
        O.near(a, w, f"{what} {size} {dtype}")
    places = torch.full((2, n, b, P, ch + 3), float("nan"), dtype=dt, device=DEV)
    px, pdy = places[0, ..., 1:1 + ch], places[1, ..., 1:1 + ch]
    px.copy_(x)
    pdy.copy_(dy)
    got = ops.aet_group_norm_backward(pdy, px, mean, rstd, gamma, beta, act="silu", out=(pdy, None, None))
    assert all(torch.equal(a, c) for a, c in zip(got, want)) and torch.equal(px, x)
    out = ops.aet_group_norm_forward(px, G, gamma, beta, act="silu", out=px)
    assert torch.equal(px, y) and torch.equal(out[1], mean) and torch.equal(out[2], rstd)
    assert bool(torch.isnan(places[..., 0]).all()) and bool(torch.isnan(places[..., 1 + ch:]).all())
