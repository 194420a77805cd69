"""The linear operator and its gradient against their definitions in 64 bits, within bounds that follow from the number
formats, at the sizes, strides and alignments where tiles, vectors and splits begin and end."""
import pytest
import torch

import ops_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    from paper_2112_13935_amd import ops
    ops.load_library()
    # PyTorch hands out streams from a ring of 32, and which hardware queue a stream has depends on the order of their first
    # use; tests of streams that come later find the ring where it was.
    ring = [torch.cuda.Stream().cuda_stream for _ in range(32)]
    yield ops
    for _ in range(32):
        if torch.cuda.Stream().cuda_stream == ring[-1]:
            break


def rand(g, shape, dtype, scale=1.0, pad=0, skip=0):
    """Values whose rows lie pad elements further apart, starting skip elements past a 256-byte boundary."""
    *lead, cols = shape
    rows = 1
    for k in lead:
        rows *= k
    flat = torch.randn(skip + rows * (cols + pad) + 1, generator=g) * scale
    flat = flat.to(dtype).to(DEV)
    return flat[skip:skip + rows * (cols + pad)].view(*lead, cols + pad)[..., :cols]


def d64(t):
    return None if t is None else t.double().cpu()


# n, rows, in, out: a single value; single rows; rows that end inside every tile; one and several clients; few rows with
# long sums; odd sizes; sums that end inside a step; more outputs or rows than one tile
SIZES = [(1, 1, 1, 1), (1, 1, 784, 128), (3, 1, 50, 7), (1, 5, 1000, 33), (2, 16, 64, 16), (4, 17, 72, 130), (1, 33, 257, 65),
         (2, 64, 128, 96), (3, 100, 40, 200), (1, 129, 192, 128), (1, 256, 64, 256), (1, 300, 520, 264), (2, 257, 129, 255),
         (1, 8, 4096, 48), (16, 32, 784, 128), (1, 511, 1024, 384), (1, 1024, 96, 10), (1, 40, 8, 1000), (1, 640, 640, 640)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward(ops, size, dtype):
    n, rows, inp, out = size
    dt = TYPES[dtype]
    for k, (name, p, with_bias, with_res, with_pre) in enumerate([
            ("none", 0.0, False, False, False), ("gelu", 0.1, True, True, True), ("relu", 0.0, True, False, True),
            ("silu", 0.5, False, True, False)]):
        g = torch.Generator().manual_seed(k + 10 * rows + out)
        x, w = rand(g, (n, rows, inp), dt), rand(g, (n, out, inp), dt, inp ** -0.5)
        b = rand(g, (n, out), dt) if with_bias else None
        res = rand(g, (n, rows, out), dt) if with_res else None
        y, pre = ops.aet_linear_forward(x, w, b, residual=res, act=name, p=p, seed=77 + k, first_row=k * (1 << 33), keep_pre=with_pre)
        wy, wpre = O.linear_forward(d64(x), d64(w), d64(b), d64(res), name, p, 77 + k, k * (1 << 33), dt)
        O.near(y, wy, f"y {size} {dtype} {name}")
        if with_pre:
            O.near(pre, wpre, f"pre {size} {dtype} {name}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_backward(ops, size, dtype):
    n, rows, inp, out = size
    dt = TYPES[dtype]
    for k, (name, p) in enumerate([("none", 0.0), ("gelu", 0.1), ("relu", 0.5), ("silu", 0.0), ("none", 0.25)]):
        g = torch.Generator().manual_seed(k + 10 * rows + out)
        x, w = rand(g, (n, rows, inp), dt), rand(g, (n, out, inp), dt, inp ** -0.5)
        dy, pre = rand(g, (n, rows, out), dt), rand(g, (n, rows, out), dt) if name != "none" else None
        got = ops.aet_linear_backward(dy, x, w, pre, act=name, p=p, seed=5 + k, first_row=3 * k)
        want = O.linear_backward(d64(dy), d64(x), d64(w), d64(pre), name, p, 5 + k, 3 * k, dt)
        for what, a, b in zip(("dx", "dw", "db"), got, want):
            O.near(a, b, f"{what} {size} {dtype} {name}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size,pad", [((2, 2568, 2624, 2632), 0), ((2, 2568, 2624, 2632), 3), ((1, 3000, 700, 4104), 0)], ids=str)
def test_large(ops, size, pad, dtype):
    """Many tiles of the largest kind, whole and at the edges."""
    n, rows, inp, out = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(pad)
    x, w, b = rand(g, (n, rows, inp), dt, pad=pad), rand(g, (n, out, inp), dt, inp ** -0.5), rand(g, (n, out), dt)
    dy, pre = rand(g, (n, rows, out), dt), rand(g, (n, rows, out), dt)
    y, z = ops.aet_linear_forward(x, w, b, act="gelu", p=0.1, seed=1, keep_pre=True)
    got = ops.aet_linear_backward(dy, x, w, pre, act="gelu", p=0.1, seed=1)
    torch.cuda.synchronize()
    wy, wz = O.linear_forward(d64(x), d64(w), d64(b), None, "gelu", 0.1, 1, 0, dt)
    O.near(y, wy, "y")
    O.near(z, wz, "pre")
    for what, a, b_ in zip(("dx", "dw", "db"), got, O.linear_backward(d64(dy), d64(x), d64(w), d64(pre), "gelu", 0.1, 1, 0, dt)):
        O.near(a, b_, what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,skip", [(1, 0), (8, 0), (0, 1), (5, 3), (24, 8)])
@pytest.mark.parametrize("size", [(2, 9, 56, 40), (1, 150, 264, 136), (1, 256, 128, 256)], ids=str)
def test_strides_and_alignment(ops, size, pad, skip, dtype):
    n, rows, inp, out = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(pad + 7 * skip)
    more = dict(pad=pad, skip=skip)
    x, w, b = rand(g, (n, rows, inp), dt, **more), rand(g, (n, out, inp), dt, inp ** -0.5, **more), rand(g, (n, out), dt, **more)
    res, dy, pre = (rand(g, (n, rows, out), dt, **more) for _ in range(3))
    out_t = rand(g, (n, rows, out), dt, **more)
    around = out_t.clone()
    y, z = ops.aet_linear_forward(x, w, b, residual=res, act="silu", p=0.2, seed=1, keep_pre=True, out=out_t)
    assert y is out_t and not torch.equal(around, out_t)
    wy, wz = O.linear_forward(d64(x), d64(w), d64(b), d64(res), "silu", 0.2, 1, 0, dt)
    O.near(y, wy, "y")
    O.near(z, wz, "pre")
    got = ops.aet_linear_backward(dy, x, w, pre, act="gelu", p=0.2, seed=1)
    for what, a, b_ in zip(("dx", "dw", "db"), got, O.linear_backward(d64(dy), d64(x), d64(w), d64(pre), "gelu", 0.2, 1, 0, dt)):
        O.near(a, b_, what)
    # y may be the residual itself
    want = ops.aet_linear_forward(x, w, b, residual=res, p=0.2, seed=1)[0]
    ops.aet_linear_forward(x, w, b, residual=res, p=0.2, seed=1, out=res)
    assert torch.equal(res, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_outputs_leave_what_lies_between_rows(ops, dtype):
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(0)
    for rows, inp, out in ((37, 64, 50), (256, 128, 248), (3, 200, 9)):
        x, w = rand(g, (1, rows, inp), dt), rand(g, (1, out, inp), dt)
        whole = torch.full((1, rows + 2, out + 11), 7.0, dtype=dt, device=DEV)
        ops.aet_linear_forward(x, w, act="relu", out=whole[:, 1:-1, 4:4 + out])
        inner = torch.zeros_like(whole, dtype=torch.bool)
        inner[:, 1:-1, 4:4 + out] = True
        assert bool((whole[~inner] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_shared_weights_and_broadcast_inputs(ops, dtype):
    """One W and bias for all clients: their gradients are sums over the clients, bit for bit those of one client with all
    rows; one x for all clients; a leading axis of clients left out."""
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(3)
    n, rows, inp, out = 3, 21, 72, 40
    x, w, b = rand(g, (n, rows, inp), dt), rand(g, (out, inp), dt, inp ** -0.5), rand(g, (out,), dt)
    dy, res = rand(g, (n, rows, out), dt), rand(g, (n, rows, out), dt)
    y, pre = ops.aet_linear_forward(x, w, b, residual=res, act="gelu", p=0.1, seed=4, keep_pre=True)
    per = [t.expand(n, *t.shape).contiguous() for t in (w, b)]
    wy, _ = O.linear_forward(d64(x), d64(per[0]), d64(per[1]), d64(res), "gelu", 0.1, 4, 0, dt)
    O.near(y, wy, "y")
    dx, dw, db = ops.aet_linear_backward(dy, x, w, pre, act="gelu", p=0.1, seed=4)
    flat = [t.view(1, n * rows, -1) for t in (dy, x, pre)]
    fx, fw, fb = ops.aet_linear_backward(flat[0], flat[1], w[None], flat[2], act="gelu", p=0.1, seed=4)
    assert torch.equal(dx.view(1, n * rows, -1), fx) and torch.equal(dw[None], fw) and torch.equal(db[None], fb)
    one = ops.aet_linear_forward(x[0], w, b, act="silu")[0]
    assert torch.equal(one, ops.aet_linear_forward(x[:1], w[None], b[None], act="silu")[0][0])
    wide = ops.aet_linear_forward(x[:1].expand(n, rows, inp), per[0], per[1])[0]
    for c in range(n):
        assert torch.equal(wide[c], wide[0])
    wy, _ = O.linear_forward(d64(x[:1]), d64(w[None]), d64(b[None]), None, "none", 0, 0, 0, dt)
    O.near(wide[:1], wy, "broadcast x")
    # dx with rows apart and one W for all
    apart = rand(g, (n, rows, inp), dt, pad=3)
    dx, _, _ = ops.aet_linear_backward(dy, apart, w, need=(True, False, False))
    want = O.linear_backward(d64(dy), d64(apart), d64(per[0]), None, "none", 0, 0, 0, dt)
    O.near(dx, want[0], "dx")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sizes_of_zero(ops, dtype):
    dt = TYPES[dtype]
    z = lambda *s: torch.ones(*s, dtype=dt, device=DEV)   # noqa: E731
    y, _ = ops.aet_linear_forward(z(2, 3, 0), z(2, 4, 0), z(2, 4) * 2, residual=z(2, 3, 4), act="relu")
    assert torch.equal(y, z(2, 3, 4) * 3)
    dx, dw, db = ops.aet_linear_backward(z(2, 0, 4), z(2, 0, 5), z(2, 4, 5))
    assert dx.numel() == 0 and torch.equal(dw, z(2, 4, 5) * 0) and torch.equal(db, z(2, 4) * 0)
    dx, dw, db = ops.aet_linear_backward(z(2, 3, 0), z(2, 3, 5), z(2, 0, 5))
    assert torch.equal(dx, z(2, 3, 5) * 0) and dw.numel() == db.numel() == 0
    dx, dw, db = ops.aet_linear_backward(z(2, 3, 4), z(2, 3, 0), z(2, 4, 0))
    assert torch.equal(db, z(2, 4) * 3)
    for shape in ((0, 3, 5), (2, 0, 5)):
        y, pre = ops.aet_linear_forward(z(*shape), z(shape[0], 4, 5), keep_pre=True)
        assert y.numel() == pre.numel() == 0
    assert [t.numel() for t in ops.aet_linear_backward(z(0, 3, 4), z(0, 3, 5), z(0, 4, 5))] == [0, 0, 0]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_that_are_not_finite(ops, dtype):
    """Where the definition has an infinity or a NaN, so has the result, and nowhere else; what dropout takes out is 0
    whatever it was."""
    dt = TYPES[dtype]
    big = torch.finfo(dt).max
    for rows in (3, 70, 300):
        g = torch.Generator().manual_seed(rows)
        n, inp, out = 1, 192, 72
        x, w = rand(g, (n, rows, inp), dt), rand(g, (n, out, inp), dt, inp ** -0.5)
        w[0, 0] = 0
        w[0, 0, 5] = 1
        x[0, 0, 5], x[0, 1, 5], x[0, 2, 5] = float("inf"), float("nan"), big
        for name in ("none", "relu"):
            y, _ = ops.aet_linear_forward(x, w, act=name)
            want = O.act(d64(x) @ d64(w).transpose(1, 2), name)
            if name == "relu":
                want[0, 1] = float("nan")
            col = y.double().cpu()
            assert col[0, 0, 0] == float("inf") and torch.isnan(col[0, 1]).all()
            assert float((col[0, 2, 0] - float(big)).abs()) <= float(big) * 2 ** -8   # finite
            assert torch.equal(torch.isfinite(col[0, 3:]), torch.ones_like(col[0, 3:], dtype=torch.bool))
            ok = torch.isfinite(want[0, 0])
            assert torch.equal(torch.isnan(col[0, 0]), torch.isnan(want[0, 0])) and torch.equal(torch.isfinite(col[0, 0]), ok)
        y, _ = ops.aet_linear_forward(x, w, p=0.5, seed=9)
        gone = O.kept(9, 0, rows, out, 0.5) == 0
        assert bool((y[0].cpu()[gone] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
def test_what_dropout_took_out_has_no_gradient(ops, dtype, act):
    """Infinities and NaN in z and dy, where the mask is 0, leave no trace."""
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(4)
    n, rows, inp, out = 1, 70, 40, 72
    x, w = rand(g, (n, rows, inp), dt), rand(g, (n, out, inp), dt)
    dy, pre = rand(g, (n, rows, out), dt), rand(g, (n, rows, out), dt)
    gone = (O.kept(9, 0, rows, out, 0.5) == 0).to(DEV)[None]
    want = ops.aet_linear_backward(dy, x, w, pre, act=act, p=0.5, seed=9)
    for bad in (float("nan"), float("inf"), -float("inf")):
        z, d = pre.clone(), dy.clone()
        z[gone] = bad
        d[gone] = bad
        got = ops.aet_linear_backward(d, x, w, z, act=act, p=0.5, seed=9)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_into_given_places(ops, dtype):
    """dw and db as parts of one row of parameters a client, dx with rows apart."""
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(6)
    n, rows, inp, out = 3, 45, 56, 24
    x, w, dy = rand(g, (n, rows, inp), dt), rand(g, (n, out, inp), dt), rand(g, (n, rows, out), dt)
    want = ops.aet_linear_backward(dy, x, w)
    flat = torch.full((n, out * inp + out + 9), 5.0, dtype=dt, device=DEV)
    dw, db = flat[:, 3:3 + out * inp].view(n, out, inp), flat[:, 3 + out * inp:3 + out * inp + out]
    wide = torch.full((n, rows, inp + 7), 5.0, dtype=dt, device=DEV)
    got = ops.aet_linear_backward(dy, x, w, out=(wide[:, :, 2:2 + inp], dw, db))
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and got[1].data_ptr() == dw.data_ptr()
    assert bool((flat[:, :3] == 5).all()) and bool((flat[:, 3 + out * inp + out:] == 5).all())
    assert bool((wide[:, :, :2] == 5).all()) and bool((wide[:, :, 2 + inp:] == 5).all())


def test_differences(ops):
    """The gradient of the whole operator against central differences of the forward call, in fp32: sum(y * c) along
    random directions.  Steps of 1/64 with values of order one: the third derivatives give 1e-4 of relative error at
    most, rounding of sums of 640 terms 64 * 1e-5."""
    g = torch.Generator().manual_seed(8)
    n, rows, inp, out = 2, 20, 24, 16
    x, w, b = rand(g, (n, rows, inp), torch.float32), rand(g, (n, out, inp), torch.float32, 0.2), rand(g, (n, out), torch.float32, 0.2)
    cst = rand(g, (n, rows, out), torch.float32)
    for name in ("none", "silu", "gelu"):
        more = dict(act=name, p=0.3, seed=11)
        _, pre = ops.aet_linear_forward(x, w, b, keep_pre=True, **more)
        grads = ops.aet_linear_backward(cst, x, w, pre, **more)
        for k in range(3):
            t = [x, w, b]
            v = rand(g, t[k].shape, torch.float32)
            h = 2.0 ** -6
            f = []
            for s in (h, -h):
                u = list(t)
                u[k] = t[k] + s * v
                f.append((ops.aet_linear_forward(*u, **more)[0].double() * cst.double()).sum())
            want = float((f[0] - f[1]) / (2 * h))
            got = float((grads[k].double() * v.double()).sum())
            scale = float((grads[k].double().square().sum() * v.double().square().sum()).sqrt())
            assert abs(got - want) <= 5e-3 * scale, (name, k, got, want)


def test_other_streams_and_graphs(ops):
    """On a stream of the caller's, and captured into a graph that is replayed with other work in between."""
    g = torch.Generator().manual_seed(2)
    for dt, (n, rows, inp, out) in ((torch.float32, (2, 40, 96, 64)), (torch.bfloat16, (1, 300, 256, 192)), (torch.bfloat16, (1, 1, 1024, 64))):
        x, w, dy = rand(g, (n, rows, inp), dt), rand(g, (n, out, inp), dt, 0.1), rand(g, (n, rows, out), dt)
        want_y, want_pre = ops.aet_linear_forward(x, w, act="gelu", p=0.1, seed=3, keep_pre=True)
        want = ops.aet_linear_backward(dy, x, w, want_pre, act="gelu", p=0.1, seed=3)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        y, pre = ops.aet_linear_forward(x, w, act="gelu", p=0.1, seed=3, keep_pre=True, stream=s)
        got = ops.aet_linear_backward(dy, x, w, pre, act="gelu", p=0.1, seed=3, stream=s)
        s.synchronize()
        assert torch.equal(y, want_y) and all(torch.equal(a, b) for a, b in zip(got, want))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y, pre = ops.aet_linear_forward(x, w, act="gelu", p=0.1, seed=3, keep_pre=True)
            got = ops.aet_linear_backward(dy, x, w, pre, act="gelu", p=0.1, seed=3)
        for _ in range(3):
            for t in (y, pre, *got):
                t.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want_y) and torch.equal(pre, want_pre) and all(torch.equal(a, b) for a, b in zip(got, want))
            (x @ x.transpose(1, 2).contiguous()).sum().item()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_clients_of_a_shared_layer(ops, dtype):
    """One W and bias of all clients, of whom there are none: their gradients are sums of nothing."""
    dt = TYPES[dtype]
    z = lambda *s: torch.ones(*s, dtype=dt, device=DEV)   # noqa: E731
    out = (None, torch.full((6, 8), 5.0, dtype=dt, device=DEV), torch.full((6,), 5.0, dtype=dt, device=DEV))
    dx, dw, db = ops.aet_linear_backward(z(0, 3, 6), z(0, 3, 8), z(6, 8), z(0, 3, 6), act="relu", out=out)
    assert dx.shape == (0, 3, 8) and torch.equal(dw, z(6, 8) * 0) and torch.equal(db, z(6) * 0)


def test_outputs_on_another_stream_are_its_own(ops):
    """Memory given back on the current stream may still be in use there: a call on another stream gets its own."""
    x, w = torch.randn(4, 64, device=DEV), torch.randn(96, 64, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y, _ = ops.aet_linear_forward(x, w, stream=s)
    at = y.data_ptr()
    owner = [g["stream"] for g in torch.cuda.memory_snapshot() if g["address"] <= at < g["address"] + g["total_size"]]
    assert owner == [s.cuda_stream]
    s.synchronize()
    assert torch.equal(y, ops.aet_linear_forward(x, w)[0])


def among_nan(g, shape, dtype, scale, pad, skip):
    """rand(), with NaN in the places before, between and after the rows."""
    t = rand(g, shape, dtype, scale)
    flat = torch.full((skip + t.numel() // shape[-1] * (shape[-1] + pad) + 9,), float("nan"), dtype=dtype, device=DEV)
    to = flat[skip:flat.numel() - 9].view(*shape[:-1], shape[-1] + pad)[..., :shape[-1]]
    to.copy_(t)
    return to


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,skip", [(0, 0), (1, 0), (0, 1), (1, 1), (3, 2), (8, 8)])
@pytest.mark.parametrize("size", [(2, 27, 2101, 40), (1, 1, 4097, 33), (3, 16, 2080, 20), (2, 20, 300, 50), (1, 3, 64, 17), (3, 9, 31, 16),
                                  (2, 150, 200, 77), (1, 70, 129, 131), (2, 65, 64, 9), (1, 260, 515, 261)], ids=str)
def test_places_between_rows(ops, size, pad, skip, dtype):
    """Rows that begin at odd places, and memory around them that must not count."""
    n, rows, inp, out = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(rows + inp + pad)
    x, w = among_nan(g, (n, rows, inp), dt, 1.0, pad, skip), among_nan(g, (n, out, inp), dt, inp ** -0.5, 2 * pad, skip)
    dy, pre = among_nan(g, (n, rows, out), dt, 1.0, pad, skip), among_nan(g, (n, rows, out), dt, 1.0, 0, 1)
    b = among_nan(g, (n, out), dt, 1.0, pad, skip)
    for xx in (x, x.contiguous()):   # the operands' rows begin alike, or not
        y, _ = ops.aet_linear_forward(xx, w, b, act="silu")
        O.near(y, O.linear_forward(d64(x), d64(w), d64(b), None, "silu", 0.0, 0, 0, dt)[0], f"y {size} {dtype} {pad} {skip}")
        got = ops.aet_linear_backward(dy, xx, w, pre, act="silu")
        want = O.linear_backward(d64(dy), d64(x), d64(w), d64(pre), "silu", 0.0, 0, 0, dt)
        for what, a, c in zip(("dx", "dw", "db"), got, want):
            O.near(a, c, f"{what} {size} {dtype} {pad} {skip}")
        got = ops.aet_linear_backward(dy, xx, w, need=(True, True, False))   # the products' operand is dy itself
        want = O.linear_backward(d64(dy), d64(x), d64(w), None, "none", 0.0, 0, 0, dt)
        for what, a, c in zip(("dx", "dw"), got, want):
            O.near(a, c, f"{what} of dy {size} {dtype} {pad} {skip}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 200, 264, 333), (2, 300, 72, 70), (1, 520, 1000, 1000), (1, 40, 4104, 72), (1, 72, 8, 520), (3, 33, 136, 200),
                                  (1, 300, 1992, 40), (1, 1992, 64, 328)], ids=str)
def test_sums_that_end_inside_a_stage(ops, size, dtype):
    """What lies behind the end of a sum, the next row's first values, must not count: they are infinite in every second row."""
    n, rows, inp, out = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(rows + inp)
    x, w, dy, pre = (rand(g, s, dt, c) for s, c in (((n, rows, inp), 1.0), ((n, out, inp), inp ** -0.5), ((n, rows, out), 1.0), ((n, rows, out), 1.0)))
    y, _ = ops.aet_linear_forward(x, w)
    O.near(y, O.linear_forward(d64(x), d64(w), None, None, "none", 0.0, 0, 0, dt)[0], f"y {size} {dtype}")
    got = ops.aet_linear_backward(dy, x, w, pre, act="gelu", p=0.1, seed=9)
    want = O.linear_backward(d64(dy), d64(x), d64(w), d64(pre), "gelu", 0.1, 9, 0, dt)
    for what, a, c in zip(("dx", "dw", "db"), got, want):
        O.near(a, c, f"{what} {size} {dtype}")
    bad = x.clone()
    bad[:, 1::2, 0] = float("inf")
    assert torch.equal(ops.aet_linear_forward(bad, w)[0][:, ::2], y[:, ::2])
    dx, dw, _ = ops.aet_linear_backward(dy, x, w)
    bad = dy.clone()
    bad[:, 1::2, 0] = float("inf")
    assert torch.equal(ops.aet_linear_backward(bad, x, w)[0][:, ::2], dx[:, ::2])
    bad = x.clone()
    bad[..., 1::2] = float("nan")   # columns of the gradient of w
    assert torch.equal(ops.aet_linear_backward(dy, bad, w)[1][..., ::2], dw[..., ::2])
