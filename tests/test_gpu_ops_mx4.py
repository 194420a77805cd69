"""Microscaled 4-bit values, there and back, bit for bit, and the linear layer of them and its gradient against their
definitions in 64 bits."""
import ctypes as C

import pytest
import torch

import mx4_oracle as M
import ops_oracle as O
from test_gpu_ops_linear import DEV, TYPES, d64, ops, rand  # noqa: F401

pytestmark = pytest.mark.gpu


def bytes_of(g, shape, pad=0, skip=0, top=256):
    """Random bytes whose rows lie pad apart, from an odd place on."""
    *lead, cols = shape
    rows = 1
    for k in lead:
        rows *= k
    flat = torch.randint(0, top, (skip + rows * (cols + pad) + 1,), generator=g, dtype=torch.uint8).to(DEV)
    return flat[skip:skip + rows * (cols + pad)].view(*lead, cols + pad)[..., :cols]


def held(g, shape, pad=0, skip=0, spread=8):
    """Codes and scales of an [n, rows, cols] tensor of values around 1, scales of each block its own."""
    cols = shape[-1]
    codes = bytes_of(g, (*shape[:-1], (cols + 1) // 2), pad, skip)
    scales = bytes_of(g, (*shape[:-1], (cols + 31) // 32), pad, skip, spread)
    scales += 126 - spread // 2
    return codes, scales


SIZES = [(1, 1, 1), (2, 3, 5), (1, 7, 32), (3, 5, 33), (1, 9, 64), (2, 4, 127), (1, 130, 96), (1, 3, 771), (2, 33, 784), (1, 2, 2050), (1, 1030, 40), (1, 3, 5001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_there_and_back(ops, size, dtype):   # noqa: F811
    n, rows, cols = size
    dt = TYPES[dtype]
    for k, (pad, skip) in enumerate(((0, 0), (3, 1), (16, 0))):
        g = torch.Generator().manual_seed(cols + k)
        x = rand(g, size, dt, pad=pad, skip=skip)
        x *= torch.exp2(torch.randint(-40, 40, (n, rows, 1), generator=g).float()).to(dt).to(DEV)   # rows of their own size
        x[0, 0, :1] = 0.0
        codes, scales = ops.aet_mx4_quantise(x)
        wc, ws = M.quantise(d64(x).reshape(n * rows, cols))
        assert torch.equal(scales.cpu().view(n * rows, -1), ws) and torch.equal(codes.cpu().view(n * rows, -1), wc)
        want = M.values(codes, scales, cols)
        for to in (torch.float32, torch.bfloat16):
            assert torch.equal(d64(ops.aet_mx4_dequantise(codes, scales, cols=cols, dtype=to)), want)
        # places of other strides, whose gaps stay as they are
        pc, ps = torch.full((n, rows, codes.shape[-1] + 3), 7, dtype=torch.uint8, device=DEV), torch.full((n, rows, scales.shape[-1] + 1), 7, dtype=torch.uint8, device=DEV)
        ops.aet_mx4_quantise(x, out=(pc[..., 1:-2], ps[..., 1:]))
        assert torch.equal(pc[..., 1:-2], codes) and torch.equal(ps[..., 1:], scales)
        assert bool((pc[..., 0] == 7).all() and (pc[..., -2:] == 7).all() and (ps[..., 0] == 7).all())
        py = torch.full((n, rows, cols + 3), 7.0, dtype=dt, device=DEV)
        ops.aet_mx4_dequantise(pc[..., 1:-2], ps[..., 1:], cols=cols, dtype=dt, out=py[..., 1:-2])
        assert torch.equal(d64(py[..., 1:-2]), want) and bool((py[..., 0] == 7).all() and (py[..., -2:] == 7).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_and_edges(ops, dtype):   # noqa: F811
    """Every border between neighbours, from both sides, at every exponent; subnormal and largest values; zeros of both signs."""
    dt = TYPES[dtype]
    t = torch.tensor([0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 7.0], dtype=torch.float64)
    eps = torch.finfo(dt).eps
    rows = []
    for x in list(range(-152, -118)) + [-1, 0, 1] + list(range(120, 128)):
        for near in (1.0, 1 - eps / 2, 1 + eps):
            v = torch.cat((t * near, -t * near)) * 2.0 ** (x - 2)
            rows.append(v[v.abs() < 3.38e38 if dt == torch.bfloat16 else v.abs() < 3.4028e38])
            rows[-1] = torch.cat((rows[-1], torch.zeros(32 - len(rows[-1]))))
    x = torch.stack(rows).to(dt).to(DEV)
    codes, scales = ops.aet_mx4_quantise(x)
    wc, ws = M.quantise(d64(x))
    assert torch.equal(scales.cpu(), ws) and torch.equal(codes.cpu(), wc)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_blocks_that_are_not_finite(ops, dtype):   # noqa: F811
    dt = TYPES[dtype]
    x = torch.ones(4, 100, dtype=dt, device=DEV)
    x[1, 40], x[2, 99], x[3, 0] = float("nan"), float("inf"), -float("inf")
    codes, scales = ops.aet_mx4_quantise(x)
    y = ops.aet_mx4_dequantise(codes, scales, dtype=dt)
    want = torch.ones(4, 100, dtype=torch.bool)
    want[1, 32:64], want[2, 96:], want[3, :32] = False, False, False
    assert torch.equal(y.cpu() == 1, want) and torch.equal(y.cpu().isnan(), ~want)


def test_every_code_and_scale(ops):   # noqa: F811
    codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1)[:, :, None].repeat(1, 1, 16).to(DEV)
    scales = torch.arange(256, dtype=torch.uint8)[:, None, None].repeat(1, 256, 1).to(DEV)
    want = M.values(codes, scales, 32)
    for dt in (torch.float32, torch.bfloat16):
        y = d64(ops.aet_mx4_dequantise(codes, scales, dtype=dt))
        fine = want.abs() < 2.0 ** 128
        assert torch.equal(y[fine], want[fine]) and torch.equal(y.isnan(), want.isnan())
        assert bool(torch.isinf(y[want.abs() >= 2.0 ** 128]).all())


# n, rows, in, out: single values and rows; sums that end inside a block, a byte, a step and a stage; odd sizes; rows and outputs that
# end inside tiles; more than one tile each way; long sums of few rows
LINEAR = [(1, 1, 1, 1), (1, 1, 784, 128), (3, 1, 50, 7), (1, 5, 1000, 33), (2, 16, 64, 16), (4, 17, 72, 130), (1, 33, 257, 65), (2, 64, 128, 96),
          (3, 100, 33, 200), (1, 129, 192, 128), (1, 256, 256, 256), (1, 300, 520, 264), (2, 257, 1155, 255), (1, 8, 4096, 48), (16, 32, 784, 128),
          (1, 511, 1024, 384), (1, 1024, 96, 10), (1, 40, 8, 1000), (1, 513, 2048, 640), (1, 2, 8200, 40)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", LINEAR, ids=str)
def test_linear(ops, size, dtype):   # noqa: F811
    n, rows, inp, out = size
    dt = TYPES[dtype]
    for k, (name, p, with_bias, with_res, pad, skip) in enumerate((("none", 0.0, False, False, 0, 0), ("gelu", 0.1, True, True, 0, 0),
                                                                   ("relu", 0.0, True, False, 1, 1), ("silu", 0.5, False, True, 16, 0))):
        g = torch.Generator().manual_seed(k + 10 * rows + out)
        (x, xs), (w, ws) = held(g, (n, rows, inp), pad, skip), held(g, (n, out, inp), pad, skip)
        b = rand(g, (n, out), dt) if with_bias else None
        res = rand(g, (n, rows, out), dt, pad=pad, skip=skip) if with_res else None
        y, pre = ops.aet_mx4_linear_forward(x, xs, w, ws, b, cols=inp, residual=res, act=name, p=p, seed=7 + k, first_row=3, keep_pre=True, dtype=dt)
        vx, vw = M.values(x, xs, inp), M.values(w, ws, inp)
        wy, wz = O.linear_forward(vx, vw, d64(b), d64(res), name, p, 7 + k, 3, dt)
        what = f"{size} {dtype} {name}"
        O.near(pre, wz, "pre " + what)
        O.near(y, wy, "y " + what)
        dy = rand(g, (n, rows, out), dt, pad=pad, skip=skip)
        got = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, cols=inp, act=name, p=p, seed=7 + k, first_row=3)
        for t, want, part in zip(got, O.linear_backward(d64(dy), vx, vw, d64(pre), name, p, 7 + k, 3, dt), ("dx", "dw", "db")):
            O.near(t, want, f"{part} {what}")


# Sizes at which the gradient takes all operands in fp16: odd ones, several clients, rows and columns that end inside tiles and pieces
LARGE = [(1, 2055, 1031, 1543), (3, 1030, 1030, 1030), (1, 4096, 520, 2048), (16, 257, 512, 1000)]
WIDE = [(1, 1500, 1024, 1500), (1, 2600, 1024, 2500)]


def gradient(dy, vx, vw, pre, name, p, seed, dt):
    """Like the oracle's, which multiplies in 64 bits: on the GPU, for the time that it takes."""
    m = O.mask3(dy.shape, seed, 0, p) if p else 1.0
    dz = dy * m * (O.slope(pre, name) if name != "none" else 1.0)
    off = dz.abs() * ((4 * 1.13 + 10 * (pre.abs() + 1)) * O.U32 if name in ("silu", "gelu") else 4 * O.U32)
    # dz as the products see it: in bf16 one fp16 value, which is off by half a step, torch.finfo(torch.float16).eps / 2 = 2^-11 (or two bf16
    # ones), in fp32 two, the second of which is off by 2^-11 of the at most 2^-11 that the first leaves
    dzr = off + dz.abs() * (2.0 ** -11 if dt == torch.bfloat16 else 2.0 ** -22)
    r = O.ROUND[dt]

    def product(a, aoff, b):
        g = [t.to(DEV) for t in (a, aoff, b)]
        v, S = torch.matmul(g[0], g[2]).cpu(), torch.matmul(g[0].abs(), g[2].abs()).cpu()
        o = torch.matmul(g[1], g[2].abs()).cpu() + (a.shape[-1] + 4) * O.U32 * S
        return v, o + r * (v.abs() + o)

    t = lambda v: v.transpose(1, 2).contiguous()   # noqa: E731
    db = dz.sum(1)
    o = off.sum(1) + (dz.shape[1] + 4) * O.U32 * dz.abs().sum(1)
    return product(dz, dzr, vw), product(t(dz), t(dzr), vx), (db, o + r * (db.abs() + o))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", LARGE, ids=str)
def test_large_gradients(ops, size, dtype):   # noqa: F811
    n, rows, inp, out = size
    dt = TYPES[dtype]
    for k, (name, p, pad, skip) in enumerate((("silu", 0.0, 0, 0), ("gelu", 0.3, 1, 1), ("none", 0.0, 0, 0))):
        g = torch.Generator().manual_seed(k + rows)
        (x, xs), (w, ws) = held(g, (n, rows, inp), pad, skip), held(g, (n, out, inp), pad, skip)
        dy, pre = rand(g, (n, rows, out), dt, 1e-3, pad, skip), rand(g, (n, rows, out), dt, pad=pad, skip=skip)
        want = gradient(d64(dy), M.values(x, xs, inp), M.values(w, ws, inp), d64(pre), name, p, 5, dt)
        got = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, cols=inp, act=name, p=p, seed=5)
        for t, q, part in zip(got, want, ("dx", "dw", "db")):
            O.near(t, q, f"{part} {size} {dtype} {name}")
        for need in ((True, False, False), (False, True, True)):
            some = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, cols=inp, act=name, p=p, seed=5, need=need)
            for t, q, yes in zip(some, want, need):
                assert (t is None) != yes
                if yes:
                    O.near(t, q, f"{need} {size} {dtype} {name}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", WIDE, ids=str)
def test_large_gradients_of_rows_of_all_sizes(ops, size, dtype):   # noqa: F811
    """Rows of dz, of x and of W whose sizes are 2^-50 to 2^50 of each other, a row of zeros each, and blocks of zeros with the largest scale."""
    dt = TYPES[dtype]
    n, rows, inp, out = size
    g = torch.Generator().manual_seed(3)
    (x, xs), (w, ws) = held(g, (n, rows, inp)), held(g, (n, out, inp))
    for t in (xs, ws):
        t += torch.randint(-50, 50, (n, t.shape[1], 1), generator=g, dtype=torch.int8).to(torch.uint8).to(DEV)
    for c, s in ((x, xs), (w, ws)):
        c[0, 7] = 0
        c[0, 9, 16:32] = 0x80   # a block of zeros
        s[0, 9, 1] = 254
    dy = rand(g, (n, rows, out), dt) * torch.exp2(torch.randint(-20, 20, (n, rows, 1), generator=g).float()).to(dt).to(DEV)
    dy[0, 11] = 0
    pre = rand(g, (n, rows, out), dt)
    want = gradient(d64(dy), M.values(x, xs, inp), M.values(w, ws, inp), d64(pre), "silu", 0.0, 5, dt)
    got = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, act="silu")
    for t, (v, bound), part in zip(got, want, ("dx", "dw", "db")):
        # (beside the bound: 2^-39 of the largest term of the row of the contraction, for each)
        room = 2.0 ** -39 * v.abs().amax(-1, keepdim=True) * max(rows, out) if part != "db" else 0
        O.near(t, (v, bound + room), part)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", WIDE, ids=str)
def test_large_gradients_beside_rows_of_zeros(ops, size, dtype):   # noqa: F811
    """Every second row of W and x is zeros, the others are tiny: what the zeros have for a scale is no matter."""
    dt = TYPES[dtype]
    n, rows, inp, out = size
    g = torch.Generator().manual_seed(3)
    (x, xs), (w, ws) = held(g, (n, rows, inp)), held(g, (n, out, inp))
    for c, s in ((x, xs), (w, ws)):
        s -= 70
        c[:, ::2] = 0
    dy, pre = rand(g, (n, rows, out), dt), rand(g, (n, rows, out), dt)
    want = gradient(d64(dy), M.values(x, xs, inp), M.values(w, ws, inp), d64(pre), "silu", 0.0, 5, dt)
    got = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, act="silu")
    for t, (v, bound), part in zip(got, want, ("dx", "dw", "db")):
        # (beside the bound: 2^-39 of the largest term of the row of the contraction, for each)
        room = 2.0 ** -39 * v.abs().amax(-1, keepdim=True) * max(rows, out) if part != "db" else 0
        O.near(t, (v, bound + room), part)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", WIDE, ids=str)
def test_large_gradients_of_blocks_of_all_sizes(ops, size, dtype):   # noqa: F811
    """Neighbouring blocks of W and x, whose scales are 2^-34 to 1 of the row's largest: each column of a product sees only its own blocks,
    and dz is in as many bits for all of them."""
    dt = TYPES[dtype]
    n, rows, inp, out = size
    g = torch.Generator().manual_seed(3)
    (x, xs), (w, ws) = held(g, (n, rows, inp)), held(g, (n, out, inp))
    for t in (xs, ws):   # the same for all rows: a row of the contraction has its large blocks where the others have
        t.copy_((127 - 34 * torch.arange(inp // 32) // (inp // 32 - 1)).to(torch.uint8).expand(t.shape))
    dy, pre = rand(g, (n, rows, out), dt), rand(g, (n, rows, out), dt)
    want = gradient(d64(dy), M.values(x, xs, inp), M.values(w, ws, inp), d64(pre), "silu", 0.0, 5, dt)
    got = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, act="silu")
    for t, q, part in zip(got, want, ("dx", "dw", "db")):
        O.near(t, q, part)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", WIDE, ids=str)
def test_large_gradients_that_are_not_finite(ops, size, dtype):   # noqa: F811
    dt = TYPES[dtype]
    n, rows, inp, out = size
    g = torch.Generator().manual_seed(3)
    (x, xs), (w, ws) = held(g, (n, rows, inp)), held(g, (n, out, inp))
    dy, pre = rand(g, (n, rows, out), dt), rand(g, (n, rows, out), dt)
    want = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, act="gelu")
    dy[0, 3, 5] = float("nan")
    xs[0, 10, 2], ws[0, 20, 4] = 255, 255
    dx, dw, db = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, act="gelu")
    fine = torch.ones(rows, inp, dtype=torch.bool, device=DEV)
    fine[3], fine[:, 128:160] = False, False
    assert bool(dx[0][~fine].isnan().all()) and torch.equal(dx[0][fine], want[0][0][fine])
    fine = torch.ones(out, inp, dtype=torch.bool, device=DEV)
    fine[5], fine[:, 64:96] = False, False
    assert bool(dw[0][~fine].isnan().all()) and torch.equal(dw[0][fine], want[1][0][fine])
    assert bool(db[0, 5].isnan()) and int(db.isnan().sum()) == 1


def test_large_gradient_of_one_w_for_all_clients(ops):   # noqa: F811
    g = torch.Generator().manual_seed(4)
    n, rows, inp, out = 5, 400, 512, 1024
    (x, xs), (w, ws) = held(g, (n, rows, inp)), held(g, (out, inp))
    dy, pre = rand(g, (n, rows, out), torch.bfloat16), rand(g, (n, rows, out), torch.bfloat16)
    flat = lambda t: t.reshape(1, n * rows, t.shape[-1])   # noqa: E731
    want = gradient(flat(d64(dy)), flat(M.values(x, xs, inp)), M.values(w, ws, inp)[None], flat(d64(pre)), "gelu", 0.0, 0, torch.bfloat16)
    apart = torch.zeros(n, rows + 3, inp // 2, dtype=torch.uint8, device=DEV)[:, :rows]   # held inputs of clients that lie apart
    apart.copy_(x)
    for held_x in (x, apart):
        dx, dw, db = ops.aet_mx4_linear_backward(dy, held_x, xs, w, ws, pre, act="gelu")
        for t, q, part in zip((flat(dx), dw[None], db[None]), want, ("dx", "dw", "db")):
            O.near(t, q, part)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 40])
def test_one_w_for_all_clients(ops, dtype, rows):   # noqa: F811
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(4)
    (x, xs), (w, ws) = held(g, (5, rows, 96)), held(g, (24, 96))
    b, dy = rand(g, (24,), dt), rand(g, (5, rows, 24), dt)
    vx, vw = M.values(x, xs, 96), M.values(w, ws, 96)
    want, _ = O.linear_forward(vx, vw.expand(5, 24, 96), d64(b).expand(5, 24), None, "relu", 0.0, 0, 0, dt)
    y, pre = ops.aet_mx4_linear_forward(x, xs, w, ws, b, act="relu", keep_pre=True, dtype=dt)
    O.near(y, want, "y")
    apart, aparts = torch.zeros(5, rows + 2, 48, dtype=torch.uint8, device=DEV)[:, :rows], torch.zeros(5, rows + 1, 3, dtype=torch.uint8, device=DEV)[:, 1:]
    apart.copy_(x)
    aparts.copy_(xs)
    O.near(ops.aet_mx4_linear_forward(apart, aparts, w, ws, b, act="relu", dtype=dt)[0], want, "y of clients that lie apart")
    got = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, act="relu")
    flat = lambda t: t.reshape(1, 5 * rows, t.shape[-1])   # noqa: E731
    wants = O.linear_backward(flat(d64(dy)), flat(vx), vw[None], flat(d64(pre)), "relu", 0.0, 0, 0, dt)
    O.near(got[0].view(1, 5 * rows, 96), wants[0], "dx")
    O.near(got[1][None], wants[1], "dw")
    O.near(got[2][None], wants[2], "db")


def test_large_gradient_captured_and_replayed(ops):   # noqa: F811
    g = torch.Generator().manual_seed(6)
    (x, xs), (w, ws) = held(g, (1500, 1024)), held(g, (1500, 1024))
    dy, pre = rand(g, (1500, 1500), torch.bfloat16), rand(g, (1500, 1500), torch.bfloat16)
    step = lambda: ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, act="silu")   # noqa: E731
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        dy.copy_(rand(g, (1500, 1500), torch.bfloat16, 10.0 ** -k))   # (tops of the last replay must not stay)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, step())), k


@pytest.mark.parametrize("rows", [3, 70, 300])
def test_nan_in_a_block_is_in_its_rows_products(ops, rows):   # noqa: F811
    """A block of inputs that is NaN makes its row NaN, one of weights its output; scales behind the end of a row do not count."""
    g = torch.Generator().manual_seed(8)
    (x, xs), (w, ws) = held(g, (rows, 200), pad=24), held(g, (70, 200), pad=24)
    for t in (xs, ws):   # what lies between the rows: NaN
        t.as_strided((t.shape[0], 24), (t.stride(0), 1), t.storage_offset() + t.shape[1])[:-1] = 255
    y, _ = ops.aet_mx4_linear_forward(x, xs, w, ws, cols=200)
    assert bool(y.isfinite().all())
    xs[1, 6] = 255
    x[1, 96:] = 0
    ws[5, 0] = 255
    bad, _ = ops.aet_mx4_linear_forward(x, xs, w, ws, cols=200)
    fine = torch.ones(rows, 70, dtype=torch.bool, device=DEV)
    fine[1], fine[:, 5] = False, False
    assert bool(bad[~fine].isnan().all()) and torch.equal(bad[fine], y[fine])


def test_largest_and_smallest_scales(ops):   # noqa: F811
    g = torch.Generator().manual_seed(8)
    for rows, sx, sw in ((2, 0, 250), (2, 252, 3), (80, 0, 250), (80, 252, 3)):
        (x, xs), (w, ws) = held(g, (1, rows, 128)), held(g, (1, 40, 128))
        xs.fill_(sx)
        ws.fill_(sw)
        y, _ = ops.aet_mx4_linear_forward(x, xs, w, ws, dtype=torch.float32)
        O.near(y, O.linear_forward(M.values(x, xs, 128), M.values(w, ws, 128), None, None, "none", 0.0, 0, 0, torch.float32)[0], f"{sx} {sw}")


def test_nothing_to_add(ops):   # noqa: F811
    z = lambda *s: torch.zeros(*s, dtype=torch.uint8, device=DEV)   # noqa: E731
    b = torch.arange(4.0, device=DEV)
    y, _ = ops.aet_mx4_linear_forward(z(3, 0), z(3, 0), z(4, 0), z(4, 0), b, dtype=torch.float32)
    assert torch.equal(y, b.expand(3, 4))
    y, _ = ops.aet_mx4_linear_forward(z(0, 8), z(0, 1), z(4, 8), z(4, 1), b, dtype=torch.float32)
    assert y.shape == (0, 4)
    dx, dw, db = ops.aet_mx4_linear_backward(torch.ones(0, 4, device=DEV), z(0, 8), z(0, 1), z(4, 8), z(4, 1))
    assert dx.shape == (0, 16) and bool((dw == 0).all() and (db == 0).all())
    dx, dw, db = ops.aet_mx4_linear_backward(torch.ones(3, 4, device=DEV), z(3, 0), z(3, 0), z(4, 0), z(4, 0))
    assert dx.shape == (3, 0) and dw.shape == (4, 0) and bool((db == 3).all())
    c, s = ops.aet_mx4_quantise(torch.ones(2, 0, 5, device=DEV))
    assert c.shape == (2, 0, 3) and s.shape == (2, 0, 1) and ops.aet_mx4_dequantise(c, s, cols=5).shape == (2, 0, 5)


def test_sums_over_nothing(ops):   # noqa: F811
    """No clients with one W for all of them: its gradients are 0.  And what is not looked at need not be there."""
    z = lambda *s: torch.zeros(*s, dtype=torch.uint8, device=DEV)   # noqa: E731
    places = [torch.full(s, 7.0, device=DEV) for s in ((4, 16), (4,))]
    dx, dw, db = ops.aet_mx4_linear_backward(torch.ones(0, 5, 4, device=DEV), z(0, 5, 8), z(0, 5, 1), z(4, 8), z(4, 1), out=(None, *places))
    assert dx.shape == (0, 5, 16) and dw is places[0] and bool((dw == 0).all() and (db == 0).all())
    lib, stream = ops.load_library(), torch.cuda.current_stream().cuda_stream
    for rows, out in ((0, 4), (3, 0)):
        dx, dw, db = (torch.full(s, 7.0, device=DEV) for s in ((2, max(rows, 1), 16), (2, max(out, 1), 16), (2, max(out, 1))))
        a = ops.aet_mx4_linear_grad(0, 0, 2, rows, 16, out)
        for f, t in (("dx", dx), ("dw", dw), ("db", db)):
            setattr(a, f + "_p", t.data_ptr())
            setattr(a, f + "_client", t.stride(0))
            setattr(a, f + "_row", 16)
        need = lib.aet_mx4_linear_backward_workspace_bytes(C.addressof(a))
        space = torch.empty(max(need, 1), dtype=torch.uint8, device=DEV)
        assert lib.aet_mx4_linear_backward(C.addressof(a), space.data_ptr(), need, stream) == 0
        assert bool((dx == (0 if rows else 7)).all() and (dw == (0 if out else 7)).all() and (db == (0 if out else 7)).all())


def test_what_is_wanted(ops):   # noqa: F811
    g = torch.Generator().manual_seed(2)
    (x, xs), (w, ws) = held(g, (2, 70, 96)), held(g, (2, 40, 96))
    dy = rand(g, (2, 70, 40), torch.bfloat16)
    want = ops.aet_mx4_linear_backward(dy, x, xs, w, ws)
    for need in ((True, False, False), (False, True, False), (False, False, True), (True, False, True)):
        got = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, need=need)
        for t, q, yes in zip(got, want, need):
            assert torch.equal(t, q) if yes else t is None


def test_the_layer_is_the_linear_layer_of_what_the_codes_stand_for(ops):   # noqa: F811
    """Gradients against differences: of the definition, by one step of a code each way."""
    g = torch.Generator().manual_seed(11)
    (x, xs), (w, ws) = held(g, (6, 64)), held(g, (5, 64))
    dy = rand(g, (6, 5), torch.float32)
    dx, dw, _ = ops.aet_mx4_linear_backward(dy, x, xs, w, ws)
    f = lambda vx, vw: float((vx @ vw.t() * d64(dy)).sum())   # noqa: E731
    vx, vw = M.values(x, xs, 64), M.values(w, ws, 64)
    for v, got, which in ((vx, dx, 0), (vw, dw, 1)):
        for i in range(0, v.numel(), 7):
            up = v.clone()
            up.view(-1)[i] += 2.0   # the function is linear in each
            d = (f(up, vw) if which == 0 else f(vx, up)) - f(vx, vw)
            assert abs(d / 2 - float(got.view(-1)[i])) <= 1e-5 * float((d64(dy).abs().sum() * max(vx.abs().max(), vw.abs().max())))


def test_captured_and_replayed_with_other_calls(ops):   # noqa: F811
    g = torch.Generator().manual_seed(6)
    x, dy = rand(g, (300, 200), torch.bfloat16), rand(g, (300, 264), torch.bfloat16)
    w, ws = held(g, (264, 200))

    def step():
        c, s = ops.aet_mx4_quantise(x)
        y, pre = ops.aet_mx4_linear_forward(c, s, w, ws, act="gelu", keep_pre=True)
        row, _ = ops.aet_mx4_linear_forward(c[:1], s[:1], w, ws)
        return (y, row, *ops.aet_mx4_linear_backward(dy, c, s, w, ws, pre, act="gelu"))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        x.copy_(rand(g, (300, 200), torch.bfloat16))
        dy.mul_(1.25)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, step())), k


def test_other_streams(ops):   # noqa: F811
    g = torch.Generator().manual_seed(6)
    x = rand(g, (300, 200), torch.bfloat16)
    w, ws = held(g, (264, 200))

    def step(stream):
        c, s = ops.aet_mx4_quantise(x, stream=stream)
        y, pre = ops.aet_mx4_linear_forward(c, s, w, ws, act="gelu", keep_pre=True, stream=stream)
        return (c, s, y, ops.aet_mx4_dequantise(c, s, stream=stream), *ops.aet_mx4_linear_backward(y, c, s, w, ws, pre, act="gelu", stream=stream))

    want = step(None)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = step(other)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))


def calls(ops):   # noqa: F811
    z = lambda *s: torch.ones(*s, device=DEV)   # noqa: E731
    u = lambda *s: torch.ones(*s, dtype=torch.uint8, device=DEV)   # noqa: E731
    return {
        "quantise": (lambda x, codes, scales: ops.aet_mx4_quantise(x, out=(codes, scales)), dict(x=z(2, 3, 64), codes=u(2, 3, 32), scales=u(2, 3, 2))),
        "dequantise": (lambda codes, scales, out: ops.aet_mx4_dequantise(codes, scales, dtype=torch.float32, out=out),
                       dict(codes=u(2, 3, 32), scales=u(2, 3, 2), out=z(2, 3, 64))),
        "forward": (lambda x, x_scales, w, w_scales, bias, residual, out: ops.aet_mx4_linear_forward(
            x, x_scales, w, w_scales, bias, residual=residual, dtype=torch.float32, out=out),
            dict(x=u(2, 3, 32), x_scales=u(2, 3, 2), w=u(2, 5, 32), w_scales=u(2, 5, 2), bias=z(2, 5), residual=z(2, 3, 5), out=z(2, 3, 5))),
        "backward": (lambda dy, x, x_scales, w, w_scales, pre, dx, dw, db: ops.aet_mx4_linear_backward(
            dy, x, x_scales, w, w_scales, pre, act="silu", out=(dx, dw, db)),
            dict(dy=z(2, 3, 5), x=u(2, 3, 32), x_scales=u(2, 3, 2), w=u(2, 5, 32), w_scales=u(2, 5, 2), pre=z(2, 3, 5), dx=z(2, 3, 64), dw=z(2, 5, 64),
                 db=z(2, 5)))}


PLACES = {"quantise": ["codes", "scales"], "dequantise": ["out"], "forward": ["out"], "backward": ["dx", "dw", "db"]}


@pytest.mark.parametrize("name", sorted(PLACES))
def test_binding(ops, name):   # noqa: F811
    call, tensors = calls(ops)[name]
    before = {k: t._version for k, t in tensors.items()}
    call(**tensors)
    assert all((t._version > before[k]) == (k in PLACES[name]) for k, t in tensors.items())
    for k, t in tensors.items():
        if t.is_floating_point():
            with pytest.raises(ValueError, match="requires a gradient"):
                call(**dict(tensors, **{k: t.clone().requires_grad_()}))
        for bad in (t.half(), t.cpu(), t.new_zeros(*t.shape, 2)[..., 0], t.new_zeros(*t.shape[:-1], t.shape[-1] + 1), t[None, None]):
            if k == "x" and name == "quantise" and bad.dim() == 3 and bad.is_cuda and bad.dtype == t.dtype and bad.stride(-1) == 1:
                continue   # says the size itself; the others do not agree with it then
            with pytest.raises(ValueError):
                call(**dict(tensors, **{k: bad}))
    torch.cuda.synchronize()


def test_arguments_that_do_not_agree(ops):   # noqa: F811
    from paper_2112_13935_amd import AetError
    u = lambda *s: torch.ones(*s, dtype=torch.uint8, device=DEV)   # noqa: E731
    with pytest.raises(ValueError, match="columns"):
        ops.aet_mx4_dequantise(u(3, 4), u(3, 1), cols=6)
    with pytest.raises(ValueError, match="dtype"):
        ops.aet_mx4_dequantise(u(3, 4), u(3, 1), dtype=torch.float16)
    with pytest.raises(ValueError, match="w: "):
        ops.aet_mx4_linear_forward(u(3, 4), u(3, 1), u(4), u(1))
    with pytest.raises(ValueError, match="scales"):
        ops.aet_mx4_linear_forward(u(3, 32), u(3, 1), u(4, 32), u(4, 2))
    with pytest.raises(ValueError, match="pre"):
        ops.aet_mx4_linear_backward(torch.ones(3, 4, device=DEV), u(3, 4), u(3, 1), u(4, 4), u(4, 1), act="gelu")
    with pytest.raises(ValueError, match="act is one of"):
        ops.aet_mx4_linear_forward(u(3, 4), u(3, 1), u(4, 4), u(4, 1), act="tanh")
    with pytest.raises(AetError, match="p is not in"):
        ops.aet_mx4_linear_forward(u(3, 4), u(3, 1), u(4, 4), u(4, 1), p=1.0)
    with pytest.raises(AetError, match="overlaps itself"):
        ops.aet_mx4_quantise(torch.ones(3, 8, device=DEV), out=(u(1, 4).expand(3, 4), None))
    with pytest.raises(AetError, match="client after client"):
        ops.aet_mx4_linear_backward(torch.ones(2, 4, 5, device=DEV)[:, :3], u(2, 3, 4), u(2, 3, 1), u(5, 4), u(5, 1))
