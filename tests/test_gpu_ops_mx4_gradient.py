"""The gradient of the linear layer of 4-bit values where its products' operands are hard to hold: blocks of zeros of any scale, differences of
nearly equal terms, blocks far below their row's largest."""
import pytest
import torch

import mx4_oracle as M
import ops_oracle as O
from test_gpu_ops_linear import DEV, TYPES, d64, ops, rand  # noqa: F401
from test_gpu_ops_mx4 import held

pytestmark = pytest.mark.gpu

# rows, in, out: small; and of several tiles each way
SIZES = [(600, 96, 610), (2600, 1024, 2500)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_zeros_of_every_scale(ops, size, dtype):   # noqa: F811
    """A block of zeros is zeros whatever its scale says (but NaN), beside a block with values and in a row of nothing else."""
    rows, inp, out = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(1)
    (x, xs), (w, ws) = held(g, (rows, inp)), held(g, (out, inp))
    dy, pre = rand(g, (rows, out), dt), rand(g, (rows, out), dt)
    every = torch.arange(255, dtype=torch.uint8, device=DEV)
    for c, s in ((x, xs), (w, ws)):
        s.fill_(100)
        c[:255, 16:32] = torch.tensor([0, 0x80, 0x08, 0x88] * 4, dtype=torch.uint8, device=DEV)
        c[300:555] = 0
    want = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, act="silu")
    for s in (xs, ws):
        s[:255, 1] = every
        s[300:555] = every[:, None]
    got = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, act="silu")
    assert all(bool(t.isfinite().all()) and torch.equal(t, q) for t, q in zip(got, want))


def held_differences(rows, cols):
    """Codes and scales of a matrix whose column i is 1 in row 2 i and -1 in row 2 i + 1."""
    v = torch.zeros(rows, cols, dtype=torch.uint8, device=DEV)
    i = torch.arange(min(cols, rows // 2), device=DEV)
    v[2 * i, i], v[2 * i + 1, i] = 0x2, 0xA
    return v[:, 0::2] | v[:, 1::2] << 4, torch.full((rows, (cols + 31) // 32), 127, dtype=torch.uint8, device=DEV)


def pairs(g, shape, dt):
    """Values of which neighbouring rows, and columns, differ by some percent."""
    v = torch.randn(shape[0] // 2, shape[1] // 2, generator=g).repeat_interleave(2, 0).repeat_interleave(2, 1)
    v[1::2] *= 1 + 2.0 ** -6
    v[:, 1::2] *= 1 - 2.0 ** -5
    return v.to(dt).to(DEV)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_differences_of_nearly_equal_terms(ops, size, dtype):   # noqa: F811
    """What a product takes of dz shows where its terms cancel: in bf16 two bf16 values (2^-16 of it), in fp32 all 24 bits."""
    rows, inp, out = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(2)
    x, w = held_differences(rows, inp), held_differences(out, inp)
    dy, pre = pairs(g, (rows, out), dt), pairs(g, (rows, out), dt)
    dx, dw, _ = ops.aet_mx4_linear_backward(dy, *x, *w, pre, act="silu")
    dz = d64(dy) * O.slope(d64(pre), "silu")
    # dz itself as the oracle bounds it (the slope, which may be near 0, is off by up to 10 U32 (|z| + 1), not by a share of it: that times dy),
    # and its parts; a sum of two terms, of up to three parts each
    off = d64(dy).abs() * (4 * 1.13 + 10 * (d64(pre).abs() + 1)) * O.U32 + dz.abs() * (2.0 ** -16 if dt == torch.bfloat16 else O.U32)
    for got, d, o in ((dx, dz, off), (dw, dz.t(), off.t())):
        n = min(inp, d.shape[1] // 2)
        v, b = d[:, :2 * n:2] - d[:, 1:2 * n:2], (o + 6 * O.U32 * d.abs())
        b = b[:, :2 * n:2] + b[:, 1:2 * n:2]
        O.near(got[:, :n], (v, b + O.ROUND[dt] * (v.abs() + b)), "sums of two")
        assert not bool(got[:, n:].any())


def tiny_blocks(g, rows, cols):
    """Codes without zeros, whose second blocks are 2^-60 and whose third ones 2^-45 of the others."""
    codes = torch.randint(1, 8, (rows, cols), generator=g, dtype=torch.uint8)
    codes += 8 * torch.randint(0, 2, (rows, cols), generator=g, dtype=torch.uint8)
    scales = torch.full((rows, cols // 32), 127, dtype=torch.uint8)
    scales[:, 1], scales[:, 2] = 67, 82
    return (codes[:, 0::2] | codes[:, 1::2] << 4).to(DEV), scales.to(DEV)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_blocks_far_below_their_rows_largest(ops, size, dtype):   # noqa: F811
    """Columns of W, and of x, are sums of their own: that others are 2^60 times as large is no matter to them."""
    rows, inp, out = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(3)
    x, w = tiny_blocks(g, rows, inp), tiny_blocks(g, out, inp)
    dy = rand(g, (rows, out), dt)
    dy[3] *= 2.0 ** -50
    dx, dw, _ = ops.aet_mx4_linear_backward(dy, *x, *w)
    d, vx, vw = (t.to(DEV) for t in (d64(dy), M.values(*x, inp), M.values(*w, inp)))
    for got, a, b in ((dx, d, vw), (dw, d.t().contiguous(), vx)):
        v = a @ b
        # dz is held whole; three parts of each term at most, in fp32
        off = (3 * a.shape[1] + 4) * O.U32 * (a.abs() @ b.abs())
        O.near(got, (v.cpu(), (off + O.ROUND[dt] * (v.abs() + off)).cpu()), "with tiny blocks")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_an_infinite_gradient_beside_tiny_blocks(ops, size, dtype):   # noqa: F811
    """Infinity times a value that is not 0 is infinity, however small the value."""
    rows, inp, out = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(3)
    x, w = tiny_blocks(g, rows, inp), tiny_blocks(g, out, inp)
    dy = rand(g, (rows, out), dt)
    dy[4, 7] = float("inf")
    dx, dw, _ = ops.aet_mx4_linear_backward(dy, *x, *w)
    assert torch.equal(dx[4].double().cpu(), float("inf") * M.values(*w, inp)[7].sign())
    assert torch.equal(dw[7].double().cpu(), float("inf") * M.values(*x, inp)[4].sign())
    assert bool(dx[5:].isfinite().all() and dw[8:].isfinite().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("scale,power", [(254, -40), (253, -40), (0, 100), (1, 100), (2, 100)])
def test_largest_and_smallest_scales(ops, size, act, dtype, scale, power):   # noqa: F811
    """Codes stand for values beyond fp32's largest, and below its smallest normal one, whose gradients are ordinary."""
    rows, inp, out = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(4)
    (x, xs), (w, ws) = held(g, (rows, inp)), held(g, (out, inp))
    for s in (xs, ws):
        s.fill_(scale)
    dy, pre = rand(g, (rows, out), dt, 2.0 ** power), rand(g, (rows, out), dt)
    dx, dw, _ = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, act=act)
    d = d64(dy) * (O.slope(d64(pre), act) if act != "none" else 1.0)
    doff = d64(dy).abs() * (4 * 1.13 + 10 * (d64(pre).abs() + 1)) * O.U32 + (d.abs() * 2.0 ** -16 if dt == torch.bfloat16 and act != "none" else 0)
    d, doff, vx, vw = (t.to(DEV) for t in (d, doff, M.values(x, xs, inp), M.values(w, ws, inp)))
    for got, a, o, b in ((dx, d, doff, vw), (dw, d.t().contiguous(), doff.t().contiguous(), vx)):
        v = a @ b
        off = o @ b.abs() + (3 * a.shape[1] + 4) * O.U32 * (a.abs() @ b.abs())
        O.near(got, (v.cpu(), (off + O.ROUND[dt] * (v.abs() + off)).cpu()), f"scales of {scale}")


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 1000, 64, 64), (1, 700, 96, 130), (1, 40, 64, 1500), (16, 257, 512, 1000), (3, 1030, 1030, 1030), (2, 2055, 512, 1543)], ids=str)
def test_results_do_not_depend_on_what_else_is_wanted(ops, size, dtype, act):   # noqa: F811
    n, rows, inp, out = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(5)
    (x, xs), (w, ws) = held(g, (n, rows, inp)), held(g, (n, out, inp))
    dy, pre = rand(g, (n, rows, out), dt), rand(g, (n, rows, out), dt)
    want = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, act=act)
    for need in ((True, False, False), (False, True, False), (False, False, True), (False, True, True), (True, True, False)):
        got = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, act=act, need=need)
        assert all(torch.equal(t, q) if yes else t is None for t, q, yes in zip(got, want, need)), need


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype,act", [("f32", "none"), ("f32", "silu"), ("bf16", "none"), ("bf16", "silu")])
def test_the_largest_gradients(ops, size, act, dtype):   # noqa: F811
    """A finite dz is finite in the products, also where its first part by itself would round to infinity."""
    rows, inp, out = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(6)
    (x, xs), (w, ws) = held(g, (rows, inp)), held(g, (out, inp))
    for s in (xs, ws):
        s.fill_(127 - 40)
    most = torch.finfo(dt).max
    dy = torch.where(torch.rand(rows, out, generator=g) < 0.5, most, -most).to(dt).to(DEV)
    pre = torch.full((rows, out), 30.0, dtype=dt, device=DEV)   # where SiLU's slope is 1
    dx, dw, db = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, act=act)
    d, vx, vw = (t.to(DEV) for t in (d64(dy), M.values(x, xs, inp), M.values(w, ws, inp)))
    for got, a, b in ((dx, d, vw), (dw, d.t().contiguous(), vx)):
        v, S = a @ b, a.abs() @ b.abs()
        off = ((3 * a.shape[1] + 4) * O.U32 + (2.0 ** -16 if dt == torch.bfloat16 else 2 * O.U32)) * S
        assert bool(((got.double() - v).abs() <= off + O.ROUND[dt] * (v.abs() + off)).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_what_the_dropout_took_out_has_no_gradient(ops, size, dtype):   # noqa: F811
    """Whatever dy and z are there: infinities and NaN do not come through."""
    rows, inp, out = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(7)
    (x, xs), (w, ws) = held(g, (rows, inp)), held(g, (out, inp))
    dy, pre = rand(g, (rows, out), dt), rand(g, (rows, out), dt)
    gone = ops.aet_dropout_forward(torch.ones(rows, out, dtype=dt, device=DEV), p=0.4, seed=9, first_row=2) == 0
    want = ops.aet_mx4_linear_backward(torch.where(gone, 0, dy), x, xs, w, ws, torch.where(gone, 0, pre), act="gelu", p=0.4, seed=9, first_row=2)
    bad = [torch.where(gone, v, t) for t, v in ((dy, float("inf")), (pre, float("nan")))]
    got = ops.aet_mx4_linear_backward(bad[0], x, xs, w, ws, bad[1], act="gelu", p=0.4, seed=9, first_row=2)
    assert bool(gone.any()) and all(torch.equal(a, b) for a, b in zip(got, want))
