"""How near the operators come to their definitions in 64 bits where a bound of the worst case says little: the rounding
errors of whole tensors."""
import pytest
import torch

import ops_oracle as O
from test_ops_bounds import product_norm
from test_gpu_ops_linear import DEV, TYPES, d64, ops, rand  # noqa: F401

pytestmark = pytest.mark.gpu


# n, rows, in, out: the pair of small products, tiles of each kind, sums in slices, ends inside stages, rows that are no whole
# pieces (through registers)
GRADIENTS = [(2, 40, 96, 64), (3, 64, 784, 128), (1, 300, 520, 264), (1, 129, 72, 1000), (1, 4096, 64, 40), (2, 257, 129, 255), (1, 640, 640, 640),
             (2, 1032, 520, 1032)]


@pytest.mark.parametrize("size", GRADIENTS, ids=str)
@pytest.mark.parametrize("name,p", [("gelu", 0.1), ("silu", 0.0), ("none", 0.25)])
def test_gradients_in_bf16_are_rounded_once(ops, size, name, p):   # noqa: F811
    """dx and dw are the sums over the fp32 dz, rounded to bf16: what comes before the one rounding is within 2^-16 of dz, and the
    rounding of the products' sums in fp32, per value and in the 2-norm (where 2^-16 beside 2^-9 adds less than a thousandth;
    2 % are allowed for)."""
    n, rows, inp, out = size
    bf16 = torch.bfloat16
    g = torch.Generator().manual_seed(rows + out)
    x, w = rand(g, (n, rows, inp), bf16), rand(g, (n, out, inp), bf16, inp ** -0.5)
    dy, pre = rand(g, (n, rows, out), bf16), rand(g, (n, rows, out), bf16) if name != "none" else None
    dx, dw, _ = ops.aet_linear_backward(dy, x, w, pre, act=name, p=p, seed=5)
    dz = d64(dy) * O.mask3(dy.shape, 5, 0, p)
    off = (2.0 ** -16 + 4 * O.U32) * dz.abs()
    if name != "none":
        off = off * 1.13 + dz.abs() * 10 * O.U32 * (d64(pre).abs() + 1)
        dz = dz * O.slope(d64(pre), name)
    T = lambda t: t.transpose(1, 2).contiguous()   # noqa: E731
    for what, got, a, aoff, b in (("dx", dx, dz, off, d64(w)), ("dw", dw, T(dz), T(off), d64(x))):
        want = a @ b
        o = aoff @ b.abs() + (a.shape[-1] + 4) * O.U32 * ((a.abs() + aoff) @ b.abs())
        O.near(got, (want, o + O.ROUND[bf16] * (want.abs() + o)), f"{what} {size}")
        error, least = (got.double().cpu() - want).norm(), (want.to(bf16).double() - want).norm()
        assert float(error) <= 1.02 * float(least), (what, size, float(error / least))


def test_gradients_in_bf16_of_values_at_the_ends_of_the_range(ops):   # noqa: F811
    """An infinite dz is infinite in dx (not NaN), and so is one that is beyond bf16's largest value; a NaN stays in its row."""
    bf16, big = torch.bfloat16, torch.finfo(torch.bfloat16).max
    g = torch.Generator().manual_seed(3)
    rows, inp, out = 70, 40, 72
    x, w = rand(g, (1, rows, inp), bf16), rand(g, (1, out, inp), bf16).abs() + 0.5
    dy = rand(g, (1, rows, out), bf16)
    kept = (O.kept(9, 0, rows, out, 0.5) > 0).nonzero()
    place = {int(r): int(c) for r, c in kept}   # a column that stays, of each row
    for r, v in ((0, float("inf")), (1, -float("inf")), (2, big), (3, float("nan"))):
        dy[0, r, place[r]] = v
    dx, _, db = ops.aet_linear_backward(dy, x, w, p=0.5, seed=9)
    assert bool((dx[0, 0] == float("inf")).all()) and bool((dx[0, 1] == -float("inf")).all()) and bool((dx[0, 2] == float("inf")).all())
    assert bool(torch.isnan(dx[0, 3]).all()) and bool(torch.isfinite(dx[0, 4:]).all())


def one_first(x, others):
    """x of N(0, 1): the first position is unlike the others, which are about `others`."""
    x += others
    x[:, :, 0] = 1000.0 if others == 0 else 0.0
    return x


def border(x):
    """Zeros around values about 100."""
    x += 100
    x[:, :, :64] = 0
    x[:, :, -64:] = 0
    return x


def trend(x):
    """A mean that moves through the sample by a hundred times what values differ by next to each other."""
    return x + torch.linspace(-50, 50, x.shape[2], device=x.device)[:, None]


VALUES = {"first_0_others_100": lambda x: one_first(x, 100.0), "first_1000_others_0": lambda x: one_first(x, 0.0), "border": border, "trend": trend,
          "one_value_last": lambda x: one_first(x, 100.0).flip(2), "far": lambda x: x + 1000.0}


@pytest.mark.parametrize("values", VALUES)
# n, batch, positions, groups, width: strips as long as the sample, and parts of it; samples that are no whole pieces; one that a
# workgroup holds
@pytest.mark.parametrize("size", [(4, 256, 4096, 8, 4), (1, 256, 16384, 2, 4), (1, 2, 65536, 3, 5), (2, 550, 9003, 1, 3), (1, 3, 9001, 2, 40),
                                  (2, 3, 300, 4, 8)], ids=str)
def test_group_norm_of_values_unlike_each_other(ops, size, values):   # noqa: F811
    """Statistics and results in fp32, whichever value comes first: mean and rstd within 64 units of 2^-24 (the mean, of its
    magnitude and the spread; rstd, also by the mean's error squared), y as much of the largest value's."""
    n, b, P, G, width = size
    g = torch.Generator(device=DEV).manual_seed(P + width)
    x = VALUES[values](torch.randn(n * b, 1, P, G * width, generator=g, device=DEV)).view(n, b, P, G * width).contiguous()
    y, mean, rstd = ops.aet_group_norm_forward(x, G, eps=1e-5)
    for c in range(n):
        for b0 in range(0, b, 64):
            at = (slice(c, c + 1), slice(b0, b0 + 64))
            v = x[at].double().view(1, -1, P, G, width)
            m = v.mean((2, 4), keepdim=True)
            r = 1 / torch.sqrt((v - m).square().mean((2, 4), keepdim=True) + 1e-5)
            xh, big = (v - m) * r, v.abs().amax((2, 4), keepdim=True) * r
            O.near(mean[at], (m[:, :, 0, :, 0].cpu(), 64 * O.U32 * (m.abs() + 1 / r)[:, :, 0, :, 0].cpu()), "mean")
            O.near(rstd[at], (r[:, :, 0, :, 0].cpu(), (64 * O.U32 * r * (1 + O.U32 * (m * r).square()))[:, :, 0, :, 0].cpu()), "rstd")
            off = (y[at].double().view(xh.shape) - xh).abs() - 64 * O.U32 * (big + xh.abs())
            assert float(off.max()) <= 0, ("y", float(off.max()))


@pytest.mark.parametrize("rows", [1, 4096])
def test_gelu_in_fp32(ops, rows):   # noqa: F811
    """Through a layer of one input and w = 1, where z is x.  The definition's factors rounded once each, and their product, give a
    relative 2-norm of about 2/3 of a unit of 2^-24 (with erf 0.64; the slope's two terms 0.66): one unit is allowed for the value, and
    for the slope, a sum, one and a half.  The tail is itself to 2^-15 as far as z = -5."""
    out = 1 << 16 if rows == 1 else 16
    g = torch.Generator().manual_seed(1)
    x = rand(g, (rows, 1), torch.float32)
    w = torch.ones(out, 1, device=DEV) if rows > 1 else rand(g, (out, 1), torch.float32)   # one row: z is w instead
    if rows == 1:
        x.fill_(1.0)
    y, z = ops.aet_linear_forward(x, w, act="gelu", keep_pre=True)
    assert torch.equal(z, x * w.t())
    want = O.act(d64(z), "gelu")
    assert float((d64(y) - want).norm() / want.norm()) <= 2.0 ** -24
    low = (d64(z) < -2) & (d64(z) > -5)
    assert int(low.sum()) > 10 and float(((d64(y) - want) / want)[low].abs().max()) <= 2.0 ** -15
    # dy has one 1 a row, and db is the slope there; with rows of one value, dx is
    one = torch.ones(1, z.numel(), device=DEV)
    _, _, db = ops.aet_linear_backward(one, one[:, :1], torch.ones(z.numel(), 1, device=DEV), z.reshape(1, -1), act="gelu")
    slope = O.slope(d64(z).reshape(-1), "gelu")
    assert float((d64(db) - slope).norm() / slope.norm()) <= 1.5 * 2.0 ** -24


def test_gelu_at_the_ends_of_the_range(ops):   # noqa: F811
    z = torch.tensor([[0.0, -0.0, 1e-30, -1e-30, 6.0, 1e20, torch.finfo(torch.float32).max, float("inf"), -12.0, -1e20, -torch.finfo(torch.float32).max,
                       float("nan")]], device=DEV)
    y = ops.aet_linear_forward(torch.ones(1, 1, device=DEV), z.t().contiguous(), act="gelu")[0][0].cpu()
    assert torch.equal(y[4:8], z[0, 4:8].cpu()) and bool((y[:2] == 0).all()) and bool((y[2:4].abs() < 1e-30).all())
    assert bool((y[8:11].abs() < 1e-30).all()) and bool(torch.isnan(y[11]))
    one = torch.ones_like(z)
    _, _, db = ops.aet_linear_backward(one, one[:, :1], torch.ones(z.shape[1], 1, device=DEV), z, act="gelu")
    assert torch.equal(db[4:7].cpu(), torch.ones(3)) and bool((db[8:11].abs() < 1e-28).all())


# (n, batch, positions, groups, width) of the norm's tests, and larger ones of one launch and of three
RELU = [(1, 1, 20, 1, 1), (2, 3, 1, 4, 8), (1, 2, 50, 16, 1), (2, 2, 35, 3, 5), (1, 1, 784, 4, 4), (3, 4, 64, 8, 4), (2, 2, 256, 2, 24), (1, 3, 100, 1, 33),
        (1, 1, 4096, 8, 40), (1, 2, 3001, 5, 7), (1, 1, 20000, 2, 16), (4, 30, 9, 2, 6), (1, 2, 17, 32, 40), (1, 1, 1, 1, 2000), (1, 1, 900, 3, 96),
        (2, 40, 300, 6, 7), (2, 64, 1024, 9, 10)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", RELU, ids=str)
def test_group_norm_gradient_behind_relu(ops, size, dtype):   # noqa: F811
    """Every size: where the value before the activation is so near 0 that its sign in fp32 is open, dy is 0."""
    n, b, P, G, width = size
    dt, ch = TYPES[dtype], G * width
    g = torch.Generator().manual_seed(P + ch)
    x, dy = rand(g, (n, b, P, ch), dt) + 0.5, rand(g, (n, b, P, ch), dt)
    gamma, beta = rand(g, (n, ch), dt), rand(g, (n, ch), dt)
    _, mean, rstd = ops.aet_group_norm_forward(x, G, gamma, beta, eps=1e-3, act="relu")
    t = ((d64(x).view(n, b, P, G, width) - d64(mean)[:, :, None, :, None]) * d64(rstd)[:, :, None, :, None]).reshape(n, b, P, ch)
    t = t * d64(gamma)[:, None, None] + d64(beta)[:, None, None]
    near = t.abs() < 1e-5 * (t.abs().amax() + 1)
    dy[near.to(DEV)] = 0
    assert float(near.double().mean()) < 0.01 or near.numel() < 100
    got = ops.aet_group_norm_backward(dy, x, mean, rstd, gamma, beta, act="relu")
    want = O.group_norm_backward(d64(dy), d64(x), d64(mean), d64(rstd), d64(gamma), d64(beta), "relu", dt)
    for what, a, c in zip(("dx", "dgamma", "dbeta"), got, want):
        O.near(a, c, f"{what} {size} {dtype}")


# n, rows, in, out: the products of a layer and of both its gradients in tiles of 128 x 128, 64 x 128 and 64 x 64, in one sum and in
# slices, and the pair of small ones
TILES = [(1, 2048, 1024, 2048), (1, 1024, 2048, 2048), (1, 3000, 700, 4104), (2, 2568, 2624, 2632), (64, 64, 1024, 512), (3, 1001, 1155, 771),
         (1, 640, 640, 640), (1, 4096, 64, 40), (2, 40, 96, 64), (2, 257, 129, 255)]


@pytest.mark.parametrize("size", TILES, ids=str)
def test_products_in_fp32_hold_24_bits(ops, size):   # noqa: F811
    """Relative 2-norms of normal deviates' products, more than 32 rows, within product_norm of their sums' lengths."""
    n, rows, inp, out = size
    f32 = torch.float32
    g = torch.Generator().manual_seed(rows)
    x, w, dy = rand(g, (n, rows, inp), f32), rand(g, (n, out, inp), f32), rand(g, (n, rows, out), f32)
    y, _ = ops.aet_linear_forward(x, w)
    dx, dw, _ = ops.aet_linear_backward(dy, x, w)
    T = lambda t: t.transpose(1, 2).contiguous()   # noqa: E731
    for what, got, a, b in (("y", y, x, T(w)), ("dx", dx, dy, w), ("dw", dw, T(dy), x)):
        want = d64(a) @ d64(b)
        off, most = float((d64(got) - want).norm() / want.norm()), product_norm(a.shape[-1])
        assert off <= most, (what, size, off, most)


@pytest.mark.parametrize("rows", [20, 48, 300])
def test_tiny_operands_in_fp32(ops, rows):   # noqa: F811
    """Operands of 2^-125 to 2^-105 beside others of 2^60: taken to within 2^-134 (those of a call of up to 32 rows whole), beside the
    rounding of the sums."""
    inp, out = 96, 80
    f32 = torch.float32
    g = torch.Generator().manual_seed(rows)

    def tiny(*shape):
        return (torch.randn(*shape, generator=g) * 2.0 ** (-105 - 20 * torch.rand(*shape, generator=g))).to(DEV)

    def product(what, got, a, b, low):
        want, S = d64(a) @ d64(b), d64(a).abs() @ d64(b).abs()
        off = (a.shape[-1] + 4) * O.U32 * S + low * (torch.ones_like(d64(a)) @ d64(b).abs())
        O.near(got * 2.0 ** 60, (want * 2.0 ** 60, (off + O.U32 * (want.abs() + off)) * 2.0 ** 60), what)

    x, w, dy = tiny(1, rows, inp), rand(g, (1, out, inp), f32, 2.0 ** 60), tiny(1, rows, out)
    big = rand(g, (1, rows, inp), f32, 2.0 ** 60)
    T = lambda t: t.transpose(1, 2).contiguous()   # noqa: E731
    product("y", ops.aet_linear_forward(x, w)[0], x, T(w), 0.0 if rows <= 32 else 2.0 ** -134)
    dx, dw, _ = ops.aet_linear_backward(dy, big, w)
    product("dx", dx, dy, w, 2.0 ** -134)
    product("dw", dw, T(dy), big, 2.0 ** -134)


def test_gradients_in_bf16_beyond_its_largest_value(ops):   # noqa: F811
    """dz between bf16's largest value and fp32's is finite, and so is what it gives."""
    bf16 = torch.bfloat16
    big, p = torch.finfo(bf16).max, 0.0025
    rows, inp, out = 70, 40, 72
    g = torch.Generator().manual_seed(3)
    w, x = rand(g, (1, out, inp), bf16, 2.0 ** -20), rand(g, (1, rows, inp), bf16, 2.0 ** -20)
    dy = rand(g, (1, rows, out), bf16)
    m = O.mask3((1, rows, out), 9, 0, p)
    assert bool((m[0, 5:8, 3] > 0).all()) and big < big / (1 - p) < torch.finfo(torch.float32).max
    dy[0, 5, 3], dy[0, 6, 3], dy[0, 7, 3] = big, -big, big
    dx, dw, _ = ops.aet_linear_backward(dy, x, w, p=p, seed=9)
    dz = d64(dy) * m
    T = lambda t: t.transpose(1, 2).contiguous()   # noqa: E731
    for what, got, a, b in (("dx", dx, dz, d64(w)), ("dw", dw, T(dz), d64(x))):
        want, S = a @ b, a.abs() @ b.abs()
        o = (2.0 ** -16 + (a.shape[-1] + 8) * O.U32) * S
        O.near(got, (want, o + O.ROUND[bf16] * (want.abs() + o)), what)
