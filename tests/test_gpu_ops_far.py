"""Tensors of more than 2^31 elements, and lines of more than 2^22: what lies far from the beginning is what it is by itself."""
import pytest
import torch

from test_gpu_ops_linear import DEV, TYPES, ops  # noqa: F401

pytestmark = pytest.mark.gpu
B = torch.bfloat16


def normal(*shape, seed=1, dtype=B):
    t = torch.empty(*shape, device=DEV, dtype=dtype)
    return t.normal_(generator=torch.Generator(device=DEV).manual_seed(seed))


@pytest.fixture(autouse=True)
def room():
    yield
    torch.cuda.empty_cache()


def test_values_and_codes(ops):   # noqa: F811
    x = normal(70000, 32768)
    codes, scales = ops.aet_mx4_quantise(x)
    y = ops.aet_mx4_dequantise(codes, scales)
    for part in (slice(0, 3), slice(65530, 65540), slice(69990, None)):
        c, s = ops.aet_mx4_quantise(x[part].contiguous())
        assert torch.equal(codes[part], c) and torch.equal(scales[part], s) and torch.equal(y[part], ops.aet_mx4_dequantise(c, s))


@pytest.mark.parametrize("cols", [32768, 40000])
def test_layer_norm(ops, cols):   # noqa: F811
    rows = 70000
    x, dy, gamma = normal(rows, cols), normal(rows, cols, seed=2), normal(cols)
    y, _, mean, rstd = ops.aet_layer_norm_forward(x, gamma)
    dx, _, _ = ops.aet_layer_norm_backward(dy, x, mean, rstd, gamma)
    for part in (slice(0, 3), slice(65530, 65540), slice(69990, None)):
        a, _, m, r = ops.aet_layer_norm_forward(x[part].contiguous(), gamma)
        assert torch.equal(y[part], a) and torch.equal(mean[part], m) and torch.equal(rstd[part], r)
        assert torch.equal(dx[part], ops.aet_layer_norm_backward(dy[part].contiguous(), x[part].contiguous(), m, r, gamma)[0])


def signs(rows, cols, seed):
    """(codes, scales, values) of 1 and -1; cols even."""
    v = torch.randint(0, 2, (rows, cols), device=DEV, dtype=torch.uint8, generator=torch.Generator(device=DEV).manual_seed(seed))
    codes = 2 + 8 * v
    return codes[:, 0::2] | codes[:, 1::2] << 4, torch.full((rows, (cols + 31) // 32), 127, dtype=torch.uint8, device=DEV), 1 - 2 * v.to(torch.int8)


@pytest.mark.parametrize("act", ["none", "relu"])
def test_the_layer_of_4_bit_values(ops, act):   # noqa: F811
    """Sums of whole numbers, which every type here holds: rows far from the first are those of a call with them alone."""
    rows, inp, out = 70000, 32, 32768
    (x, xs, vx), (w, ws, vw) = signs(rows, inp, 1), signs(out, inp, 2)
    y, pre = ops.aet_mx4_linear_forward(x, xs, w, ws, act=act, keep_pre=True)
    dy = normal(rows, out)
    dx, dw, db = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, pre, act=act)
    for part in (slice(0, 3), slice(65530, 65540), slice(69990, None)):
        z = vx[part].double() @ vw.double().t().contiguous()
        assert torch.equal(pre[part].double(), z) and torch.equal(y[part].double(), z if act == "none" else z.clamp(min=0))
        dz = dy[part].double() * (1.0 if act == "none" else (z > 0))
        want, most = dz @ vw.double(), dz.abs().sum(1, keepdim=True)
        assert bool(((dx[part].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -16 + out * 2.0 ** -24) * most).all())
    # all rows: column by column, some outputs
    for part in (slice(0, 2), slice(32766, None)):
        z = vx.double() @ vw[part].double().t().contiguous()
        dz = dy[:, part].double() * (1.0 if act == "none" else (z > 0))
        for got, want in ((dw[part], dz.t().contiguous() @ vx.double()), (db[part], dz.sum(0))):
            most = dz.abs().sum(0)
            most = most[:, None] if got.dim() == 2 else most
            assert bool(((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -16 + rows * 2.0 ** -24) * most).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(3, 8, (1 << 22) + 8), (40, 24, (1 << 22) + 2), (3, (1 << 24) + 32, 2), (40, (1 << 24) + 34, 3)], ids=str)
def test_long_lines(ops, size, dtype):   # noqa: F811
    """Lines whose tiles' places pass 32 bits.  Whole numbers below 2^24 all through, whose sums are exact in any order."""
    rows, inp, out = size
    dt = TYPES[dtype]
    (x, xs, vx), (w, ws, vw) = signs(rows, inp, 1), signs(out, inp, 2)
    z = vx.double() @ vw.double().t().contiguous()
    y, _ = ops.aet_mx4_linear_forward(x, xs, w, ws, cols=inp, dtype=dt)
    assert torch.equal(y, z.to(dt))
    dy = torch.randint(-1, 2, (rows, out), device=DEV, generator=torch.Generator(device=DEV).manual_seed(3)).to(dt)
    for act in ("none", "relu"):
        dx, dw, db = ops.aet_mx4_linear_backward(dy, x, xs, w, ws, z.to(dt), cols=inp, act=act)
        dz = dy.double() * (1.0 if act == "none" else (z > 0))
        assert torch.equal(dx, (dz @ vw.double()).to(dt)) and torch.equal(dw, (dz.t().contiguous() @ vx.double()).to(dt)) and torch.equal(db, dz.sum(0).to(dt))
