"""How near the operators come to their definitions in 64 bits where a bound of the worst case says little: the rounding
errors of whole tensors."""
import pytest
import torch

import ops_oracle as O
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
