"""The gradient of the linear layer of 4-bit values where its products' operands are hard to hold: blocks of zeros of any scale, differences of
nearly equal terms."""
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
