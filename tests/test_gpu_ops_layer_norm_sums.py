"""The sums over rows in layer normalisation's gradient, in the 2-norm: as near as the same sums by PyTorch in fp32."""
import pytest
import torch

from test_gpu_ops_linear import DEV, ops  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [(16, 333, 771), (1, 20000, 771), (1, 300, 4096), (1, 5000, 1024), (4, 1000, 100)], ids=str)
def test_sums_over_rows(ops, size):   # noqa: F811
    """Roundings add up over the additions that a term goes through, at random.  Strips and their sums by twos are no more of them than
    a tree of short runs, which PyTorch adds by; a tenth is for chance (there are more than a hundred sums)."""
    n, rows, cols = size
    g = torch.Generator(device=DEV).manual_seed(1)
    normal = lambda *s: torch.randn(*s, generator=g, device=DEV)   # noqa: E731
    x, dy, gamma = normal(n, rows, cols) + 0.5, normal(n, rows, cols), normal(n, cols)
    _, _, mean, rstd = ops.aet_layer_norm_forward(x, gamma)
    got = ops.aet_layer_norm_backward(dy, x, mean, rstd, gamma, need=(False, True))[1:]
    sums = lambda t: ((t(dy) * ((t(x) - t(mean)[..., None]) * t(rstd)[..., None])).sum(1), t(dy).sum(1))   # noqa: E731
    want, near = sums(torch.Tensor.double), sums(torch.Tensor.float)
    for a, w, b, what in zip(got, want, near, ("dgamma", "dbeta")):
        off, other = (float((v.double() - w).norm() / w.norm()) for v in (a, b))
        print(size, what, f"{off:.3g} {other:.3g}")
        assert off <= 1.1 * other, f"{what}: off by {off:.3g}, sums in fp32 by {other:.3g}"
