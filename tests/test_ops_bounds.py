"""How far fp32 products may be off in the 2-norm, and that the bound tells a product whose corrections are lost."""
import pytest
import torch


def product_norm(K):
    """Sums of K products of normal deviates, rounded to fp32.  The three-part products were measured at 1.0e-7 (288 terms), 1.4e-7
    (576) and 3.9e-7 (4096), 6e-9 sqrt(K), and the rounding of the result is 2^-24 / sqrt(2) at most: three times their sum."""
    return 3 * (6e-9 * K ** 0.5 + 4e-8)


def parts(t):
    """Three bf16 parts of fp32 values, in 64 bits."""
    out, left = [], t.float()
    for _ in range(3):
        p = left.to(torch.bfloat16).float()
        out.append(p.double())
        left = left - p
    assert float(left.abs().max()) == 0
    return out


@pytest.mark.parametrize("K", [40, 129, 264, 520, 1024, 2624, 4104])
def test_a_product_without_its_corrections_is_told(K):
    """Each of the six products that is left out, but for those of the last bits, shows."""
    g = torch.Generator().manual_seed(K)
    a, b = torch.randn(200, K, generator=g), torch.randn(200, K, generator=g)
    want = a.double() @ b.double().t()
    pa, pb = parts(a), parts(b)
    six = [(0, 0), (0, 1), (1, 0), (1, 1), (0, 2), (2, 0)]

    def off(pairs):
        return float((sum(pa[i] @ pb[j].t() for i, j in pairs) - want).norm() / want.norm())

    assert off(six) < 2.0 ** -24 < product_norm(K)
    for lost in six:
        assert off([p for p in six if p != lost]) > product_norm(K), lost
    assert off(six[:3]) > product_norm(K)
