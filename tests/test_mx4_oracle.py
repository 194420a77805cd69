"""The 64-bit form of microscaled 4-bit values against the table of the format, element by element."""
import torch

import mx4_oracle as M


def test_table():
    # 2 bits of exponent with a bias of 1, a bit of mantissa; a block whose largest value is 4 has an exponent of 0
    v = torch.tensor([[0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]])
    codes, scales = M.quantise(v)
    assert scales.tolist() == [[127]]
    assert codes.tolist() == [[(2 * k) | (2 * k + 1) << 4 for k in range(8)]]
    assert torch.equal(M.values(codes, scales, 16), v.double())


def test_borders():
    at = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    low, itself, high = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0], [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0], [0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    for shift, want in ((-2.0 ** -20, low), (0.0, itself), (2.0 ** -20, high)):
        v = torch.tensor([[b + shift for b in at] + [7.9]])
        codes, scales = M.quantise(v)
        assert M.values(codes, scales, 8).tolist() == [want + [6.0]]


def test_scales():
    for top, want in ((0.0, 0), (2.0 ** -149, 0), (2.0 ** -125, 0), (1.99 * 2.0 ** -125, 0), (2.0 ** -124, 1), (1.0, 125), (1.99, 125), (2.0, 126),
                      (3.4e38, 252), (float("inf"), 255), (float("nan"), 255)):
        assert M.quantise(torch.tensor([[top] + [0.0] * 40]))[1].tolist() == [[want, 0]], top
