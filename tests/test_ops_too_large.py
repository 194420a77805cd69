"""Calls of which a launch would have 2^32 threads or more are refused before anything is launched: no GPU is needed."""
import ctypes as C

import pytest

from paper_2112_13935_amd import ops
from test_more_ops_refusals import codes, linear, linear_grad, norm, norm_grad, orthogonal, values
from test_ops_refusals import P, lib  # noqa: F401

EHIP = -3   # AET_EHIP
N = 1 << 25
CALLS = {
    "aet_mx4_quantise": values(n=N, rows=1),
    "aet_mx4_dequantise": codes(n=N, rows=1),
    "aet_mx4_linear_forward": linear(n=N, rows=1),
    "aet_mx4_linear_backward": linear_grad(n=N, rows=1),
    "aet_layer_norm_forward": norm(n=1, rows=1 << 23, cols=20000, x_row=20000, residual_p=None, h_p=None, y_row=20000),
    "aet_layer_norm_backward": norm_grad(n=N, rows=1),
    "aet_orthogonalise": orthogonal(n=N),
    "aet_dropout_forward": ops.aet_dropout(0, N, 2, 8, 0.0, 0, 0, P, 24, 8, None, 0, 0, P, 24, 8),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_too_large(lib, name):   # noqa: F811
    space = (P, 1 << 62) if "linear" in name or "backward" in name or "orthogonal" in name else ()
    assert getattr(lib, name)(C.addressof(CALLS[name]), *space, None) == EHIP
    assert b"2^32" in lib.aet_ops_last_error()
