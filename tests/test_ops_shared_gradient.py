"""Gradients of one W for all clients: what lies how does not matter where it is neither read nor written.  On the host: a call
that passes the checks asks for its workspace, and nothing is launched."""
import ctypes as C

import pytest

from paper_2112_13935_amd import ops

EINVAL, ENOMEM = -1, -2
P = 1 << 20   # an address that is never read
N, ROWS, IN, OUT = 2, 1000, 8, 4


def grad(**k):
    """Everything shared and wanted, rows one after another."""
    a = ops.aet_linear_grad(0, 1, N, ROWS, IN, OUT, 0.1, 1, 0, P, ROWS * OUT, OUT, P, ROWS * IN, IN, P, 0, IN, P, ROWS * OUT, OUT, P, ROWS * IN, IN,
                            P, 0, IN, P, 0, 0)
    for f, v in k.items():
        setattr(a, f, v)
    return a


def status(a):
    lib = ops.load_library()
    assert lib.aet_linear_backward_workspace_bytes(C.addressof(a)) == 0 or lib.aet_linear_backward(C.addressof(a), None, 0, None) == ENOMEM
    return lib.aet_linear_backward(C.addressof(a), None, 0, None)


NO_DX, NO_DW = dict(dx_p=None), dict(dw_p=None)


@pytest.mark.parametrize("what", [dict(), dict(NO_DW, x_client=ROWS * IN + 8), dict(NO_DW, **NO_DX, x_client=3, x_row=IN + 1), dict(NO_DX, w_client=OUT * IN),
                                  dict(NO_DX, dx_client=5), dict(act=0, pre_client=7), dict(NO_DW, dw_client=OUT * IN)], ids=str)
def test_taken(what):
    assert status(grad(**what)) == ENOMEM


@pytest.mark.parametrize("what", [dict(x_client=ROWS * IN + 8), dict(dy_client=ROWS * OUT + 4), dict(pre_client=0), dict(dx_client=ROWS * IN + 8),
                                  dict(w_client=OUT * IN), dict(NO_DX, x_client=ROWS * IN + 8), dict(NO_DX, dw_client=OUT * IN)], ids=str)
def test_refused(what):
    assert status(grad(**what)) == EINVAL


def one_row(rows, **k):
    """Clients' rows with gaps, and strides of rows that say nothing."""
    big = 200   # enough clients for a workspace
    return grad(n=big, rows=rows, dy_client=3 * OUT, dy_row=1, x_client=5 * IN, x_row=7, pre_client=0, pre_row=2, dx_client=IN + 1, dx_row=0, **k)


def test_one_row_a_client():
    assert status(one_row(1)) == ENOMEM
    assert status(one_row(2)) == EINVAL

