"""What the entry points of layer normalisation refuse, on the host: nothing is launched, so no GPU is needed."""
import ctypes as C

import pytest
import torch

from paper_2112_13935_amd import ops
from test_ops_refusals import EINVAL, ENOMEM, P, lib  # noqa: F401


def made(a, k):
    for f, v in k.items():
        setattr(a, f, v)
    return a


def norm(**k):
    return made(ops.aet_layer_norm(0, 2, 3, 8, 1e-5, P, 24, 8, P, 24, 8, P, 8, 0, P, 8, 0, P, 24, 8, P + 4096, 24, 8, P, P), k)


def norm_grad(**k):
    return made(ops.aet_layer_norm_grad(0, 2, 3000, 8, P, 24000, 8, P, 24000, 8, P, 24000, 8, P, 8, 0, P, P, P, 24000, 8, P, 8, 0, P, 8, 0), k)


COMMON = [dict(dtype=2), dict(dtype=-1), dict(n=-1), dict(rows=-1), dict(cols=-1), dict(cols=(1 << 30) + 1)]
NORM = COMMON + [dict(eps=-1.0), dict(eps=float("nan")), dict(x_p=None), dict(y_p=None), dict(x_p=P + 2), dict(x_row=-8), dict(x_client=1 << 60),
                 dict(residual_row=-1), dict(gamma_client=-1), dict(beta_p=P + 1), dict(y_row=7), dict(y_client=23), dict(h_row=7), dict(h_p=P + 2),
                 dict(h_p=P), dict(mean=P + 2), dict(rstd=P + 1)]
NORM_GRAD = COMMON + [dict(dy_p=None), dict(x_p=None), dict(dh_row=-1), dict(gamma_p=P + 2), dict(mean=None), dict(rstd=None), dict(rstd=P + 2),
                      dict(dx_row=7), dict(dx_client=0), dict(dgamma_client=7), dict(dbeta_client=-1), dict(dgamma_client=0), dict(dbeta_client=0)]


@pytest.mark.parametrize("wrong", NORM, ids=str)
def test_layer_norm_refused(lib, wrong):   # noqa: F811
    assert lib.aet_layer_norm_forward(C.addressof(norm(**wrong)), None) == EINVAL and lib.aet_ops_last_error()


@pytest.mark.parametrize("wrong", NORM_GRAD, ids=str)
def test_layer_norm_gradient_refused(lib, wrong):   # noqa: F811
    a = norm_grad(**wrong)
    assert lib.aet_layer_norm_backward(C.addressof(a), P, 1 << 40, None) == EINVAL and lib.aet_ops_last_error()
    assert lib.aet_layer_norm_backward_workspace_bytes(C.addressof(a)) == 0


def test_layer_norm_edges(lib):   # noqa: F811
    assert lib.aet_layer_norm_forward(None, None) == EINVAL and lib.aet_layer_norm_backward(None, None, 0, None) == EINVAL
    for nothing in (dict(n=0), dict(rows=0)):
        assert lib.aet_layer_norm_forward(C.addressof(norm(**nothing)), None) == 0
    a = norm_grad()
    need = lib.aet_layer_norm_backward_workspace_bytes(C.addressof(a))
    assert need > 0
    for ws, size in ((None, need), (P, need - 1), (P + 128, need)):
        assert lib.aet_layer_norm_backward(C.addressof(a), ws, size, None) == ENOMEM
        assert str(need).encode() in lib.aet_ops_last_error()
    assert lib.aet_layer_norm_backward(C.addressof(norm_grad(cols=0)), None, 0, None) == 0


def test_binding_refuses_host_tensors():
    with pytest.raises(ValueError, match="on a GPU"):
        ops.aet_layer_norm_forward(torch.zeros(2, 3))
