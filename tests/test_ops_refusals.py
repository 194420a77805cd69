"""What the operators' entry points refuse, on the host: nothing is launched, so no GPU is needed."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2112_13935_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ENOMEM = -1, -2
P = 1 << 20   # an address that is never read


@pytest.fixture(scope="module")
def lib():
    return ops.load_library()


def test_library_exports_what_the_header_declares(lib):
    text = open(os.path.join(ROOT, "include", "aet_ops.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(aet_[a-zA-Z0-9_]+)\s*\(", text)))
    assert names == sorted(ops.EXPORTS)
    for name in names:
        assert hasattr(lib, name)


def linear(**k):
    a = ops.aet_linear(0, 1, 2, 3, 8, 4, 0.1, 1, 0, P, 24, 8, P, 32, 8, P, 4, 0, P, 12, 4, P, 12, 4, P, 12, 4)
    for f, v in k.items():
        setattr(a, f, v)
    return a


def grad(**k):
    a = ops.aet_linear_grad(0, 1, 2, 3, 8, 4, 0.1, 1, 0, P, 12, 4, P, 24, 8, P, 32, 8, P, 12, 4, P, 24, 8, P, 32, 8, P, 4, 0)
    for f, v in k.items():
        setattr(a, f, v)
    return a


def norm(**k):
    a = ops.aet_group_norm(0, 1, 2, 3, 5, 2, 4, 1e-5, P, 120, 40, 8, P, 8, 0, P, 8, 0, P, 120, 40, 8, P, P)
    for f, v in k.items():
        setattr(a, f, v)
    return a


def norm_grad(**k):
    a = ops.aet_group_norm_grad(0, 1, 2, 3, 5, 2, 4, P, 120, 40, 8, P, 120, 40, 8, P, P, P, 8, 0, P, 8, 0, P, 120, 40, 8, P, 8, 0, P, 8, 0)
    for f, v in k.items():
        setattr(a, f, v)
    return a


def dropout(**k):
    a = ops.aet_dropout(0, 2, 3, 8, 0.1, 1, 0, P, 24, 8, P, 24, 8, P, 24, 8)
    for f, v in k.items():
        setattr(a, f, v)
    return a


COMMON = [dict(dtype=2), dict(dtype=-1), dict(n=-1)]
DROP = [dict(p=1.0), dict(p=-0.1), dict(p=float("nan")), dict(first_row=-1), dict(first_row=2 ** 63 - 2)]
ACT = [dict(act=4), dict(act=-1)]
LINEAR = COMMON + DROP + ACT + [dict(rows=-1), dict(out=-1), {"in": -1}, dict(x_p=None), dict(w_p=None), dict(y_p=None),
                                dict(x_p=P + 2), dict(bias_p=P + 1), dict(x_row=-8), dict(w_client=-1), dict(y_row=3),
                                dict(y_client=8), dict(pre_row=0), dict(x_client=1 << 60), dict(residual_row=-1)]
GRAD = COMMON + DROP + ACT + [dict(rows=-1), dict(dy_p=None), dict(x_p=None), dict(w_p=None), dict(pre_p=None), dict(dx_row=7),
                              dict(dw_client=31), dict(dw_row=7), dict(db_client=3), dict(dx_client=0), dict(dy_p=P + 2),
                              dict(dw_client=0), dict(dw_client=0, w_client=0),   # db has a place for each client
                              dict(dw_client=0, db_client=0),   # w has not the same for all
                              dict(dw_client=0, db_client=0, w_client=0, x_client=32)]   # rows do not follow one another
NORM = COMMON + ACT + [dict(batch=-1), dict(positions=-1), dict(groups=0), dict(width=0), dict(groups=1 << 13, width=1 << 13),
                       dict(eps=-1.0), dict(eps=float("nan")), dict(x_p=None), dict(y_p=None), dict(y_row=7), dict(y_sample=39),
                       dict(y_client=119), dict(x_row=-1), dict(gamma_client=-1), dict(beta_p=P + 2), dict(mean=P + 2)]
NORM_GRAD = COMMON + ACT + [dict(dy_p=None), dict(x_p=None), dict(mean=None), dict(rstd=None), dict(dx_row=7), dict(dx_sample=0),
                            dict(dgamma_client=7), dict(dbeta_client=-1), dict(rstd=P + 1)]
DROPOUT = COMMON + DROP + [dict(rows=-1), dict(cols=-1), dict(x_p=None), dict(y_p=None), dict(y_row=7), dict(y_client=0),
                           dict(x_row=-1), dict(residual_p=P + 2)]


@pytest.mark.parametrize("fn,make,wrong", [("aet_linear_forward", linear, w) for w in LINEAR] + [("aet_linear_backward", grad, w) for w in GRAD]
                         + [("aet_group_norm_forward", norm, w) for w in NORM] + [("aet_group_norm_backward", norm_grad, w) for w in NORM_GRAD],
                         ids=str)
def test_refused(lib, fn, make, wrong):
    a = make(**wrong)
    big = 1 << 40
    assert getattr(lib, fn)(C.addressof(a), P, big, None) == EINVAL
    assert lib.aet_ops_last_error()
    sizes = fn.replace("_forward", "") + "_workspace_bytes"
    assert getattr(lib, sizes)(C.addressof(a)) == 0


@pytest.mark.parametrize("wrong", DROPOUT, ids=str)
def test_dropout_refused(lib, wrong):
    a = dropout(**wrong)
    assert lib.aet_dropout_forward(C.addressof(a), None) == EINVAL and lib.aet_ops_last_error()


def test_gradient_of_dropout_takes_no_residual(lib):
    assert lib.aet_dropout_backward(C.addressof(dropout()), None) == EINVAL


def test_no_record(lib):
    for fn in ("aet_linear_forward", "aet_linear_backward", "aet_group_norm_forward", "aet_group_norm_backward"):
        assert getattr(lib, fn)(None, None, 0, None) == EINVAL
    assert lib.aet_dropout_forward(None, None) == EINVAL and lib.aet_dropout_backward(None, None) == EINVAL


def test_workspace_too_small(lib):
    a = grad()
    need = lib.aet_linear_backward_workspace_bytes(C.addressof(a))
    assert need > 0
    for ws, size in ((None, need), (P, need - 1), (P + 128, need)):
        assert lib.aet_linear_backward(C.addressof(a), ws, size, None) == ENOMEM
        assert str(need).encode() in lib.aet_ops_last_error()


def test_nothing_to_do_needs_no_gpu(lib):
    for fn, a in (("aet_linear_forward", linear(n=0)), ("aet_linear_forward", linear(rows=0)), ("aet_linear_backward", grad(n=0)),
                  ("aet_group_norm_forward", norm(n=0)), ("aet_group_norm_backward", norm_grad(n=0))):
        assert getattr(lib, fn)(C.addressof(a), None, 0, None) == 0
    assert lib.aet_dropout_forward(C.addressof(dropout(rows=0)), None) == 0


def test_binding_refuses():
    x = torch.zeros(2, 3)
    with pytest.raises(ValueError, match="on a GPU"):
        ops.aet_linear_forward(x, torch.zeros(4, 3))
    with pytest.raises(ValueError, match="on a GPU"):
        ops.aet_dropout_forward(x, p=0.1, seed=0)
    with pytest.raises(ValueError, match="groups"):
        ops.aet_group_norm_forward(torch.zeros(1, 4, 6), 4)


def test_gradients_of_gamma_and_beta_agree(lib):
    """One of them the sum over the clients, the other not."""
    for wrong in (dict(dgamma_client=0), dict(dbeta_client=0)):
        a = norm_grad(**wrong)
        assert lib.aet_group_norm_backward(C.addressof(a), P, 1 << 40, None) == EINVAL
        assert b"either both or none" in lib.aet_ops_last_error()
