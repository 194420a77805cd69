"""What the entry points of layer normalisation, orthogonalised updates and microscaled 4-bit values refuse, on the host: nothing is launched, so no
GPU is needed."""
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


def values(**k):
    return made(ops.aet_mx4_values(0, 2, 3, 70, P, 210, 70, P, 105, 35, P, 9, 3), k)


def codes(**k):
    return made(ops.aet_mx4_codes(0, 2, 3, 70, P, 105, 35, P, 9, 3, P, 210, 70), k)


def linear(**k):
    return made(ops.aet_mx4_linear(0, 1, 2, 3, 70, 4, 0.1, 1, 0, P, 105, 35, P, 9, 3, P, 140, 35, P, 12, 3, P, 4, 0, P, 12, 4, P, 12, 4, P, 12, 4), k)


def linear_grad(**k):
    return made(ops.aet_mx4_linear_grad(0, 1, 2, 3, 70, 4, 0.1, 1, 0, P, 12, 4, P, 105, 35, P, 9, 3, P, 140, 35, P, 12, 3, P, 12, 4, P, 210, 70, P, 280, 70,
                                        P, 4, 0), k)


DROP = [dict(p=1.0), dict(p=float("nan")), dict(first_row=-1), dict(first_row=2 ** 63 - 2)]
SIZES = [dict(dtype=2), dict(n=-1), dict(rows=-1), dict(rows=(1 << 30) + 1)]
HELD = [dict(codes_p=None), dict(scales_p=None), dict(codes_row=-1), dict(scales_client=-1)]
WRONG = {
    "aet_mx4_quantise": (values, SIZES + HELD + [dict(cols=-1), dict(x_p=None), dict(x_p=P + 2), dict(x_row=-1), dict(codes_row=34), dict(codes_client=104),
                                                 dict(scales_row=2), dict(scales_client=8)]),
    "aet_mx4_dequantise": (codes, SIZES + HELD + [dict(cols=-1), dict(y_p=None), dict(y_p=P + 2), dict(y_row=69), dict(y_client=209)]),
    "aet_mx4_linear_forward": (linear, SIZES + DROP + [dict(act=4), dict(out=-1), {"in": -1}, dict(x_p=None), dict(x_scales_p=None), dict(w_p=None),
                                                       dict(w_scales_p=None), dict(x_row=-1), dict(w_scales_row=-1), dict(w_client=0), dict(w_scales_client=0),
                                                       dict(y_p=None), dict(y_p=P + 2), dict(y_row=3), dict(bias_p=P + 1), dict(residual_row=-1),
                                                       dict(pre_client=8), dict(n=1 << 30, rows=1 << 30), dict(x_client=1 << 60)]),
    "aet_mx4_linear_backward": (linear_grad, SIZES + DROP + [dict(act=4), dict(out=-1), {"in": -1}, dict(x_p=None), dict(x_scales_p=None), dict(w_p=None),
                                                             dict(w_scales_p=None), dict(dy_p=None), dict(pre_p=None), dict(w_client=0), dict(dx_row=69),
                                                             dict(dw_client=279), dict(db_client=3), dict(dw_client=0), dict(dy_p=P + 2),
                                                             dict(dw_client=0, db_client=0)])}


@pytest.mark.parametrize("fn,wrong", [(f, w) for f, (_, all_) in WRONG.items() for w in all_], ids=str)
def test_mx4_refused(lib, fn, wrong):   # noqa: F811
    a = WRONG[fn][0](**wrong)
    space = (P, 1 << 60) if "linear" in fn else ()
    assert getattr(lib, fn)(C.addressof(a), *space, None) == EINVAL and lib.aet_ops_last_error()
    if space:
        assert getattr(lib, fn.replace("_forward", "") + "_workspace_bytes")(C.addressof(a)) == 0


def test_mx4_edges(lib):   # noqa: F811
    for fn, (make, _) in WRONG.items():
        space = (None, 0) if "linear" in fn else ()
        assert getattr(lib, fn)(None, *space, None) == EINVAL
        assert getattr(lib, fn)(C.addressof(make(n=0)), *space, None) == 0
    assert lib.aet_mx4_quantise(C.addressof(values(cols=0)), None) == 0 and lib.aet_mx4_dequantise(C.addressof(codes(rows=0)), None) == 0
    assert lib.aet_mx4_linear_forward(C.addressof(linear(rows=0)), None, 0, None) == 0
    a = linear_grad(rows=300, dy_client=1200, x_client=10500, x_scales_client=900, pre_client=1200, dx_client=21000)
    need = lib.aet_mx4_linear_backward_workspace_bytes(C.addressof(a))
    assert need > 0
    for ws, size in ((None, need), (P, need - 1), (P + 128, need)):
        assert lib.aet_mx4_linear_backward(C.addressof(a), ws, size, None) == ENOMEM


def test_mx4_binding_refuses_host_tensors():
    u = torch.zeros(2, 4, dtype=torch.uint8)
    for call in (lambda: ops.aet_mx4_quantise(torch.zeros(2, 8)), lambda: ops.aet_mx4_dequantise(u, u[:, :1]),
                 lambda: ops.aet_mx4_linear_forward(u, u[:, :1], u, u[:, :1]), lambda: ops.aet_mx4_linear_backward(torch.zeros(2, 2), u, u[:, :1], u, u[:, :1])):
        with pytest.raises(ValueError, match="on a GPU"):
            call()


def orthogonal(**k):
    return made(ops.aet_orthogonal(0, 2, 3, 8, 5, 3.4445, -4.775, 2.0315, 1e-7, 1.0, 1.0, P, 24, 8, P, 24, 8, P, 24, 8), k)


@pytest.mark.parametrize("wrong", SIZES + [dict(cols=-1), dict(cols=(1 << 20) + 1), dict(rows=(1 << 20) + 1), dict(steps=-1), dict(steps=101), dict(eps=-1.0),
                                           dict(eps=float("nan")), dict(eps=float("inf")), dict(a=float("nan")), dict(b=float("inf")), dict(c=float("nan")),
                                           dict(keep=float("inf")), dict(keep=1e39), dict(scale=float("nan")), dict(a=1e7), dict(c=1e30), dict(b=-1e30), dict(g_p=None),
                                           dict(y_p=None), dict(g_p=P + 2), dict(w_p=P + 1), dict(g_row=-1), dict(w_client=-1), dict(y_row=7), dict(y_client=23)],
                         ids=str)
def test_orthogonalise_refused(lib, wrong):   # noqa: F811
    a = orthogonal(**wrong)
    assert lib.aet_orthogonalise(C.addressof(a), P, 1 << 60, None) == EINVAL and lib.aet_ops_last_error()
    assert lib.aet_orthogonalise_workspace_bytes(C.addressof(a)) == 0


def test_orthogonalise_edges(lib):   # noqa: F811
    assert lib.aet_orthogonalise(None, None, 0, None) == EINVAL
    for nothing in (dict(n=0), dict(rows=0), dict(cols=0)):
        assert lib.aet_orthogonalise(C.addressof(orthogonal(**nothing)), None, 0, None) == 0
    a = orthogonal()
    need = lib.aet_orthogonalise_workspace_bytes(C.addressof(a))
    assert need > 0
    for ws, size in ((None, need), (P, need - 1), (P + 128, need)):
        assert lib.aet_orthogonalise(C.addressof(a), ws, size, None) == ENOMEM
