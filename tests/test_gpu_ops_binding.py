"""What the binding makes of tensors: those that it refuses, and what automatic differentiation is told."""
import pytest
import torch

from test_gpu_ops_linear import DEV, ops  # noqa: F401

pytestmark = pytest.mark.gpu


def calls(ops):   # noqa: F811
    """name: the call and its tensors, small and right."""
    z = lambda *s: torch.ones(*s, device=DEV)   # noqa: E731
    return {
        "linear_forward": (lambda x, w, bias, residual, out: ops.aet_linear_forward(x, w, bias, residual=residual, out=out),
                           dict(x=z(2, 3, 4), w=z(2, 5, 4), bias=z(2, 5), residual=z(2, 3, 5), out=z(2, 3, 5))),
        "linear_backward": (lambda dy, x, w, pre, dx, dw, db: ops.aet_linear_backward(dy, x, w, pre, act="silu", out=(dx, dw, db)),
                            dict(dy=z(2, 3, 5), x=z(2, 3, 4), w=z(2, 5, 4), pre=z(2, 3, 5), dx=z(2, 3, 4), dw=z(2, 5, 4), db=z(2, 5))),
        "group_norm_forward": (lambda x, gamma, beta, out: ops.aet_group_norm_forward(x, 2, gamma, beta, out=out),
                               dict(x=z(2, 3, 4, 6), gamma=z(2, 6), beta=z(2, 6), out=z(2, 3, 4, 6))),
        "group_norm_backward": (lambda dy, x, mean, rstd, gamma, beta, dx, dgamma, dbeta: ops.aet_group_norm_backward(
            dy, x, mean, rstd, gamma, beta, out=(dx, dgamma, dbeta)),
            dict(dy=z(2, 3, 4, 6), x=z(2, 3, 4, 6), mean=z(2, 3, 2), rstd=z(2, 3, 2), gamma=z(2, 6), beta=z(2, 6), dx=z(2, 3, 4, 6),
                 dgamma=z(2, 6), dbeta=z(2, 6))),
        "dropout_forward": (lambda x, residual, out: ops.aet_dropout_forward(x, p=0.5, seed=1, residual=residual, out=out),
                            dict(x=z(2, 3, 4), residual=z(2, 3, 4), out=z(2, 3, 4))),
        "dropout_backward": (lambda dy, out: ops.aet_dropout_backward(dy, p=0.5, seed=1, out=out), dict(dy=z(2, 3, 4), out=z(2, 3, 4))),
    }


NAMES = ["linear_forward", "linear_backward", "group_norm_forward", "group_norm_backward", "dropout_forward", "dropout_backward"]


@pytest.mark.parametrize("name", NAMES)
def test_tensors_that_require_a_gradient(ops, name):   # noqa: F811
    """Refused while gradients are on, whichever it is; taken where they are off, or of a detached tensor."""
    call, tensors = calls(ops)[name]
    call(**tensors)
    for k in tensors:
        some = dict(tensors, **{k: tensors[k].clone().requires_grad_()})
        with pytest.raises(ValueError, match="requires a gradient"):
            call(**some)
        with torch.no_grad():
            call(**some)
        with torch.inference_mode():
            call(**some)
        call(**dict(some, **{k: some[k].detach()}))
    torch.cuda.synchronize()


# name: the places that a call writes to
PLACES = {"linear_forward": ["out"], "linear_backward": ["dx", "dw", "db"], "group_norm_forward": ["out"],
          "group_norm_backward": ["dx", "dgamma", "dbeta"], "dropout_forward": ["out"], "dropout_backward": ["out"]}


@pytest.mark.parametrize("name", NAMES)
def test_places_that_are_written_have_another_version(ops, name):   # noqa: F811
    """As PyTorch's own operations on a tensor in place; inputs keep theirs."""
    call, tensors = calls(ops)[name]
    before = {k: t._version for k, t in tensors.items()}
    call(**tensors)
    for k, t in tensors.items():
        assert (t._version > before[k]) == (k in PLACES[name]), k
    with torch.inference_mode():
        call(**{k: t.clone() for k, t in tensors.items()})


def test_a_kept_tensor_that_is_overwritten_is_found(ops):   # noqa: F811
    x = torch.ones(3, 4, device=DEV)
    w = torch.ones(4, device=DEV, requires_grad=True)
    y = (x * w).sum()   # keeps x for the gradient of w
    ops.aet_dropout_forward(x, p=0.5, seed=1, out=x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_of_a_shared_bias_does_not_ask_for_x(ops, dtype):   # noqa: F811
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator().manual_seed(2)
    dy, w = torch.randn(3, 70, 5, generator=g).to(dt).to(DEV), torch.randn(5, 8, generator=g).to(dt).to(DEV)
    apart = torch.zeros(3, 90, 8, dtype=dt, device=DEV)[:, :70]   # clients' rows do not follow one another
    want = ops.aet_linear_backward(dy, apart.contiguous(), w)
    dx, none, db = ops.aet_linear_backward(dy, apart, w, need=(True, False, True))
    assert none is None and torch.equal(dx, want[0]) and torch.equal(db, want[2])
    assert torch.equal(ops.aet_linear_backward(dy, apart, w, need=(False, False, True))[2], want[2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act,p", [("none", 0.0), ("gelu", 0.2)])
def test_one_row_a_client_of_a_shared_layer(ops, dtype, act, p):   # noqa: F811
    """Rows of a larger tensor, a client's first each, one W for all: as if they were copied together."""
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator().manual_seed(2)
    rand = lambda *s: torch.randn(*s, generator=g).to(dt).to(DEV)   # noqa: E731
    dy, x, pre, w = rand(37, 3, 24)[:, :1], rand(37, 2, 40)[:, 1:], rand(37, 4, 24)[:, 2:3], rand(24, 40)
    if act == "none":
        pre = None
    more = dict(act=act, p=p, seed=3)
    want = ops.aet_linear_backward(dy.contiguous(), x.contiguous(), w, pre if pre is None else pre.contiguous(), **more)
    place = torch.full((37, 2, 40), 5.0, dtype=dt, device=DEV)
    got = ops.aet_linear_backward(dy, x, w, pre, out=(place[:, :1], None, None), **more)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and bool((place[:, 1] == 5).all())
    same = ops.aet_linear_backward(dy, x[:1].expand(37, 1, 40), w, pre, **more)   # one x for all
    assert torch.equal(same[1], ops.aet_linear_backward(dy.contiguous(), x[:1].expand(37, 1, 40).contiguous(), w, pre if pre is None else pre.contiguous(), **more)[1])


# The first tensor says type, device and sizes; mean and rstd are fp32 always.
FIRST = {"linear_forward": "x", "linear_backward": "x", "group_norm_forward": "x", "group_norm_backward": "x", "dropout_forward": "x",
         "dropout_backward": "dy"}


def another(t, how):
    if how == "type":
        return t.to(torch.bfloat16)
    if how == "device":
        return t.cpu()
    if how == "last stride":
        return t.new_zeros(*t.shape, 2)[..., 0]
    if how == "longer":
        return t.new_zeros(*t.shape[:-1], t.shape[-1] + 1)
    if how == "shorter":
        return t.new_zeros(t.shape[0], *t.shape[1:-1], t.shape[-1] - 1)
    return t[None]   # another axis


@pytest.mark.parametrize("how", ["type", "device", "last stride", "longer", "shorter", "axis"])
@pytest.mark.parametrize("name", NAMES)
def test_tensors_that_do_not_agree(ops, name, how):   # noqa: F811
    """One tensor unlike what the others call for; nothing is written."""
    call, tensors = calls(ops)[name]
    for k in tensors:
        if k == FIRST[name] and how != "last stride":
            continue
        places = {p: torch.full_like(tensors[p], 7.0) for p in PLACES[name]}
        some = dict(tensors, **places)
        some[k] = another(some[k], how)
        with pytest.raises(ValueError) as e:
            call(**some)
        torch.cuda.synchronize()
        assert all(bool((t == 7).all()) for p, t in places.items() if p != k), (k, how)
        if how in ("type", "last stride") and name != "dropout_backward":
            assert k in str(e.value), (k, how, str(e.value))


def test_first_tensors_that_are_refused(ops):   # noqa: F811
    z = lambda *s: torch.ones(*s, device=DEV)   # noqa: E731
    for bad in (z(2, 3, 4).double(), z(2, 3, 4).half(), z(2, 3, 4).int(), torch.ones(2, 3, 4)):
        with pytest.raises(ValueError, match="float32 or bfloat16 on a GPU"):
            ops.aet_linear_forward(bad, z(2, 5, 4))
        with pytest.raises(ValueError, match="float32 or bfloat16 on a GPU"):
            ops.aet_dropout_forward(bad, p=0.5, seed=1)
        with pytest.raises(ValueError, match="float32 or bfloat16 on a GPU"):
            ops.aet_group_norm_forward(bad, 2)
    for bad in (z(4), z(1, 2, 3, 4)):
        with pytest.raises(ValueError, match="2 or 3 axes"):
            ops.aet_linear_forward(bad, z(2, 5, 4))
        with pytest.raises(ValueError, match="2 or 3 axes"):
            ops.aet_dropout_forward(bad, p=0.5, seed=1)
    for bad in (z(3, 4), z(1, 1, 2, 3, 4)):
        with pytest.raises(ValueError, match="3 or 4 axes"):
            ops.aet_group_norm_forward(bad, 2)


def test_arguments_that_do_not_agree(ops):   # noqa: F811
    from paper_2112_13935_amd import AetError
    z = lambda *s: torch.ones(*s, device=DEV)   # noqa: E731
    with pytest.raises(ValueError, match="pre"):
        ops.aet_linear_backward(z(2, 3, 5), z(2, 3, 4), z(2, 5, 4), act="gelu")
    with pytest.raises(ValueError, match="act is one of"):
        ops.aet_linear_forward(z(2, 3, 4), z(2, 5, 4), act="tanh")
    with pytest.raises(ValueError, match="groups"):
        ops.aet_group_norm_forward(z(2, 3, 4, 6), 4)
    with pytest.raises(ValueError, match="axis of clients"):
        ops.aet_group_norm_backward(z(2, 3, 4, 6), z(2, 3, 4, 6), z(2, 3, 2), z(2, 3, 2), z(2, 6), z(6))
    with pytest.raises(ValueError, match="rstd"):
        ops.aet_group_norm_backward(z(2, 3, 4, 6), z(2, 3, 4, 6), z(2, 3, 2), z(2, 2, 3).transpose(1, 2), z(2, 6), z(2, 6))
    for p in (1.0, -0.1, float("nan")):
        with pytest.raises(AetError, match="p is not in"):
            ops.aet_dropout_forward(z(3, 4), p=p, seed=1)
    with pytest.raises(AetError, match="first_row"):
        ops.aet_dropout_forward(z(3, 4), p=0.5, seed=1, first_row=-1)
    with pytest.raises(AetError, match="overlaps itself"):
        ops.aet_dropout_forward(z(3, 4), p=0.5, seed=1, out=z(1, 4).expand(3, 4))
    with pytest.raises(AetError, match="eps"):
        ops.aet_group_norm_forward(z(2, 3, 4, 6), 2, eps=-1.0)
    with pytest.raises(AetError, match="client after client"):
        ops.aet_linear_backward(z(2, 3, 5), z(2, 4, 4)[:, :3], z(5, 4))
