"""Layer normalisation of rows and its gradient against their definitions in 64 bits."""
import pytest
import torch

import ops_oracle as O
from test_gpu_ops_linear import DEV, TYPES, d64, ops, rand  # noqa: F401

pytestmark = pytest.mark.gpu

# n, rows, cols: a value, less than a piece, whole and odd pieces; each number of lanes, waves and pieces a row takes, one column more
# and less than it holds in either type; rows too long for registers; single rows and rows that end inside strips
SIZES = [(1, 1, 1), (2, 3, 3), (1, 70, 4), (2, 65, 7), (1, 300, 16), (3, 33, 17), (1, 40, 33), (2, 17, 64), (1, 9, 127), (1, 130, 129), (2, 20, 255), (1, 1, 784),
         (16, 5, 771), (1, 37, 1000), (1, 12, 1025), (3, 11, 2047), (1, 520, 2050), (1, 6, 4096), (2, 3, 4097), (1, 9, 8191), (1, 3, 8200),
         (1, 4, 16380), (1, 2, 16388), (2, 2, 20001), (1, 3, 40000), (40, 1, 50), (1, 1, 70001)]


def forward(x, res, gamma, beta, eps, dt):
    """(y, bound), (h, bound), mean, rstd in 64 bits: the group norm of one position and one group."""
    h = x if res is None else x + res
    n, rows, cols = h.shape
    (y, off), mean, rstd = O.group_norm_forward(h[:, :, None], 1, gamma, beta, eps, "none", dt)
    hoff = O.U32 * h.abs()
    return (y[:, :, 0], off[:, :, 0]), (h, hoff + O.ROUND[dt] * (h.abs() + hoff)), mean[..., 0], rstd[..., 0]


def backward(dy, x, mean, rstd, gamma, dh, dt):
    zero = torch.zeros_like(gamma)
    (dx, off), g, b = O.group_norm_backward(dy[:, :, None], x[:, :, None], mean[..., None], rstd[..., None], gamma, zero, "none", dt)
    dx, off = dx[:, :, 0], off[:, :, 0]
    if dh is not None:
        off = off + O.U32 * (dx.abs() + dh.abs()) * 2 + O.ROUND[dt] * dh.abs()
        dx = dx + dh
    return (dx, off), g, b


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_layer_norm(ops, size, dtype):   # noqa: F811
    n, rows, cols = size
    dt = TYPES[dtype]
    for k, (with_res, with_params, pad, skip) in enumerate(((False, True, 0, 0), (True, True, 0, 0), (True, False, 3, 1), (False, True, 8, 0))):
        g = torch.Generator().manual_seed(cols + k)
        x, dy, dh = (rand(g, (n, rows, cols), dt, s, pad, skip) for s in (2.0, 1.0, 1.0))
        res = rand(g, (n, rows, cols), dt, pad=pad, skip=skip) if with_res else None
        gamma, beta = (rand(g, (n, cols), dt, pad=pad, skip=skip) if with_params else None for _ in range(2))
        y, h, mean, rstd = ops.aet_layer_norm_forward(x, gamma, beta, residual=res, eps=1e-3)
        one, zero = torch.ones(n, cols).double(), torch.zeros(n, cols).double()
        wy, wh, wm, wr = forward(d64(x), d64(res), one if gamma is None else d64(gamma), zero if beta is None else d64(beta), 1e-3, dt)
        what = f"{size} {dtype} {k}"
        O.near(y, wy, "y " + what)
        assert (h is None) == (res is None)
        if h is not None:
            O.near(h, wh, "h " + what)
        O.near(mean, (wm, 64 * O.U32 * (wm.abs() + 1 / wr)), "mean " + what)
        O.near(rstd, (wr, 64 * O.U32 * wr * (1 + O.U32 * (wm * wr).square())), "rstd " + what)
        stream = dh if with_res else None
        dx, dgamma, dbeta = ops.aet_layer_norm_backward(dy, x if h is None else h, mean, rstd, gamma, dh=stream)
        wx, wg, wb = backward(d64(dy), d64(x if h is None else h), d64(mean), d64(rstd), one if gamma is None else d64(gamma), d64(stream), dt)
        O.near(dx, wx, "dx " + what)
        if gamma is None:
            assert dgamma is None and dbeta is None
        else:
            O.near(dgamma, wg, "dgamma " + what)
            O.near(dbeta, wb, "dbeta " + what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(5, 7, 40), (3, 200, 771), (64, 1, 16), (2, 9, 20001)], ids=str)
def test_one_gamma_for_all_clients(ops, size, dtype):   # noqa: F811
    n, rows, cols = size
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(rows)
    x, dy, gamma, beta = rand(g, size, dt), rand(g, size, dt), rand(g, (cols,), dt), rand(g, (cols,), dt)
    y, _, mean, rstd = ops.aet_layer_norm_forward(x, gamma, beta)
    (wy, off), _, _, _ = forward(d64(x), None, d64(gamma).expand(n, cols), d64(beta).expand(n, cols), 1e-5, dt)
    O.near(y, (wy, off), "y")
    dx, dgamma, dbeta = ops.aet_layer_norm_backward(dy, x, mean, rstd, gamma)
    flat = lambda t: d64(t).reshape(1, n * rows, *t.shape[2:])   # noqa: E731
    wx, wg, wb = backward(flat(dy), flat(x), flat(mean), flat(rstd), d64(gamma)[None], None, dt)
    O.near(dx.view(1, n * rows, cols), wx, "dx")
    O.near(dgamma[None], wg, "dgamma")
    O.near(dbeta[None], wb, "dbeta")


def test_gradient_against_differences(ops):   # noqa: F811
    """Of a weighted sum of the outputs of the definition in 64 bits, at an input in fp32."""
    g = torch.Generator().manual_seed(3)
    x, dy, gamma, beta = rand(g, (1, 3, 24), torch.float32), rand(g, (1, 3, 24), torch.float32), rand(g, (24,), torch.float32), rand(g, (24,), torch.float32)
    _, _, mean, rstd = ops.aet_layer_norm_forward(x, gamma, beta)
    dx, dgamma, dbeta = ops.aet_layer_norm_backward(dy, x, mean, rstd, gamma)
    t = [d64(v) for v in (x[0], gamma, beta)]

    def f(x, gamma, beta):
        m = x.mean(-1, keepdim=True)
        return float((((x - m) / torch.sqrt((x - m).square().mean(-1, keepdim=True) + 1e-5) * gamma + beta) * d64(dy[0])).sum())

    step = 2.0 ** -17   # third derivatives of some tens: the difference is off by 1e-9, rounding by 1e-10
    for k, got in ((0, dx[0]), (1, dgamma), (2, dbeta)):
        for i in range(t[k].numel()):
            up, down = [v.clone() for v in t], [v.clone() for v in t]
            up[k].view(-1)[i] += step
            down[k].view(-1)[i] -= step
            assert abs((f(*up) - f(*down)) / (2 * step) - float(got.reshape(-1)[i])) < 2e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [21, 515, 1023, 4099, 40001])
def test_in_place(ops, cols, dtype):   # noqa: F811
    """Outputs in their inputs' places, at sizes whose last pieces share columns, are the outputs elsewhere."""
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(cols)
    x, res, dy, dh = (rand(g, (2, 37, cols), dt) for _ in range(4))
    gamma = rand(g, (2, cols), dt)
    y, h, mean, rstd = ops.aet_layer_norm_forward(x, gamma, residual=res)
    for places in ((0, 1), (1, 0)):
        a = [x.clone(), res.clone()]
        ops.aet_layer_norm_forward(a[0], gamma, residual=a[1], out=(a[places[0]], a[places[1]]))
        assert torch.equal(a[places[0]], y) and torch.equal(a[places[1]], h)
    want = ops.aet_layer_norm_backward(dy, h, mean, rstd, gamma, dh=dh)
    for which in (0, 1):
        a = [dy.clone(), dh.clone()]
        got = ops.aet_layer_norm_backward(a[0], h, mean, rstd, gamma, dh=a[1], out=(a[which], None, None))
        assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_wanted(ops, dtype):   # noqa: F811
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(1)
    x, dy, gamma = rand(g, (3, 50, 40), dt), rand(g, (3, 50, 40), dt), rand(g, (3, 40), dt)
    _, _, mean, rstd = ops.aet_layer_norm_forward(x, gamma)
    want = ops.aet_layer_norm_backward(dy, x, mean, rstd, gamma)
    dx, a, b = ops.aet_layer_norm_backward(dy, x, mean, rstd, gamma, need=(True, False))
    assert a is None and b is None and torch.equal(dx, want[0])
    dx, a, b = ops.aet_layer_norm_backward(dy, x, mean, rstd, gamma, need=(False, True))
    assert dx is None and torch.equal(a, want[1]) and torch.equal(b, want[2])
    # the gradient of beta alone, without gamma, into a place of other strides
    place = torch.full((3, 50), 7.0, dtype=dt, device=DEV)
    _, a, b = ops.aet_layer_norm_backward(dy, x, mean, rstd, need=(False, False), out=(None, None, place[:, 5:45]))
    assert a is None and torch.equal(b, want[2]) and bool((place[:, :5] == 7).all() and (place[:, 45:] == 7).all())
    assert ops.aet_layer_norm_backward(dy, x, mean, rstd, gamma, need=(False, False)) == (None, None, None)
    # rows that are one row, clients that are one client
    same = ops.aet_layer_norm_forward(x[:1, :1].expand(3, 50, 40), gamma)
    once = ops.aet_layer_norm_forward(x[:1, :1].expand(3, 50, 40).contiguous(), gamma)
    assert all(torch.equal(p, q) for p, q in zip((same[0], *same[2:]), (once[0], *once[2:])))


def test_sizes_of_zero(ops):   # noqa: F811
    z = lambda *s: torch.ones(*s, device=DEV)   # noqa: E731
    for shape in ((0, 3, 4), (2, 0, 4), (0, 4)):
        y, _, mean, rstd = ops.aet_layer_norm_forward(z(*shape))
        assert y.shape == shape and mean.shape == shape[:-1]
        out = ops.aet_layer_norm_backward(z(*shape), z(*shape), mean, rstd, z(4))
        assert out[0].shape == shape and bool((out[1] == 0).all() and (out[2] == 0).all()), shape
    y, _, mean, rstd = ops.aet_layer_norm_forward(z(2, 3, 0), eps=0.25)
    assert y.shape == (2, 3, 0) and bool((mean == 0).all() and (rstd == 2).all())
    out = ops.aet_layer_norm_backward(z(2, 3, 0), z(2, 3, 0), mean, rstd, z(2, 0))
    assert [t.shape for t in out] == [(2, 3, 0), (2, 0), (2, 0)]
    out = ops.aet_layer_norm_backward(z(2, 0, 4), z(2, 0, 4), z(2, 0), z(2, 0), z(2, 4))
    assert bool((out[1] == 0).all() and (out[2] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [40, 771, 40001])
def test_values_that_are_not_finite_stay_in_their_row(ops, cols, dtype):   # noqa: F811
    dt = TYPES[dtype]
    g = torch.Generator().manual_seed(7)
    x, dy, gamma = rand(g, (1, 9, cols), dt), rand(g, (1, 9, cols), dt), rand(g, (cols,), dt)
    y, _, mean, rstd = ops.aet_layer_norm_forward(x, gamma)
    dx = ops.aet_layer_norm_backward(dy, x, mean, rstd, gamma)[0]
    bad = x.clone()
    bad[0, 4, cols - 1], bad[0, 6, 0] = float("nan"), float("inf")
    by, _, bm, br = ops.aet_layer_norm_forward(bad, gamma)
    bx, bg, _ = ops.aet_layer_norm_backward(dy, bad, bm, br, gamma)
    fine = [r for r in range(9) if r not in (4, 6)]
    assert torch.equal(by[0, fine], y[0, fine]) and torch.equal(bx[0, fine], dx[0, fine])
    assert bool(by[0, [4, 6]].isnan().all() and bx[0, [4, 6]].isnan().all() and bg.isnan().all())


def test_large_and_small_values(ops):   # noqa: F811
    """The mean is taken out before squares are added: an offset of 1e4 leaves the spread of 1, values of 1e-18 theirs."""
    g = torch.Generator().manual_seed(9)
    for scale, shift, eps in ((1.0, 1e4, 1e-5), (1e-18, 0.0, 0.0), (1e15, 0.0, 1e-5)):
        x = (torch.randn(1, 5, 500, generator=g) * scale + shift).to(DEV)
        y, _, mean, rstd = ops.aet_layer_norm_forward(x, eps=eps)
        one, zero = torch.ones(1, 500).double(), torch.zeros(1, 500).double()
        wy, _, wm, wr = forward(d64(x), None, one, zero, eps, torch.float32)
        O.near(y, wy, f"y {scale} {shift}")


def test_the_same_bits_every_time_and_on_other_streams(ops):   # noqa: F811
    g = torch.Generator().manual_seed(5)
    x, dy, gamma = rand(g, (2, 1500, 515), torch.bfloat16), rand(g, (2, 1500, 515), torch.bfloat16), rand(g, (2, 515), torch.bfloat16)
    y, _, mean, rstd = ops.aet_layer_norm_forward(x, gamma)
    want = (y, *ops.aet_layer_norm_backward(dy, x, mean, rstd, gamma))
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for stream in (None, other, None):
        y, _, m, r = ops.aet_layer_norm_forward(x, gamma, stream=stream)
        got = (y, *ops.aet_layer_norm_backward(dy, x, m, r, gamma, stream=stream))
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_captured_and_replayed(ops):   # noqa: F811
    g = torch.Generator().manual_seed(6)
    x, res, dy, gamma = (rand(g, s, torch.float32) for s in ((2, 600, 300), (2, 600, 300), (2, 600, 300), (300,)))

    def step():
        y, h, mean, rstd = ops.aet_layer_norm_forward(x, gamma, residual=res)
        return (y, h, *ops.aet_layer_norm_backward(dy, h, mean, rstd, gamma, dh=y))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        x.copy_(rand(g, (2, 600, 300), torch.float32))
        dy.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, step())), k


def calls(ops):   # noqa: F811
    z = lambda *s: torch.ones(*s, device=DEV)   # noqa: E731
    return {
        "forward": (lambda x, gamma, beta, residual, y, h: ops.aet_layer_norm_forward(x, gamma, beta, residual=residual, out=(y, h)),
                    dict(x=z(2, 3, 4), gamma=z(2, 4), beta=z(2, 4), residual=z(2, 3, 4), y=z(2, 3, 4), h=z(2, 3, 4))),
        "backward": (lambda dy, x, mean, rstd, gamma, dh, dx, dgamma, dbeta: ops.aet_layer_norm_backward(
            dy, x, mean, rstd, gamma, dh=dh, out=(dx, dgamma, dbeta)),
            dict(dy=z(2, 3, 4), x=z(2, 3, 4), mean=z(2, 3), rstd=z(2, 3), gamma=z(2, 4), dh=z(2, 3, 4), dx=z(2, 3, 4), dgamma=z(2, 4),
                 dbeta=z(2, 4)))}


PLACES = {"forward": ["y", "h"], "backward": ["dx", "dgamma", "dbeta"]}


@pytest.mark.parametrize("name", sorted(PLACES))
def test_binding(ops, name):   # noqa: F811
    """Gradients that nobody records, tensors that do not agree, versions of what is written."""
    call, tensors = calls(ops)[name]
    before = {k: t._version for k, t in tensors.items()}
    call(**tensors)
    assert all((t._version > before[k]) == (k in PLACES[name]) for k, t in tensors.items())
    for k in tensors:
        with pytest.raises(ValueError, match="requires a gradient"):
            call(**dict(tensors, **{k: tensors[k].clone().requires_grad_()}))
        for how in ("type", "device", "last stride", "longer"):
            t = tensors[k]
            t = {"type": t.bfloat16(), "device": t.cpu(), "last stride": t.new_zeros(*t.shape, 2)[..., 0],
                 "longer": t.new_zeros(*t.shape[:-1], t.shape[-1] + 1)}[how]
            with pytest.raises(ValueError):
                call(**dict(tensors, **{k: t}))
    torch.cuda.synchronize()


def test_arguments_that_do_not_agree(ops):   # noqa: F811
    from paper_2112_13935_amd import AetError
    z = lambda *s: torch.ones(*s, device=DEV)   # noqa: E731
    with pytest.raises(ValueError, match="no residual"):
        ops.aet_layer_norm_forward(z(2, 3), out=(None, z(2, 3)))
    x = z(2, 3)
    with pytest.raises(AetError, match="the same"):
        ops.aet_layer_norm_forward(z(2, 3), residual=z(2, 3), out=(x, x))
    with pytest.raises(AetError, match="eps"):
        ops.aet_layer_norm_forward(z(2, 3), eps=-1.0)
    with pytest.raises(AetError, match="overlaps itself"):
        ops.aet_layer_norm_forward(z(2, 3), out=(z(1, 3).expand(2, 3), None))
    with pytest.raises(ValueError, match="axis of clients"):
        ops.aet_layer_norm_backward(z(2, 3, 4), z(2, 3, 4), z(2, 3), z(2, 3), z(2, 4), out=(None, z(2, 4), z(4)))
