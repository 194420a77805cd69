"""The orthogonalised update against its definition in 64 bits."""
import pytest
import torch

import ops_oracle as O
from test_gpu_ops_linear import DEV, TYPES, d64, ops, rand  # noqa: F401

pytestmark = pytest.mark.gpu
MUON, CUBIC = (3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0)


def definition(g, steps, polynomial, eps=1e-7):
    """In 64 bits, client by client."""
    a, b, c = polynomial
    out = []
    for x in g:
        x = x / (x.norm() + eps)
        for _ in range(steps):
            p = x @ x.t()
            x = a * x + (b * p + c * p @ p) @ x
        out.append(x)
    return torch.stack(out)


def close(got, want, scale, w, keep, steps, dt, what):
    """In the 2-norm.  A step's products and roundings are off by some 10 e of X's norm, e = 2^-22: three products of two factors in two
    parts each (2^-23), and four roundings; sums of K products in fp32 add as independent roundings of 2^-24, less than that.  Errors
    grow from step to step as what they lie in does, in the mean as X's own norm: 8 times the sum over the steps is allowed for
    directions that grow more.  With 5 steps that is 1e-4; a second part that is lost gives 1e-3 (fp16 rounds by 2^-12)."""
    bound = 8 * 10 * 2.0 ** -22 * max(steps, 1) * float((scale * want).norm())
    total = scale * want + (0 if w is None else keep * w)
    bound += O.ROUND[dt] * float(total.norm()) + 2 * O.U32 * float(total.norm() + (0 if w is None else (keep * w).norm()))
    off = float((d64(got) - total).norm())
    assert off <= bound, f"{what}: off by {off:.3g}, allowed {bound:.3g} of {float(total.norm()):.3g}"


# n, rows, cols: single values, rows and columns; wide, square and tall; odd sizes; sides that end inside tiles of every kind
SIZES = [(1, 1, 1), (3, 1, 40), (2, 40, 1), (2, 7, 5), (1, 16, 16), (1, 64, 64), (3, 33, 130), (2, 130, 33), (16, 128, 784), (1, 127, 129), (1, 200, 200),
         (2, 257, 771), (1, 1001, 515), (1, 320, 1024), (5, 250, 250), (1, 640, 640), (40, 10, 30), (1, 128, 5000), (2, 130, 2000),
         (3, 1500, 70), (1, 520, 2600)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_orthogonalise(ops, size, dtype):   # noqa: F811
    n, rows, cols = size
    dt = TYPES[dtype]
    for k, (polynomial, steps, with_w, pad, skip) in enumerate(((MUON, 5, False, 0, 0), (MUON, 5, True, 3, 1), (CUBIC, 8, False, 8, 0), (MUON, 1, True, 0, 0),
                                                                (MUON, 0, False, 0, 0), (MUON, 7, False, 0, 0), (CUBIC, 14, False, 0, 0))):
        gen = torch.Generator().manual_seed(rows + k)
        g = rand(gen, size, dt, 1e-3 if k else 30.0, pad, skip)
        w = rand(gen, size, dt, pad=pad, skip=skip) if with_w else None
        y = ops.aet_orthogonalise(g, steps=steps, polynomial=polynomial, w=w, keep=0.99, scale=-0.2)
        close(y, definition(d64(g), steps, polynomial), -0.2, d64(w), 0.99, steps, dt, f"{size} {dtype} {k}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(2, 64, 96), (1, 300, 200), (1, 1400, 130), (2, 256, 2048)], ids=str)
def test_few_directions(ops, size, dtype):   # noqa: F811
    """Gradients of mini-batches: a rank below the sides, and singular values over five orders."""
    dt = TYPES[dtype]
    gen = torch.Generator().manual_seed(5)
    n, rows, cols = size
    low = (torch.randn(n, rows, 12, generator=gen) @ torch.randn(n, 12, cols, generator=gen)).to(dt).to(DEV)
    close(ops.aet_orthogonalise(low), definition(d64(low), 5, MUON), 1.0, None, 1.0, 5, dt, "low rank")
    u, v = (torch.linalg.qr(torch.randn(s, s, generator=gen).double())[0] for s in (rows, cols))
    m = min(rows, cols)
    g = ((u[:, :m] * torch.logspace(0, -5, m).double()) @ v[:, :m].t()).expand(n, rows, cols).to(dt).to(DEV)
    close(ops.aet_orthogonalise(g), definition(d64(g), 5, MUON), 1.0, None, 1.0, 5, dt, "five orders")


def test_the_result_is_orthogonal(ops):   # noqa: F811
    """The cubic polynomial's fixed point: X X^T = 1, to rounding, once all singular values are there."""
    gen = torch.Generator().manual_seed(5)
    u = torch.linalg.qr(torch.randn(96, 96, generator=gen))[0]
    g = (u * torch.linspace(0.5, 1.0, 96)).contiguous().to(DEV)   # (the factor comes column after column)
    x = d64(ops.aet_orthogonalise(g, steps=14, polynomial=CUBIC))
    assert float((x @ x.t() - torch.eye(96).double()).norm()) < 96 * 2.0 ** -20
    assert float((x - d64(u)).norm()) < 96 * 2.0 ** -20


@pytest.mark.parametrize("scale", [1e-30, 1e-18, 1.0, 1e18, 3e37])
def test_scales_of_the_gradient(ops, scale):   # noqa: F811
    """Squares beyond fp32's range either way are no matter (eps is beside them)."""
    gen = torch.Generator().manual_seed(2)
    g = (torch.randn(2, 40, 70, generator=gen) * scale).to(DEV)
    close(ops.aet_orthogonalise(g, eps=0.0), definition(d64(g), 5, MUON, 0.0), 1.0, None, 1.0, 5, torch.float32, f"{scale}")
    close(ops.aet_orthogonalise(g), definition(d64(g), 5, MUON), 1.0, None, 1.0, 5, torch.float32, f"{scale}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_zeros_and_values_that_are_not_finite(ops, dtype):   # noqa: F811
    dt = TYPES[dtype]
    gen = torch.Generator().manual_seed(2)
    g, w = rand(gen, (4, 30, 50), dt), rand(gen, (4, 30, 50), dt)
    want = ops.aet_orthogonalise(g, w=w, keep=0.5)
    g[1] = 0
    g[2, 29, 49], g[3, 0, 0] = float("nan"), float("inf")
    for eps in (1e-7, 0.0):
        y = ops.aet_orthogonalise(g, w=w, keep=0.5, eps=eps)
        assert torch.equal(y[1], (0.5 * w[1].float()).to(dt)) and bool(y[2:].isnan().all())
    assert torch.equal(ops.aet_orthogonalise(g, w=w, keep=0.5)[0], want[0])
    assert bool(ops.aet_orthogonalise(g, steps=0)[2:].isnan().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(2, 50, 70), (2, 70, 50), (1, 300, 130)], ids=str)
def test_in_place_and_strided(ops, size, dtype):   # noqa: F811
    dt = TYPES[dtype]
    gen = torch.Generator().manual_seed(2)
    g, w = rand(gen, size, dt), rand(gen, size, dt)
    want = ops.aet_orthogonalise(g, w=w, keep=0.9, scale=0.1)
    a = w.clone()
    assert ops.aet_orthogonalise(g, w=a, keep=0.9, scale=0.1, out=a) is not None and torch.equal(a, want)
    a = g.clone()
    ops.aet_orthogonalise(a, w=w, keep=0.9, scale=0.1, out=a)
    assert torch.equal(a, want)
    place = torch.full((size[0], size[1] + 1, size[2] + 5), 7.0, dtype=dt, device=DEV)
    ops.aet_orthogonalise(g, w=w, keep=0.9, scale=0.1, out=place[:, 1:, 2:-3])
    assert torch.equal(place[:, 1:, 2:-3], want) and bool((place[:, 0] == 7).all() and (place[..., :2] == 7).all() and (place[..., -3:] == 7).all())
    # one matrix for all, and two axes
    one = ops.aet_orthogonalise(g[0], w=w[0], keep=0.9, scale=0.1)
    close(one[None], definition(d64(g[:1]), 5, MUON), 0.1, d64(w[:1]), 0.9, 5, dt, "two axes")
    same = ops.aet_orthogonalise(g[:1].expand(3, *size[1:]))
    assert torch.equal(same[0], same[2])


def test_other_polynomials(ops):   # noqa: F811
    """Values that the scales have to follow: far above 1, and far below."""
    gen = torch.Generator().manual_seed(4)
    g = rand(gen, (2, 60, 90), torch.float32)
    for steps, polynomial in ((3, (20.0, 0.0, 0.0)), (4, (0.01, 0.0, 0.0)), (2, (3.0, 2.0, 1.0)), (1, (0.0, 1.0, 0.0)), (2, (-2.0, 1.5, -0.5)), (1, (0.0, 0.0, 1.0))):
        close(ops.aet_orthogonalise(g, steps=steps, polynomial=polynomial), definition(d64(g), steps, polynomial), 1.0, None, 1.0, 4 * steps,
              torch.float32, f"{polynomial}")


def test_an_eps_far_above_the_gradient(ops):   # noqa: F811
    """Singular values whose squares are nothing in 64 bits."""
    gen = torch.Generator().manual_seed(4)
    g, w = rand(gen, (2, 60, 90), torch.float32), rand(gen, (2, 60, 90), torch.float32)
    for eps in (1e30, 1e100, 1e150, 1e156, 1e160, 1e165, 1e200, 1e308):
        for polynomial in (MUON, (0.0, 1.0, 0.0)):
            assert torch.equal(ops.aet_orthogonalise(g, w=w, keep=0.5, eps=eps, polynomial=polynomial), 0.5 * w), eps


def test_nothing_to_do(ops):   # noqa: F811
    for shape in ((0, 3, 4), (2, 0, 4), (2, 3, 0), (0, 5)):
        assert ops.aet_orthogonalise(torch.ones(*shape, device=DEV)).shape == shape


def test_captured_and_replayed_with_another_graph(ops):   # noqa: F811
    """Two graphs with workspaces of their own, replayed in turn and with eager calls between."""
    gen = torch.Generator().manual_seed(6)
    sizes = ((2, 130, 200), (3, 96, 64))
    gs = [rand(gen, s, torch.float32) for s in sizes]
    graphs, outs = [], []
    for g in gs:
        ops.aet_orthogonalise(g)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(ops.aet_orthogonalise(g))
    for k in range(4):
        for g, s in zip(gs, sizes):
            g.copy_(rand(gen, s, torch.float32))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for g, out in zip(gs, outs):
            assert torch.equal(out, ops.aet_orthogonalise(g)), k


def test_the_same_bits_every_time_and_on_other_streams(ops):   # noqa: F811
    gen = torch.Generator().manual_seed(6)
    g = rand(gen, (2, 300, 500), torch.bfloat16)
    want = ops.aet_orthogonalise(g)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    a, b = ops.aet_orthogonalise(g, stream=other), ops.aet_orthogonalise(g)
    torch.cuda.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want)


def test_binding(ops):   # noqa: F811
    from paper_2112_13935_amd import AetError
    z = lambda *s: torch.ones(*s, device=DEV)   # noqa: E731
    tensors = dict(g=z(2, 3, 4), w=z(2, 3, 4), out=z(2, 3, 4))
    call = lambda g, w, out: ops.aet_orthogonalise(g, w=w, out=out)   # noqa: E731
    before = {k: t._version for k, t in tensors.items()}
    call(**tensors)
    assert all((t._version > before[k]) == (k == "out") for k, t in tensors.items())
    for k, t in tensors.items():
        with pytest.raises(ValueError, match="requires a gradient"):
            call(**dict(tensors, **{k: t.clone().requires_grad_()}))
        for bad in (t.half(), t.cpu(), t.new_zeros(*t.shape, 2)[..., 0], t.new_zeros(2, 3, 5), t[None]):
            with pytest.raises(ValueError):
                call(**dict(tensors, **{k: bad}))
    for more, what in ((dict(steps=-1), "steps"), (dict(steps=101), "steps"), (dict(eps=-1.0), "eps"), (dict(eps=float("inf")), "eps"), (dict(scale=float("nan")), "finite"),
                       (dict(polynomial=(float("inf"), 0.0, 0.0)), "finite"), (dict(polynomial=(1e9, 0.0, 0.0), steps=2), "grow"), (dict(polynomial=(0.0, 0.0, 1e20)), "grow"),
                       (dict(out=z(1, 3, 4).expand(2, 3, 4)), "overlaps itself")):
        with pytest.raises(AetError, match=what):
            ops.aet_orthogonalise(z(2, 3, 4), **more)
