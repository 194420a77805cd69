"""The orthogonalised update at sizes that take the larger tiles and split sums, and what it is off by below the rounding of its result."""
import pytest
import torch

from test_gpu_ops_linear import DEV, TYPES, ops  # noqa: F401
from test_gpu_ops_orthogonal import CUBIC, MUON

pytestmark = pytest.mark.gpu


def recurrence(g, steps, polynomial, dtype, eps=1e-7):
    """The definition in this type, client by client, from the shorter side."""
    a, b, c = polynomial
    out = []
    for x in g.to(dtype):
        x = x / (x.double().norm() + eps).to(dtype)
        tall = x.shape[0] > x.shape[1]
        x = x.t().contiguous() if tall else x
        for _ in range(steps):
            p = x @ x.t().contiguous()
            x = a * x + (b * p + c * p @ p) @ x
        out.append(x.t().contiguous() if tall else x)
    return torch.stack(out)


def gradient(size, kind, dtype, seed=3):
    """normal: all singular values of a size; rank k: k of them, and the rounding of the type; decades k: over k decades."""
    n, rows, cols = size
    gen = torch.Generator(device=DEV).manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, device=DEV, dtype=torch.float64)   # noqa: E731
    name, k = kind
    if name == "normal":
        return normal(*size).to(dtype)
    if name == "rank":
        return torch.stack([normal(rows, k) @ normal(k, cols) for _ in range(n)]).to(dtype)
    m = min(rows, cols)
    u, v = (torch.linalg.qr(normal(s, m))[0] for s in (rows, cols))
    return ((u * torch.logspace(0, -k, m, device=DEV, dtype=torch.float64)) @ v.t().contiguous()).expand(n, rows, cols).to(dtype)


def check(ops, g, steps, polynomial, scale=1.0, what=""):   # noqa: F811
    """In the 2-norm.  What is between the steps has 22 bits where the recurrence in fp32 has 24: each of its roundings is at most 4 times as
    large, and they grow from step to step alike, so the call is off by at most 4 times what that recurrence is.  (In bf16 matrices go several steps
    by A alone, as far as that leaves this so.)  In bf16 w is what the result would be rounded to, with which the call leaves its own rounding of
    at most 2^-8 of that: what is left is rounded by 2^-8 of itself.  In fp32 the result is rounded, and scaled, by 2^-24 each."""
    want = recurrence(g, steps, polynomial, torch.float64)
    near = recurrence(g, steps, polynomial, torch.float32).double()
    size = float(want.norm())
    w = -(scale * want).to(g.dtype)
    got = ops.aet_orthogonalise(g, steps=steps, polynomial=polynomial, w=w, keep=1.0, scale=scale)
    off = float((got.double() - (scale * want + w.double())).norm()) / abs(scale) / size
    allowed = 4 * float((near - want).norm()) / size + (2.0 ** -16 if g.dtype == torch.bfloat16 else 2.0 ** -22)
    assert off <= allowed, f"{what}: off by {off:.3g}, allowed {allowed:.3g}"


# tiles of 128 and 256, of both in one call; tall and wide, with ragged sides; products of 2, 4 and 16 parts; several steps by A alone in bf16
LARGE = [(4, 1000, 4090), (4, 4090, 1000), (1, 3900, 4000), (1, 2000, 1900), (1, 1000, 9000), (3, 3000, 3000), (1, 5100, 5000), (1, 1530, 3070)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", LARGE, ids=str)
def test_large(ops, size, dtype):   # noqa: F811
    for kind, steps, scale in ((("normal", 0), 5, 1.0), (("rank", 20), 3, -0.25)):
        check(ops, gradient(size, kind, TYPES[dtype]), steps, MUON, scale, f"{size} {dtype} {kind}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(4, 1000, 4090), (2, 4089, 1001), (3, 2999, 3001)], ids=str)
def test_large_strided_and_in_place(ops, size, dtype):   # noqa: F811
    """Rows that lie apart, results in w's and in g's place: the same as elsewhere, and nothing between the rows."""
    dt = TYPES[dtype]
    n, rows, cols = size
    g, w = gradient(size, ("normal", 0), dt), gradient(size, ("normal", 0), dt, 4)
    want = ops.aet_orthogonalise(g, w=w, keep=0.9, scale=0.5, steps=4)
    place = torch.full((n, rows + 1, cols + 5), 7.0, dtype=dt, device=DEV)
    places = [place[:, 1:, 2:-3] for _ in range(2)]
    for source in (w, g):
        places[0].copy_(source)
        a = dict(g=g, w=places[0]) if source is w else dict(g=places[0], w=w)
        ops.aet_orthogonalise(**a, keep=0.9, scale=0.5, steps=4, out=places[0])
        assert torch.equal(places[0], want)
        assert bool((place[:, 0] == 7).all() and (place[..., :2] == 7).all() and (place[..., -3:] == 7).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", [("normal", 0), ("rank", 1), ("rank", 16), ("rank", 512), ("decades", 3), ("decades", 5)], ids=str)
@pytest.mark.parametrize("size", [(2, 130, 2000), (1, 2000, 130), (1, 520, 2600), (2, 256, 2048), (4, 1000, 4090), (2, 60, 90)], ids=str)
def test_below_the_rounding_of_the_result(ops, size, kind, dtype):   # noqa: F811
    g = gradient(size, kind, TYPES[dtype])
    for polynomial, steps in ((MUON, 5), (MUON, 8), (CUBIC, 10), ((2.0, -1.5, 0.5), 6)):
        check(ops, g, steps, polynomial, what=f"{size} {dtype} {kind} {polynomial} {steps}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_captured_and_replayed(ops, dtype):   # noqa: F811
    """Two graphs with workspaces of their own, replayed in turn and with eager calls between."""
    sizes = ((4, 1000, 4090), (1, 3900, 4000))
    gs = [gradient(s, ("normal", 0), TYPES[dtype]) for s in sizes]
    graphs, outs = [], []
    for g in gs:
        ops.aet_orthogonalise(g)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(ops.aet_orthogonalise(g))
    for k in range(3):
        for g, s in zip(gs, sizes):
            g.copy_(gradient(s, ("normal", 0), TYPES[dtype], 5 + k))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for g, out in zip(gs, outs):
            assert torch.equal(out, ops.aet_orthogonalise(g)), k
