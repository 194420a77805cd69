"""The operators together: a residual network's gradient against PyTorch's automatic differentiation of the same model in
64 bits on the CPU, and clients that learn in rounds."""
import math
import os
import sys

import pytest
import torch

import ops_oracle as O

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.fail("no GPU visible")
    import residual_clients
    return residual_clients


def reference(net, X, y, dtype):
    """The clients' losses and gradients in 64 bits."""
    w = net.w.double().cpu().requires_grad_()
    n, b = X.shape[:2]
    P, rows = net.positions, X.shape[1] * net.positions

    def v(name):
        at, shape = net.places[name]
        return w[:, at:at + math.prod(shape)].view(n, *shape)

    def mask(k, cols):
        return O.mask3((n, rows, cols), net.seed + (net.blocks + 1) * net.step + k, 0, net.p)

    x = net.patches(X).double().cpu().view(n, rows, -1)
    x = (x @ v("embed").transpose(1, 2) + v("embed_b")[:, None])
    x = x * mask(net.blocks, x.shape[-1])
    for k in range(net.blocks):
        m = x.view(n, b, P, net.groups, -1)
        mean = m.mean((2, 4), keepdim=True)
        var = (m - mean).square().mean((2, 4), keepdim=True)
        t = ((m - mean) / torch.sqrt(var + 1e-5)).view(n, b, P, -1) * v(f"gamma{k}")[:, None, None] + v(f"beta{k}")[:, None, None]
        h = (t * torch.sigmoid(t)).view(n, rows, -1)
        z = h @ v(f"w1{k}").transpose(1, 2) + v(f"b1{k}")[:, None]
        u = z * 0.5 * torch.erfc(-z / math.sqrt(2))
        o = u @ v(f"w2{k}").transpose(1, 2) + v(f"b2{k}")[:, None]
        x = x + o * mask(k, o.shape[-1])
    logits = x.view(n, b, P, -1).mean(2) @ v("head").transpose(1, 2) + v("head_b")[:, None]
    loss = -torch.log_softmax(logits, -1).gather(2, y.long().cpu()[..., None]).mean((1, 2))
    loss.sum().backward()
    return loss.detach(), w.grad


@pytest.mark.parametrize("dtype,tol", [("f32", 1e-5), ("bf16", 0.03)])
def test_gradient_of_the_whole_network(example, dtype, tol):
    """Relative 2-norm of every parameter's gradient.  fp32: some ten operators in a row, each within about 64 units of
    2^-24 of its outputs' size, 4e-6 a value, 1e-5 with sums of values that cancel.  bf16: twelve roundings of 2^-9 (rms
    of a rounding, 2^-8 / sqrt(3)) on the way down and up add up to 2^-9 * sqrt(24) * 1.2 = 0.011; three times that."""
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    net = example.ResidualClients(3, width=48, hidden=100, blocks=2, groups=6, p=0.1, seed=7, dtype=dt, hw=16)
    g = torch.Generator().manual_seed(1)
    X = torch.randn(3, 5, 3, 16, 16, generator=g).cuda()
    y = torch.randint(10, (3, 5), generator=g).cuda()
    net.w += 0.1 * torch.randn(net.w.shape, generator=g).cuda().to(dt)
    want_loss, want = reference(net, X, y, dt)
    loss = net.loss_and_gradient(X, y).double().cpu()
    assert float(((loss - want_loss) / want_loss).abs().max()) < tol
    for name in net.places:
        a, b = net.view(net.g, name).double().cpu(), net.view(want, name)
        assert float((a - b).norm() / b.norm()) < tol, name


def test_clients_learn(example):
    losses = example.train(clients=4, rows=120, a=32, b=64, batch=16, rounds=4, say=lambda s: None)
    assert losses[-1] < 0.7 * losses[0] and losses[0] < 3.5
