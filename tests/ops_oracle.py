"""The operators of aet_ops.h in 64 bits on the CPU, from their definitions, and how far an output may be off."""
import math

import numpy as np
import torch

U32 = 2.0 ** -24   # half a unit in the last place of 1, fp32
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def kept(seed, first_row, rows, cols, p):
    """Mask times 1 / (1 - p), rows x cols."""
    if p == 0:
        return torch.ones(rows, cols, dtype=torch.float64)
    half = (cols + 1) // 2
    out = torch.zeros(rows, cols, dtype=torch.float64)
    least = min(math.floor(p * 2 ** 32 + 0.5), 2 ** 32 - 1)
    M = (1 << 64) - 1

    def mix(z):
        z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & M
        z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & M
        return z ^ (z >> 31)

    key = mix((seed + 4 * 0x9E3779B97F4A7C15) & M)
    q = np.array([((first_row + r) * half) & M for r in range(rows)], dtype=np.uint64)[:, None] + np.arange(half, dtype=np.uint64)
    z = np.uint64(key) + (q + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15)
    z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    z = z ^ (z >> np.uint64(31))
    for j in range(cols):
        part = (z[:, j // 2] >> np.uint64(32 * (j % 2))) & np.uint64(0xFFFFFFFF)
        out[:, j] = torch.from_numpy((part >= least).astype(np.float64)) / (1 - p)
    return out


def act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2))
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    if name == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def mask3(shape, seed, first_row, p):
    n, rows, cols = shape
    return kept(seed, first_row, n * rows, cols, p).view(n, rows, cols)


# Bounds.  A sum of K products in fp32 in any order is at most (K - 1) U32 * sum |a b| off, and the products in parts
# drop at most U32 |a b| of each; an output is rounded once, by at most ROUND of it.  The slope of every activation is
# below 1.13, of every slope below 1.  Activations are within 8 U32 of |z| + 1 (their own value is below |z|, one of the
# factors has an error of at most 1.5e-7 = 2.6 U32, exp and reciprocal 1 unit each; exp's argument is off by U32 of it,
# which e^-x x <= 0.37 bounds).


def linear_forward(x, w, bias, residual, name, p, seed, first_row, dtype):
    """(y, bound), (pre, bound); tensors [n, rows, in], [n, out, in], [n, out], [n, rows, out] in 64 bits."""
    K = x.shape[-1]
    z = x @ w.transpose(1, 2)
    S = x.abs() @ w.abs().transpose(1, 2)
    if bias is not None:
        z = z + bias[:, None]
        S = S + bias.abs()[:, None]
    off = (K + 4) * U32 * S
    m = mask3(z.shape, seed, first_row, p)
    y = act(z, name) * m
    yoff = (1.13 * off + (8 * U32 * (z.abs() + 1) if name in ("silu", "gelu") else 0) + 2 * U32 * z.abs()) * m
    if residual is not None:
        y = y + residual
        yoff = yoff + 2 * U32 * (y.abs() + residual.abs())
    r = ROUND[dtype]
    return (y, yoff + r * (y.abs() + yoff)), (z, off + r * (z.abs() + off))


def linear_backward(dy, x, w, pre, name, p, seed, first_row, dtype):
    """(dx, bound), (dw, bound), (db, bound)."""
    m = mask3(dy.shape, seed, first_row, p)
    dz = dy * m
    off = 4 * U32 * dz.abs()
    if name != "none":
        off = off * 1.13 + dz.abs() * (10 * U32 * (pre.abs() + 1) if name in ("silu", "gelu") else 0)
        dz = dz * slope(pre, name)
    r = ROUND[dtype]
    dzr = off + (r * dz.abs() if dtype == torch.bfloat16 else 0)   # dz as the products see it

    def product(a, aoff, b):
        K = a.shape[-1]
        v = a @ b
        o = aoff @ b.abs() + (K + 4) * U32 * ((a.abs() + aoff) @ b.abs())
        return v, o + r * (v.abs() + o)

    db = dz.sum(1)
    o = off.sum(1) + (dz.shape[1] + 4) * U32 * dz.abs().sum(1)
    return (product(dz, dzr, w), product(dz.transpose(1, 2).contiguous(), dzr.transpose(1, 2).contiguous(), x),
            (db, o + r * (db.abs() + o)))


def group_norm_forward(x, groups, gamma, beta, eps, name, dtype):
    """(y, bound), mean, rstd; x [n, batch, positions, channels], gamma and beta [n, channels] in 64 bits."""
    n, b, P, ch = x.shape
    g = x.view(n, b, P, groups, ch // groups)
    mean = g.mean((2, 4), keepdim=True)
    var = (g - mean).square().mean((2, 4), keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    xh = ((g - mean) * rstd).view(x.shape)
    t = xh * gamma[:, None, None] + beta[:, None, None]
    # the mean of M values is off by less than (log2 M + 4) units of the largest when summed in a tree of short runs;
    # 64 units are allowed for, of mean and spread
    big = (g.abs().amax((2, 4), keepdim=True) * rstd).expand(g.shape).reshape(x.shape)
    off = 64 * U32 * ((big + xh.abs()) * gamma.abs()[:, None, None] + beta.abs()[:, None, None])
    y = act(t, name)
    yoff = 1.13 * off + (8 * U32 * (t.abs() + 1) if name in ("silu", "gelu") else 0)
    return (y, yoff + ROUND[dtype] * (y.abs() + yoff)), mean.view(n, b, groups), rstd.view(n, b, groups)


def group_norm_backward(dy, x, mean, rstd, gamma, beta, name, dtype):
    """(dx, bound), (dgamma, bound), (dbeta, bound) from the statistics as they are handed over."""
    n, b, P, ch = x.shape
    G = mean.shape[-1]
    shape5 = (n, b, P, G, ch // G)
    m, s = mean[:, :, None, :, None], rstd[:, :, None, :, None]
    xh = ((x.view(shape5) - m) * s).reshape(x.shape)
    xoff = (4 * U32 * (x.view(shape5).abs() + m.abs()) * s).reshape(x.shape)
    ga, be = gamma[:, None, None], beta[:, None, None]
    t = xh * ga + be
    toff = xoff * ga.abs() + 2 * U32 * (xh.abs() * ga.abs() + be.abs())
    d = dy * slope(t, name)
    doff = dy.abs() * (toff + 10 * U32 * (t.abs() + 1)) if name in ("silu", "gelu") else 2 * U32 * d.abs()
    N = b * P
    dbeta, dgamma = d.sum((1, 2)), (d * xh).sum((1, 2))
    boff = doff.sum((1, 2)) + (N + 4) * U32 * d.abs().sum((1, 2))
    goff = (doff * xh.abs() + d.abs() * xoff).sum((1, 2)) + (N + 4) * U32 * (d * xh).abs().sum((1, 2))
    e, eoff = d * ga, doff * ga.abs()
    M = P * ch // G

    def mean5(v):
        return (v.view(shape5).sum((2, 4), keepdim=True) / M).expand(shape5).reshape(x.shape)

    dx = (e - mean5(e) - xh * mean5(e * xh)) * s.expand(shape5).reshape(x.shape)
    doff = (eoff + mean5(eoff) + xh.abs() * mean5(eoff * xh.abs() + e.abs() * xoff) + xoff * mean5((e * xh).abs())
            + 64 * U32 * (e.abs() + mean5(e.abs()) + xh.abs() * mean5((e * xh).abs()))) * s.expand(shape5).reshape(x.shape)
    r = ROUND[dtype]
    return (dx, doff + r * (dx.abs() + doff)), (dgamma, goff + r * (dgamma.abs() + goff)), (dbeta, boff + r * (dbeta.abs() + boff))


def near(got, want_bound, what):
    """got within the bound of the 64-bit value, everywhere."""
    want, bound = want_bound
    got = got.detach().double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = (got - want).abs() <= bound + 1e-37
    if not bool(fine.all()):
        at = (~fine).nonzero()[0].tolist()
        raise AssertionError(f"{what}: {int((~fine).sum())} of {fine.numel()} values are off, first at {at}: "
                             f"{float(got[tuple(at)])!r}, expected {float(want[tuple(at)])!r} within {float(bound[tuple(at)]):.3g}")
