"""The operators that users compose residual blocks of clients' models from, as cases that can be
timed and compared: a linear layer with bias, activation, dropout and residual in its epilogue,
group normalisation with an activation on channels-last maps, and dropout from the counter
generator; each forward and backward, for one model or many clients' models side by side.

A case names the operator, the direction, the type and the sizes; `run` is one call through the
public entry points, or, where `own` is false, the same in elementary torch operations in 32 bits.
`listed` has the layers of workloads.py's models and generic ones from a single row to thousands;
`draw` gives more of the same ranges.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5

#: What a case of each operator says where it says nothing else.
LINEAR = dict(back=False, dtype="f32", n=1, rows=1, inp=784, out=128, act="relu", bias=True, p=0.0, residual=False,
              pre=False,      # forward: the values before the activation come back too, for the gradient
              pad=0,          # x's rows lie this many elements further apart than they are long
              first_row=0)    # number of the first row in the dropout's counters
NORM = dict(back=False, dtype="f32", n=1, batch=1, hw=784, groups=4, width=4, act="silu")   # width: channels of a group
DROPOUT = dict(back=False, dtype="f32", rows=1, cols=784, p=0.1, residual=False, first_row=0)


def listed():
    return [
        # A single sample through the hidden layer of the MLP workload: what one call costs.
        dict(name="linear_row_f32_784_128", op="linear"),
        # One row through a square layer with a residual: the weights are read once, as in serving a single request.
        dict(name="linear_row_bf16_4096", op="linear", dtype="bf16", inp=4096, out=4096, act="gelu", residual=True),
        # The MLP workload's hidden layer: 16 clients with weights and mini-batches of their own, in training.
        dict(name="linear_clients16_f32_784_128", op="linear", n=16, rows=32, pre=True),
        # Odd sizes everywhere, rows of a wider array, three clients, dropout and residual: the second half of a block.
        dict(name="linear_odd_f32_1155_771", op="linear", n=3, rows=1001, inp=1155, out=771, act="silu", p=0.1,
             residual=True, pre=True, pad=2),
        # The first half of a wide block in training, many rows.
        dict(name="linear_large_bf16_4096", op="linear", dtype="bf16", rows=16384, inp=4096, out=4096, act="gelu",
             p=0.1, pre=True),
        # The gradient of a hidden layer for 64 clients with mini-batches of 64: reading and writing weights counts.
        dict(name="linear_back_clients64_f32", op="linear", back=True, n=64, rows=64, inp=1024, out=512),
        # The gradient of a wide layer for four clients: the largest work.
        dict(name="linear_back_large_bf16", op="linear", back=True, dtype="bf16", n=4, rows=4096, inp=2048, out=8192,
             act="gelu", p=0.1),
        # One sample's 28 x 28 maps of 16 channels: what one call costs.
        dict(name="norm_one_f32_28", op="norm"),
        # The maps behind the first convolutions of the CNN workload: 32 clients, mini-batches of 64.
        dict(name="norm_maps_f32_32", op="norm", n=32, batch=64, hw=1024, groups=8, width=4),
        # The gradient on large maps of many channels, where a sample does not fit one compute unit.
        dict(name="norm_back_large_bf16_64", op="norm", back=True, dtype="bf16", n=16, batch=8, hw=4096, groups=32, width=10),
        # A mini-batch of 32 hidden vectors of the MLP workload: what one call costs.
        dict(name="dropout_small_f32_128", op="dropout", rows=32, cols=128),
        # A block's outputs onto its residual stream, many rows.
        dict(name="dropout_large_bf16_4096", op="dropout", dtype="bf16", rows=16384, cols=4096, residual=True),
    ]


def _whole(case):
    return {**{"linear": LINEAR, "norm": NORM, "dropout": DROPOUT}[case["op"]], **case}


def work(case):
    """Each input read once, each output written once; two operations per multiply-add of the products,
    and for what is element by element a round count per value."""
    c = _whole(case)
    e = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "linear":
        n, R, I, O = c["n"], c["rows"], c["inp"], c["out"]
        if c["back"]:   # x, W, dy, z; dx, dW, db
            z = R * O if c["act"] != "none" else 0
            return {"bytes": e * n * (2 * R * I + 2 * O * I + R * O + z + O), "flops": 4 * n * R * I * O}
        return {"bytes": e * n * (R * I + O * I + R * O * (1 + c["residual"] + c["pre"]) + O * c["bias"]),
                "flops": 2 * n * R * I * O}
    if c["op"] == "norm":
        samples, C = c["n"] * c["batch"], c["groups"] * c["width"]
        values = samples * c["hw"] * C
        if c["back"]:
            return {"bytes": e * (3 * values + 4 * c["n"] * C) + 8 * samples * c["groups"], "flops": 20 * values}
        return {"bytes": e * (2 * values + 2 * c["n"] * C) + 8 * samples * c["groups"], "flops": 12 * values}
    values = c["rows"] * c["cols"]
    return {"bytes": e * values * (2 + c["residual"]), "flops": 10 * values}


class State:
    pass


def _counter_seed(seed):
    return (seed * 0x9E3779B97F4A7C15 + 0x1234567) % (1 << 64)


def prepare(case, seed):
    """Inputs, weights and incoming gradients of a training step, or of one request, on the GPU."""
    c = _whole(case)
    dev, dt = torch.device("cuda:0"), TYPES[c["dtype"]]
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def normal(*shape, scale=1.0, shift=0.0):
        t = torch.empty(*shape, device=dev, dtype=dt)
        t.normal_(shift, scale, generator=g)
        return t

    s = State()
    s.case, s.seed = c, _counter_seed(seed)
    if c["op"] == "linear":
        n, R, I, O = c["n"], c["rows"], c["inp"], c["out"]
        s.x = normal(n, R, I + c["pad"])[:, :, :I]
        s.w = normal(n, O, I, scale=1 / math.sqrt(I))
        s.b = normal(n, O, scale=0.1) if c["bias"] else None
        s.res = normal(n, R, O) if c["residual"] else None
        if c["back"]:
            s.dy = normal(n, R, O, scale=0.1)
            s.z = normal(n, R, O) if c["act"] != "none" else None
    elif c["op"] == "norm":
        n, b, P, C = c["n"], c["batch"], c["hw"], c["groups"] * c["width"]
        s.x = normal(n, b, P, C, shift=0.5)
        s.gamma = normal(n, C, scale=0.1, shift=1.0)
        s.beta = normal(n, C, scale=0.1)
        if c["back"]:
            s.dy = normal(n, b, P, C, scale=0.1)
            # the statistics that the forward pass handed over
            xg = s.x.view(n * b, P, c["groups"], c["width"])
            s.mean = torch.empty(n * b, c["groups"], device=dev)
            s.rstd = torch.empty(n * b, c["groups"], device=dev)
            for k in range(n):   # by client, for the room that it takes
                part = xg[k * b:(k + 1) * b].float()
                m = part.mean((1, 3), keepdim=True)
                s.mean[k * b:(k + 1) * b] = m[:, 0, :, 0]
                s.rstd[k * b:(k + 1) * b] = ((part - m).square().mean((1, 3)) + EPS).rsqrt()
            s.mean, s.rstd = s.mean.view(n, b, -1), s.rstd.view(n, b, -1)
    else:
        s.x = normal(c["rows"], c["cols"])
        s.res = normal(c["rows"], c["cols"]) if c["residual"] else None
    return s


# ---- the plain forms ---------------------------------------------------------------------

def _signed(v):
    v %= 1 << 64
    return v - (1 << 64) if v >= 1 << 63 else v


def _key(seed):
    """The key of the dropout's stream: value 3 of the SplitMix64 stream of the seed."""
    M = (1 << 64) - 1
    z = (seed + 4 * 0x9E3779B97F4A7C15) & M
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & M
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & M
    return z ^ (z >> 31)


def _kept(seed, first_row, rows, cols, p, dev):
    """Which values of rows x cols stay: value q of the stream decides the columns 2 j (its lower
    half) and 2 j + 1 (its upper) of a row, q = row * ceil(cols / 2) + j; a value stays where its
    half is no less than p * 2^32.  Arithmetic modulo 2^64."""
    half = (cols + 1) // 2
    q = torch.arange(rows * half, device=dev, dtype=torch.int64)
    z = (q + _signed(first_row * half + 1)) * _signed(0x9E3779B97F4A7C15) + _signed(_key(seed))
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(0x94D049BB133111EB)
    z = z ^ ((z >> 31) & ((1 << 33) - 1))
    u = torch.stack((z & 0xFFFFFFFF, (z >> 32) & 0xFFFFFFFF), -1).view(rows, 2 * half)[:, :cols]
    return u >= min(int(p * (1 << 32) + 0.5), (1 << 32) - 1)


def _dropped(v, c, seed):
    """v (..., cols) with the mask and the scale of the dropout."""
    if c["p"] == 0:
        return v
    keep = _kept(seed, c["first_row"], v.numel() // v.shape[-1], v.shape[-1], c["p"], v.device).view(v.shape)
    return torch.where(keep, v * (1 / (1 - c["p"])), 0.0)


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    return torch.ones_like(z)


def _plain_linear(s):
    c, dt = s.case, TYPES[s.case["dtype"]]
    x, w = s.x.float(), s.w.float()
    if c["back"]:
        dz = _dropped(s.dy.float(), c, s.seed)
        if c["act"] != "none":
            dz = dz * _act_slope(s.z.float(), c["act"])
        return {"dx": (dz @ w).to(dt), "dw": (dz.transpose(1, 2) @ x).to(dt), "db": dz.sum(1).to(dt)}
    z = x @ w.transpose(1, 2)
    if s.b is not None:
        z = z + s.b.float()[:, None, :]
    y = _dropped(_act(z, c["act"]), c, s.seed)
    if s.res is not None:
        y = y + s.res.float()
    out = {"y": y.to(dt)}
    if c["pre"]:
        out["pre"] = z.to(dt)
    return out


def _plain_norm(s):
    c, dt = s.case, TYPES[s.case["dtype"]]
    n, b, P, C = s.x.shape
    grouped = (n, b, P, c["groups"], c["width"])
    x = s.x.float().view(grouped)
    gamma, beta = (v.float().view(n, 1, 1, *grouped[3:]) for v in (s.gamma, s.beta))
    if c["back"]:
        xh = (x - s.mean[:, :, None, :, None]) * s.rstd[:, :, None, :, None]
        dt_ = s.dy.float().view(grouped)
        if c["act"] != "none":
            dt_ = dt_ * _act_slope(xh * gamma + beta, c["act"])
        dgamma, dbeta = (dt_ * xh).sum((1, 2)).view(n, C), dt_.sum((1, 2)).view(n, C)
        dt_ = dt_ * gamma
        M = P * c["width"]
        s1 = dt_.sum((2, 4), keepdim=True) / M
        s2 = (dt_ * xh).sum((2, 4), keepdim=True) / M
        dx = (dt_ - s1 - xh * s2) * s.rstd[:, :, None, :, None]
        return {"dx": dx.view(n, b, P, C).to(dt), "dgamma": dgamma.to(dt), "dbeta": dbeta.to(dt)}
    mean = x.mean((2, 4), keepdim=True)
    x = x - mean
    rstd = (x.square().mean((2, 4), keepdim=True) + EPS).rsqrt()
    y = _act(x * rstd * gamma + beta, c["act"])
    return {"y": y.view(n, b, P, C).to(dt), "mean": mean.view(n, b, -1), "rstd": rstd.view(n, b, -1)}


def _plain_dropout(s):
    y = _dropped(s.x.float(), s.case, s.seed)
    if s.res is not None:
        y = y + s.res.float()
    return {"y": y.to(s.x.dtype)}


# ---- one pass ----------------------------------------------------------------------------

def run(state):
    """One call of the operator; all its outputs."""
    s, c = state, state.case
    if not own:
        return {"linear": _plain_linear, "norm": _plain_norm, "dropout": _plain_dropout}[c["op"]](s)
    from paper_2112_13935_amd import ops
    if c["op"] == "linear":
        more = dict(act=c["act"], p=c["p"], seed=s.seed, first_row=c["first_row"])
        if c["back"]:
            dx, dw, db = ops.aet_linear_backward(s.dy, s.x, s.w, s.z, **more)
            return {"dx": dx, "dw": dw, "db": db}
        y, pre = ops.aet_linear_forward(s.x, s.w, s.b, residual=s.res, keep_pre=c["pre"], **more)
        return {"y": y, "pre": pre} if c["pre"] else {"y": y}
    if c["op"] == "norm":
        if c["back"]:
            dx, dgamma, dbeta = ops.aet_group_norm_backward(s.dy, s.x, s.mean, s.rstd, s.gamma, s.beta, act=c["act"])
            return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
        y, mean, rstd = ops.aet_group_norm_forward(s.x, c["groups"], s.gamma, s.beta, eps=EPS, act=c["act"])
        return {"y": y, "mean": mean, "rstd": rstd}
    if c["back"]:
        return {"y": ops.aet_dropout_backward(s.x, p=c["p"], seed=s.seed, first_row=c["first_row"])}
    return {"y": ops.aet_dropout_forward(s.x, p=c["p"], seed=s.seed, first_row=c["first_row"], residual=s.res)}


# ---- the definitions in 64 bits ----------------------------------------------------------

def _factor64(seed, first_row, rows, cols, p, dev):
    """1 / (1 - p) where a value of rows x cols stays, 0 where it goes, by numpy's 64-bit integers."""
    if p == 0:
        return torch.ones(1, 1, dtype=torch.float64, device=dev)
    half = (cols + 1) // 2

    def stream(key, q):
        z = np.uint64(key) + (q + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15)
        for shift, by in ((30, 0xBF58476D1CE4E5B9), (27, 0x94D049BB133111EB)):
            z ^= z >> np.uint64(shift)
            z *= np.uint64(by)
        z ^= z >> np.uint64(31)
        return z

    key = stream(seed, np.array([3], dtype=np.uint64))[0]
    h = stream(key, np.uint64(first_row * half) + np.arange(rows * half, dtype=np.uint64))
    u = h.astype("<u8").view("<u4").reshape(rows, 2 * half)[:, :cols]
    least = min(int(p * 2.0 ** 32 + 0.5), 2 ** 32 - 1)
    return torch.from_numpy(u >= np.uint32(least)).to(dev).double().div_(1 - p)


def _value64(t, act):
    if act == "none":
        return t
    if act == "relu":
        return t.clamp(min=0)
    if act == "silu":
        return t * torch.special.expit(t)
    return t * torch.special.ndtr(t)


def _slope64(t, act):
    if act == "relu":
        return t.sign().clamp(min=0)
    if act == "silu":
        s = torch.special.expit(t)
        return s + t * s * torch.special.expit(-t)
    return torch.special.ndtr(t) + t * torch.exp(-t ** 2 / 2) / math.sqrt(2 * math.pi)


def exact(case, seed):
    """The outputs from the operators' definitions in 64 bits: client by client for the products, sample by sample for
    the normalisation."""
    s = prepare(case, seed)
    c = s.case
    dev = s.x.device
    if c["op"] == "dropout":
        y = s.x.double() * _factor64(s.seed, c["first_row"], c["rows"], c["cols"], c["p"], dev)
        return {"y": y if s.res is None else y.add_(s.res.double())}
    if c["op"] == "linear":
        n, R, O = c["n"], c["rows"], c["out"]
        found = {}
        for k in range(n):
            f = _factor64(s.seed, c["first_row"] + k * R, R, O, c["p"], dev)
            x, w = s.x[k].double(), s.w[k].double()
            if c["back"]:
                dz = s.dy[k].double() * f
                if c["act"] != "none":
                    dz *= _slope64(s.z[k].double(), c["act"])
                one = {"dx": torch.mm(dz, w), "dw": torch.mm(dz.t(), x), "db": dz.sum(0)}
            else:
                z = torch.mm(x, w.t())
                if s.b is not None:
                    z += s.b[k].double()
                y = _value64(z, c["act"]) * f
                if s.res is not None:
                    y = y + s.res[k].double()
                one = {"y": y, "pre": z} if c["pre"] else {"y": y}
            for name, v in one.items():
                found.setdefault(name, []).append(v)
        return {name: torch.stack(v) for name, v in found.items()}
    n, b, P, C = s.x.shape
    G, width = c["groups"], c["width"]
    found = {"dx": [], "dgamma": [], "dbeta": []} if c["back"] else {"y": [], "mean": [], "rstd": []}
    for k in range(n):
        x = s.x[k].double().view(b, P, G, width)
        gamma, beta = s.gamma[k].double().view(G, width), s.beta[k].double().view(G, width)
        if c["back"]:   # with the statistics as they were handed over
            mean, rstd = s.mean[k].double().view(b, 1, G, 1), s.rstd[k].double().view(b, 1, G, 1)
        else:
            var, mean = torch.var_mean(x, (1, 3), correction=0, keepdim=True)
            rstd = 1 / torch.sqrt(var + EPS)
        xh = (x - mean) * rstd
        if not c["back"]:
            found["y"].append(_value64(xh * gamma + beta, c["act"]).view(b, P, C))
            found["mean"].append(mean.view(b, G))
            found["rstd"].append(rstd.view(b, G))
            continue
        d = s.dy[k].double().view(b, P, G, width)
        if c["act"] != "none":
            d = d * _slope64(xh * gamma + beta, c["act"])
        found["dgamma"].append((d * xh).sum((0, 1)).view(C))
        found["dbeta"].append(d.sum((0, 1)).view(C))
        d = d * gamma
        d = d - d.mean((1, 3), keepdim=True) - xh * (d * xh).mean((1, 3), keepdim=True)
        found["dx"].append((d * rstd).view(b, P, C))
    return {name: torch.stack(v) for name, v in found.items()}


# ---- more cases --------------------------------------------------------------------------

def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case between the listed ones: any operator, direction and type, sizes over their
    logarithm, odd ones among them; cut to the listed cases' cost."""
    op = rng.choice(["linear", "linear", "linear", "norm", "norm", "dropout"])
    c = dict(op=op, dtype=rng.choice(["f32", "bf16"]), back=rng.random() < 0.5)
    f32 = c["dtype"] == "f32"
    if op == "linear":
        c.update(n=_log(rng, 1, 64), rows=_log(rng, 1, 16384), inp=_log(rng, 16, 8192), out=_log(rng, 10, 8192),
                 act=rng.choice(["none", "relu", "silu", "gelu"]), p=rng.choice([0.0, 0.0, 0.1, 0.5]))
        if rng.random() < 0.6:    # what most models have: multiples of 64
            c["inp"], c["out"] = (max(64, v // 64 * 64) for v in (c["inp"], c["out"]))
        if rng.random() < 0.2:
            c["pad"] = rng.randint(1, 16)
        if c["p"] and rng.random() < 0.3:
            c["first_row"] = _log(rng, 1, 1 << 34)
        if not c["back"]:
            c.update(bias=rng.random() < 0.8, residual=rng.random() < 0.4, pre=rng.random() < 0.5)
        while work(c)["flops"] > (1.5e11 if f32 else 5e11) or work(c)["bytes"] > 6e8:
            big = max(("n", "rows", "inp", "out"), key=lambda k: c[k])
            c[big] = max(1, c[big] // 2)
    elif op == "norm":
        side = _log(rng, 1, 64)
        c.update(n=_log(rng, 1, 32), batch=_log(rng, 1, 64), hw=side * rng.choice([side, side, max(1, side - 1)]),
                 groups=rng.choice([1, 2, 4, 8, 16, 32, 3, 5]), width=_log(rng, 1, 64),
                 act=rng.choice(["none", "relu", "silu", "gelu"]))
        if c["hw"] * c["width"] < 16:   # so few values normalise to the same whatever they are: nothing is left of a gradient
            c["width"] *= 16
        while work(c)["bytes"] > 6e8:
            big = max(("n", "batch"), key=lambda k: c[k])
            c[big] = max(1, c[big] // 2)
            if c["n"] == c["batch"] == 1:
                break
    else:
        c.update(rows=_log(rng, 1, 16384), cols=_log(rng, 10, 8192), p=rng.choice([0.05, 0.1, 0.5]),
                 first_row=rng.choice([0, _log(rng, 1, 1 << 34)]))
        if not c["back"]:
            c["residual"] = rng.random() < 0.5
        while work(c)["bytes"] > 4e8:
            c["rows"] = max(1, c["rows"] // 2)
    return c
