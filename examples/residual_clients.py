"""Clients that train residual networks in local rounds, with the operators of aet_ops.h.

The scheme is the one of the library's rounds: client c goes on from the server's model for s_i = a i + b
samples of its own, w_c <- w_c - eta g and U <- U + g for each mini-batch, and the server applies every
client's sum, w <- w - eta / n * sum of U.  The model is one that the rounds do not have: images of
C x H x W are cut into 4 x 4 patches (positions with channels last), embedded, go through blocks

    x <- x + dropout(W2 gelu(W1 silu(norm(x)) + b1) + b2)

and their mean over the positions through a linear layer into a softmax.  All clients' models are worked
on side by side, each with weights of its own: one call an operator for all of them.  The parameters of a
client are one row of a matrix, the operators read and write them in place by their strides.

    python examples/residual_clients.py [--clients 8] [--rounds 6] [--bf16]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import workloads as W  # noqa: E402
from paper_2112_13935_amd import ops  # noqa: E402

PATCH, CLASSES = 4, 10


class ResidualClients:
    """n clients' models: w, their parameters [n, P], and the gradient of their mini-batches, g [n, P]."""

    def __init__(self, n, channels=3, hw=32, width=64, hidden=256, blocks=2, groups=8, p=0.1, seed=1,
                 dtype=torch.float32, device="cuda:0"):
        self.n, self.blocks, self.groups, self.p, self.seed = n, blocks, groups, p, seed
        self.dtype, self.device = dtype, torch.device(device)
        self.positions, self.patch = (hw // PATCH) ** 2, channels * PATCH * PATCH
        shapes = {"embed": (width, self.patch), "embed_b": (width,)}
        for k in range(blocks):
            shapes.update({f"gamma{k}": (width,), f"beta{k}": (width,), f"w1{k}": (hidden, width), f"b1{k}": (hidden,),
                           f"w2{k}": (width, hidden), f"b2{k}": (width,)})
        shapes.update({"head": (CLASSES, width), "head_b": (CLASSES,)})
        self.places, at = {}, 0
        for name, shape in shapes.items():
            self.places[name] = (at, shape)
            at += -(-math.prod(shape) // 64) * 64      # every parameter begins on a line of memory
        self.w = torch.zeros(n, at, dtype=dtype, device=self.device)
        self.g = torch.zeros_like(self.w)
        gen = torch.Generator(device=self.device).manual_seed(seed)
        for name, (_, shape) in self.places.items():   # every client the same
            view = self.view(self.w, name)
            if len(shape) == 2:
                view.copy_(torch.randn(shape, generator=gen, device=self.device) / math.sqrt(shape[1]))
            elif name.startswith("gamma"):
                view.fill_(1.0)
        self.step = 0

    def view(self, flat, name):
        at, shape = self.places[name]
        return flat[:, at:at + math.prod(shape)].view(self.n, *shape)

    def patches(self, X):
        """[n, batch, C, H, W] to [n, batch, positions, channels of a patch]."""
        n, b, c, h, w = X.shape
        X = X.view(n, b, c, h // PATCH, PATCH, w // PATCH, PATCH).permute(0, 1, 3, 5, 2, 4, 6)
        return X.reshape(n, b, self.positions, self.patch).to(self.dtype)

    def forward(self, X, train=True):
        """The logits [n, batch, classes], and what the gradient needs."""
        n, b = X.shape[:2]
        rows, kept = b * self.positions, []
        p = self.p if train else 0.0
        v = lambda name: self.view(self.w, name)   # noqa: E731
        seed = [self.seed + (self.blocks + 1) * self.step + k for k in range(self.blocks + 1)]   # a mask of its own for each
        x0 = self.patches(X).view(n, rows, self.patch)
        e, _ = ops.aet_linear_forward(x0, v("embed"), v("embed_b"))
        x = ops.aet_dropout_forward(e, p=p, seed=seed[-1])
        for k in range(self.blocks):
            maps = x.view(n, b, self.positions, -1)
            h, mean, rstd = ops.aet_group_norm_forward(maps, self.groups, v(f"gamma{k}"), v(f"beta{k}"), act="silu")
            h = h.view(n, rows, -1)
            u, pre = ops.aet_linear_forward(h, v(f"w1{k}"), v(f"b1{k}"), act="gelu", keep_pre=True)
            kept.append((maps, mean, rstd, h, u, pre))
            x, _ = ops.aet_linear_forward(u, v(f"w2{k}"), v(f"b2{k}"), residual=x, p=p, seed=seed[k])
        pooled = x.view(n, b, self.positions, -1).float().mean(2).to(self.dtype)
        logits, _ = ops.aet_linear_forward(pooled, v("head"), v("head_b"))
        return logits, (x0, kept, pooled, p, seed)

    def backward(self, dlogits, saved):
        """The gradient of the parameters, in g."""
        x0, kept, pooled, p, seed = saved
        n, b = dlogits.shape[:2]
        v, g = lambda name: self.view(self.w, name), lambda name: self.view(self.g, name)   # noqa: E731
        dpool, _, _ = ops.aet_linear_backward(dlogits, pooled, v("head"), out=(None, g("head"), g("head_b")))
        dx = (dpool / self.positions)[:, :, None].expand(-1, -1, self.positions, -1).reshape(n, b * self.positions, -1)
        for k in reversed(range(self.blocks)):
            maps, mean, rstd, h, u, pre = kept[k]
            du, _, _ = ops.aet_linear_backward(dx, u, v(f"w2{k}"), p=p, seed=seed[k], out=(None, g(f"w2{k}"), g(f"b2{k}")))
            dh, _, _ = ops.aet_linear_backward(du, h, v(f"w1{k}"), pre, act="gelu", out=(None, g(f"w1{k}"), g(f"b1{k}")))
            dm, _, _ = ops.aet_group_norm_backward(dh.view_as(maps), maps, mean, rstd, v(f"gamma{k}"), v(f"beta{k}"), act="silu",
                                                   out=(None, g(f"gamma{k}"), g(f"beta{k}")))
            dx = dx + dm.view_as(dx)
        de = ops.aet_dropout_backward(dx, p=p, seed=seed[-1])
        ops.aet_linear_backward(de, x0, v("embed"), need=(False, True, True), out=(None, g("embed"), g("embed_b")))

    def loss_and_gradient(self, X, y):
        """The mini-batches' mean cross-entropy by client; its gradient in g."""
        logits, saved = self.forward(X)
        logp = torch.log_softmax(logits.float(), -1)
        hot = torch.nn.functional.one_hot(y.long(), CLASSES)
        self.backward(((logp.exp() - hot) / y.shape[1]).to(self.dtype).contiguous(), saved)
        self.step += 1
        return -(logp * hot).sum(-1).mean(1)


def train(clients=8, rows=400, a=64, b=128, batch=32, rounds=6, eta=0.05, dtype=torch.float32, seed=5, say=print):
    """The rounds; the mean loss of each."""
    wl = W.config4(n_clients=clients, n_per=rows, batch=batch)
    dev = torch.device("cuda:0")
    X = torch.stack([torch.from_numpy(x) for x in wl.X]).to(dev).view(clients, rows, 3, 32, 32)
    y = torch.stack([torch.from_numpy(v) for v in wl.y]).to(dev)
    net = ResidualClients(clients, seed=seed, dtype=dtype)
    gen = torch.Generator(device=dev).manual_seed(seed)
    server, who, losses = net.w[0].float(), torch.arange(clients, device=dev)[:, None], []
    for i in range(rounds):
        local = server.expand(clients, -1).clone()     # the clients' models are kept in fp32
        U, total, steps = torch.zeros_like(local), 0.0, (a * i + b) // batch
        for _ in range(steps):
            net.w.copy_(local)
            q = torch.randint(rows, (clients, batch), generator=gen, device=dev)
            total = total + net.loss_and_gradient(X[who, q], y[who, q])
            g = net.g.float()
            local -= eta * g
            U += g
        server = server - eta / clients * U.sum(0)
        losses.append(float(total.mean()) / steps)
        say(f"round {i}: {steps} mini-batches a client, mean loss {losses[-1]:.4f}")
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--clients", type=int, default=8)
    ap.add_argument("--rounds", type=int, default=6)
    ap.add_argument("--bf16", action="store_true")
    args = ap.parse_args()
    train(clients=args.clients, rounds=args.rounds, dtype=torch.bfloat16 if args.bf16 else torch.float32)
