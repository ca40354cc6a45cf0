"""Decentralized SGD (Algorithm 1) with its local half on the GPU too.

Every worker of a ring trains the same small residual network on data of its own: blocks of
    n = rms_norm(h) * gain;   h <- h + W2 gelu(W1 n + b1) + b2
fitted to a teacher network's output.  One step is
    forward and backward pass of all workers at once (training.py), the activations that the
    backward pass needs kept in 8 bits, the gradients written straight into a buffer laid out like
    the parameter stack;
    one gossip round with that gradient (pg_round_sgd).
Biases and gains are read where they are in the stack (1 x n matrices, which rank-1 gossip averages
exactly); the weights are copied to bf16 before every step.

    python -m paper_2008_01425_b200.sgd_experiment [--steps 200] [--every 20]
"""
from __future__ import annotations

import argparse
from typing import List, Tuple

import torch

from . import binding as pg
from . import training as tr

NAMES = ("W1", "b1", "W2", "b2", "gain")


class ResidualNet:
    """`blocks` residual blocks of width `width` for `n_workers` workers on a ring."""

    def __init__(self, n_workers: int = 8, width: int = 128, hidden: int = 512, blocks: int = 2, seed: int = 0,
                 device: str = "cuda:0", dtype=torch.bfloat16):
        self.blocks, self.dtype = blocks, dtype
        shapes: List[Tuple[int, int]] = []
        for _ in range(blocks):
            shapes += [(hidden, width), (1, hidden), (width, hidden), (1, width), (1, width)]
        self.net = pg.PowerGossip(kind=pg.PG_RING, n_workers=n_workers, layer_shapes=shapes, rank=1, power_steps=1, seed=seed,
                                  weight_rule=pg.PG_W_UNIFORM, device=device)
        self.device = self.net.device
        g = torch.Generator().manual_seed(seed)
        for layer, (rows, cols) in enumerate(shapes):       # identical start on all workers, as in Algorithm 1
            name = NAMES[layer % 5]
            w = torch.ones(rows, cols) if name == "gain" else torch.zeros(rows, cols) if name[0] == "b" else \
                torch.randn(rows, cols, generator=g) * (0.3 if name == "W2" else 1.0) * cols ** -0.5
            for worker in range(n_workers):
                self.net.pg_write_params(worker, layer, w)
        self.grads = self.net.gradient_buffer()

    def _params(self, block: int):
        """(W1, b1, W2, b2, gain) of all workers: weights in 16 bits, vectors as views of the stack."""
        w1, b1, w2, b2, gain = (self.net.params_layer(5 * block + i) for i in range(5))
        return w1.to(self.dtype), b1[:, 0], w2.to(self.dtype), b2[:, 0], gain[:, 0]

    def forward(self, x):
        """x (workers, tokens, width) -> (output, what the backward pass needs)."""
        kept, h, r = [], x, None
        for k in range(self.blocks):
            w1, b1, w2, b2, gain = self._params(k)
            n = tr.pg_add_rms_norm(h, gain, residual=r, eight_bit=True)            # h + r of the block before
            u, z8 = tr.pg_linear(n.y, w1, b1, activation="gelu", save_z=True)
            r = tr.pg_linear(u, w2, b2, residual=n.h if k == self.blocks - 1 else None)
            kept.append((n.h, n.rstd, n.y8, z8, tr.pg_checkpoint_write(u), w1, w2, gain))
            h = n.h
        return r, kept

    def backward(self, dout, kept) -> None:
        """Fills self.grads with the gradients of all workers."""
        g = dout
        for k in reversed(range(self.blocks)):
            h, rstd, y8, z8, u8, w1, w2, gain = kept[k]
            d1, db1, d2, db2, dgain = (self.net.gradient_layer(self.grads, 5 * k + i) for i in range(5))
            tr.pg_activation_grad(g, None, "none", out=torch.empty_like(g), bias_grad=db2[:, 0])
            tr.pg_linear_weight_grad(g, u8, out=d2)
            du = tr.pg_linear_input_grad(g, w2)
            dz, _ = tr.pg_activation_grad(du, z8, "gelu", out=du, bias_grad=db1[:, 0])
            tr.pg_linear_weight_grad(dz, y8, out=d1)
            dn = tr.pg_linear_input_grad(dz, w1)
            g, _ = tr.pg_add_rms_norm_grad(dn, h, rstd, gain, dh=g, gain_grad=dgain[:, 0])

    def step(self, x, target, eta: float):
        """One step of Algorithm 1 on every worker; returns the workers' mean squared errors before it."""
        out, kept = self.forward(x)
        diff = out.float() - target.float()
        self.backward((diff / (x.shape[1] * x.shape[2])).to(self.dtype), kept)
        self.net.pg_round_sgd(self.grads, eta, stream=torch.cuda.current_stream(self.device))
        return diff.square().mean((1, 2))

    def spread(self) -> float:
        """Squared distance of the workers' parameters from their mean, relative to the parameters'."""
        total, size = 0.0, 0.0
        for layer in range(5 * self.blocks):
            p = self.net.params_layer(layer).double()
            total += float((p - p.mean(0, keepdim=True)).square().sum())
            size += float(p.square().sum())
        return total / size


def data(net: ResidualNet, tokens: int, width: int, seed: int):
    """Inputs of every worker and what the teacher makes of them: a fixed residual map of its own."""
    g = torch.Generator(device=net.device).manual_seed(seed)
    t = torch.Generator(device=net.device).manual_seed(12345)
    a = torch.randn(width, width, device=net.device, generator=t) * width ** -0.5
    x = torch.randn(net.net.n_workers, tokens, width, device=net.device, generator=g)
    return x.to(net.dtype), (x + torch.tanh(x @ a)).to(net.dtype)


def run(steps: int, every: int, eta: float = 0.5, n_workers: int = 8, width: int = 128, tokens: int = 256, device: str = "cuda:0"):
    """[(step, mean error over workers, parameter spread)]."""
    net = ResidualNet(n_workers=n_workers, width=width, device=device)
    curve = []
    for k in range(steps + 1):
        err = net.step(*data(net, tokens, width, seed=k), eta=eta)
        if k % every == 0 or k == steps:
            curve.append((k, float(err.mean()), net.spread()))
    assert tr.pg_training_status(device=net.device) == 0 and net.net.pg_device_status() == 0
    net.net.close()
    return curve


def main() -> None:
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--every", type=int, default=20)
    args = ap.parse_args()
    print("decentralized SGD, 8 workers on a ring, rank-1 PowerGossip")
    for step, err, spread in run(args.steps, args.every):
        print("  step %5d   mean squared error %.5f   spread of the workers %.2e" % (step, err, spread))


if __name__ == "__main__":
    main()
