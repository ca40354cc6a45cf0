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

With ``--model language`` the workers train a small language model instead, on sequences of words that a fixed Markov chain draws:
blocks of
    n = layer_norm(h);  (x, z) = W_in n;  u = silu(conv(x));  (delta, b, c) = W_p u;  h <- h + W_out scan(u, delta, a, b, c, z)
and a layer norm and W_head above them, whose logits are fitted to the chain's own likeliest next words (the teacher's list) and to
the word that came (the label).

    python -m paper_2008_01425_b200.sgd_experiment [--model residual|language] [--steps 200] [--every 20]
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
        for layer in range(len(self.net.layer_shapes)):
            p = self.net.params_layer(layer).double()
            total += float((p - p.mean(0, keepdim=True)).square().sum())
            size += float(p.square().sum())
        return total / size


BLOCK = ("W_in", "conv", "conv_bias", "W_p", "a", "skip", "delta_bias", "W_out", "gain", "bias")
HEAD = ("W_head", "gain", "bias")


class LanguageNet:
    """`blocks` scan blocks of width `width` (`inner` channels, `states` states) and a head over `words` for `n_workers` workers on a ring."""

    def __init__(self, n_workers: int = 8, words: int = 500, width: int = 64, inner: int = 128, states: int = 16, blocks: int = 2, sequences: int = 4,
                 seed: int = 0, device: str = "cuda:0", dtype=torch.bfloat16):
        self.blocks, self.inner, self.states, self.sequences, self.dtype = blocks, inner, states, sequences, dtype
        of = {"W_in": (2 * inner, width), "conv": (inner, 4), "conv_bias": (1, inner), "W_p": (inner + 2 * states, inner), "a": (inner, states),
              "skip": (1, inner), "delta_bias": (1, inner), "W_out": (width, inner), "gain": (1, width), "bias": (1, width), "W_head": (words, width)}
        self.names = [(k, name) for k in range(blocks) for name in BLOCK] + [(blocks, name) for name in HEAD]
        self.layer = {key: i for i, key in enumerate(self.names)}
        self.net = pg.PowerGossip(kind=pg.PG_RING, n_workers=n_workers, layer_shapes=[of[name] for _, name in self.names], rank=1, power_steps=1, seed=seed,
                                  weight_rule=pg.PG_W_UNIFORM, device=device)
        self.device = self.net.device
        g = torch.Generator().manual_seed(seed)
        for i, (_, name) in enumerate(self.names):          # identical start on all workers
            rows, cols = of[name]
            if name == "a":
                w = -torch.arange(1, states + 1).float().repeat(inner, 1)
            elif name in ("skip", "gain"):
                w = torch.ones(rows, cols)
            elif name == "delta_bias":
                w = torch.full((rows, cols), -2.0)
            else:
                w = torch.zeros(rows, cols) if name.endswith("bias") else torch.randn(rows, cols, generator=g) * cols ** -0.5
            for worker in range(n_workers):
                self.net.pg_write_params(worker, i, w)
        self.codes = torch.randn(words, width, generator=g).to(self.device, dtype)      # what a word is read as: fixed
        self.grads = self.net.gradient_buffer()

    def _param(self, k: int, name: str):
        """A parameter of all workers: weights of products in 16 bits, everything else as a view of the stack."""
        v = self.net.params_layer(self.layer[k, name])
        return v.to(self.dtype) if name.startswith("W") else v if name in ("conv", "a") else v[:, 0]

    def _grad(self, k: int, name: str):
        v = self.net.gradient_layer(self.grads, self.layer[k, name])
        return v if name.startswith("W") or name in ("conv", "a") else v[:, 0]

    def forward(self, words):
        """words: (workers, tokens) -> (logits, what the backward pass needs)."""
        kept, h, i, m = [], self.codes[words], self.inner, self.states
        r = None
        for k in range(self.blocks):
            p = {name: self._param(k, name) for name in BLOCK}
            n = tr.pg_add_layer_norm(h, p["gain"], p["bias"], residual=r, eight_bit=True)           # h + r of the block before
            xz = tr.pg_linear(n.y, p["W_in"])
            x, z = xz[..., :i], xz[..., i:]
            u = tr.pg_causal_conv(x, p["conv"], p["conv_bias"], sequences=self.sequences)
            q = tr.pg_linear(u, p["W_p"])
            delta, b, c = q[..., :i], q[..., i:i + m], q[..., i + m:]
            y = tr.pg_selective_scan(u, delta, p["a"], b, c, p["skip"], p["delta_bias"], z, sequences=self.sequences)
            r = tr.pg_linear(y, p["W_out"])
            kept.append((n, x, z, u, delta, b, c, y, p))
            h = n.h
        p = {name: self._param(self.blocks, name) for name in HEAD}
        n = tr.pg_add_layer_norm(h, p["gain"], p["bias"], residual=r, eight_bit=True)
        kept.append((n, p))
        return tr.pg_linear(n.y, p["W_head"]), kept

    def backward(self, dlogits, kept) -> None:
        """Fills self.grads with the gradients of all workers."""
        n, p = kept[-1]
        d = {name: self._grad(self.blocks, name) for name in HEAD}
        tr.pg_linear_weight_grad(dlogits, n.y8, out=d["W_head"])
        g, _, _ = tr.pg_add_layer_norm_grad(tr.pg_linear_input_grad(dlogits, p["W_head"]), n.h, n.mean, n.rstd, p["gain"], gain_grad=d["gain"], bias_grad=d["bias"])
        for k in reversed(range(self.blocks)):
            n, x, z, u, delta, b, c, y, p = kept[k]
            d = {name: self._grad(k, name) for name in BLOCK}
            tr.pg_linear_weight_grad(g, y, out=d["W_out"])
            s = tr.pg_selective_scan_grad(tr.pg_linear_input_grad(g, p["W_out"]), u, delta, p["a"], b, c, p["skip"], p["delta_bias"], z, sequences=self.sequences,
                                          a_grad=d["a"], skip_grad=d["skip"], delta_bias_grad=d["delta_bias"])
            dq = torch.cat([s.ddelta, s.db, s.dc], -1)
            tr.pg_linear_weight_grad(dq, u, out=d["W_p"])
            du = tr.pg_linear_input_grad(dq, p["W_p"], residual=s.du)
            dx, _, _ = tr.pg_causal_conv_grad(du, x, p["conv"], p["conv_bias"], sequences=self.sequences, weight_grad=d["conv"], bias_grad=d["conv_bias"])
            dxz = torch.cat([dx, s.dz], -1)
            tr.pg_linear_weight_grad(dxz, n.y8, out=d["W_in"])
            g, _, _ = tr.pg_add_layer_norm_grad(tr.pg_linear_input_grad(dxz, p["W_in"]), n.h, n.mean, n.rstd, p["gain"], dh=g, gain_grad=d["gain"], bias_grad=d["bias"])

    def step(self, batch, eta: float, temperature: float = 2.0, alpha: float = 0.5):
        """One step of Algorithm 1 on every worker; returns the workers' mean losses before it."""
        words, ids, teacher, labels = batch
        logits, kept = self.forward(words)
        scale = torch.full(words.shape, 1.0 / words.shape[1], device=self.device)
        out = tr.pg_distillation_loss(logits, ids, teacher, labels, temperature, alpha, dloss=scale, out=logits)
        self.backward(out.dlogits, kept)
        self.net.pg_round_sgd(self.grads, eta, stream=torch.cuda.current_stream(self.device))
        return out.loss.mean(1)

    spread = ResidualNet.spread


def chain(words: int, device, top: int = 8, seed: int = 12345):
    """The Markov chain: log-probabilities of the next word (words x words), and their best `top` as (ids, logits)."""
    g = torch.Generator().manual_seed(seed)
    logp = torch.log_softmax(3.0 * torch.randn(words, words, generator=g), -1).to(device)
    best = torch.topk(logp, min(top, words), -1)
    return logp, best.indices.to(torch.int32), best.values


def sentences(net: LanguageNet, source, length: int, seed: int):
    """(words, ids, teacher, labels) of every worker: net.sequences sequences of `length` words of its own."""
    logp, ids, values = source
    g = torch.Generator(device=net.device).manual_seed(seed)
    rows = net.net.n_workers * net.sequences
    word = torch.randint(len(logp), (rows,), device=net.device, generator=g)
    line = [word]
    for _ in range(length):
        noise = -torch.log(-torch.log(torch.rand(rows, len(logp), device=net.device, generator=g).clamp(1e-7, 1 - 1e-7)))
        line.append((logp[line[-1]] + noise).argmax(-1))
    line = torch.stack(line, 1).reshape(net.net.n_workers, net.sequences, length + 1)
    words, labels = line[..., :-1].flatten(1), line[..., 1:].flatten(1)
    return words, ids[words], values[words].to(net.dtype), labels.to(torch.int32).contiguous()


def run_language(steps: int, every: int, eta: float = 0.3, n_workers: int = 8, length: int = 35, device: str = "cuda:0", **sizes):
    """[(step, mean loss over workers, parameter spread)]."""
    net = LanguageNet(n_workers=n_workers, device=device, **sizes)
    source = chain(len(net.codes), net.device)
    curve = []
    for k in range(steps + 1):
        loss = net.step(sentences(net, source, length, seed=k), eta=eta)
        if k % every == 0 or k == steps:
            curve.append((k, float(loss.mean()), net.spread()))
    assert tr.pg_training_status(device=net.device) == 0 and net.net.pg_device_status() == 0
    net.net.close()
    return curve


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
    ap.add_argument("--model", choices=("residual", "language"), default="residual")
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--every", type=int, default=20)
    args = ap.parse_args()
    print("decentralized SGD, 8 workers on a ring, rank-1 PowerGossip")
    name, curve = ("mean squared error", run) if args.model == "residual" else ("mean loss", run_language)
    for step, err, spread in curve(args.steps, args.every):
        print("  step %5d   %s %.5f   spread of the workers %.2e" % (step, name, err, spread))


if __name__ == "__main__":
    main()
