"""The sequence operators together, as a language model under gossip rounds: one step's gradients against 64-bit automatic
differentiation of the same network, and a short run."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _norm(h, gain, bias):
    c = h - h.mean(-1, keepdim=True)
    return c * torch.rsqrt(c.square().mean(-1, keepdim=True) + 1e-5) * gain[:, None] + bias[:, None]


def _reference(net, batch, tau, alpha):
    """Losses, and gradients of the mean loss per worker, in 64 bits, from the 16-bit weights the step uses."""
    words, ids, teacher, labels = batch
    b, t = words.shape
    s, i, m = net.sequences, net.inner, net.states
    length = t // s
    params = {key: net._param(*key).double().clone().requires_grad_(True) for key in net.names}
    h = net.codes[words].double()
    for k in range(net.blocks):
        p = {name: params[k, name] for _, name in net.names if (k, name) in params}
        xz = _norm(h, p["gain"], p["bias"]) @ p["W_in"].transpose(1, 2)
        x, z = xz[..., :i], xz[..., i:]
        line = torch.nn.functional.pad(x.reshape(b, s, length, i), (0, 0, 3, 0))
        u = sum(line[:, :, j:j + length] * p["conv"][:, None, None, :, j] for j in range(4)) + p["conv_bias"][:, None, None]
        u = torch.nn.functional.silu(u)
        q = u.reshape(b, t, i) @ p["W_p"].transpose(1, 2)
        step = torch.nn.functional.softplus(q[..., :i] + p["delta_bias"][:, None]).reshape(b, s, length, i)
        bb, cc = q[..., i:i + m].reshape(b, s, length, m), q[..., i + m:].reshape(b, s, length, m)
        state, rows = torch.zeros(b, s, i, m, dtype=torch.float64, device="cuda"), []
        for k_ in range(length):
            state = torch.exp(step[:, :, k_, :, None] * p["a"][:, None]) * state + (step * u)[:, :, k_, :, None] * bb[:, :, k_, None, :]
            rows.append((state * cc[:, :, k_, None, :]).sum(-1))
        y = torch.stack(rows, 2) + p["skip"][:, None, None] * u
        h = h + (y.reshape(b, t, i) * torch.nn.functional.silu(z)) @ p["W_out"].transpose(1, 2)
    p = {name: params[net.blocks, name] for name in ("W_head", "gain", "bias")}
    logits = _norm(h, p["gain"], p["bias"]) @ p["W_head"].transpose(1, 2)
    want = torch.softmax(teacher.double() / tau, -1)
    logq = torch.log_softmax(logits / tau, -1).gather(-1, ids.long())
    ce = -torch.log_softmax(logits, -1).gather(-1, labels.long()[..., None])[..., 0]
    loss = alpha * tau ** 2 * (want * (want.log() - logq)).sum(-1) + (1 - alpha) * ce
    (loss.sum() / t).backward()
    return loss.detach(), {key: v.grad for key, v in params.items()}


def test_a_step_has_the_gradients_of_the_language_model():
    from paper_2008_01425_b200 import sgd_experiment as sgd
    from paper_2008_01425_b200 import training as tr

    net = sgd.LanguageNet(n_workers=4, words=301, width=72, inner=100, states=16, blocks=2, sequences=3, seed=3)
    batch = sgd.sentences(net, sgd.chain(301, net.device), 37, seed=5)
    words, ids, teacher, labels = batch
    loss, want = _reference(net, batch, 2.0, 0.5)
    logits, kept = net.forward(words)
    out = tr.pg_distillation_loss(logits, ids, teacher, labels, 2.0, 0.5, dloss=torch.full(words.shape, 1.0 / words.shape[1], device="cuda"), out=logits)
    net.backward(out.dlogits, kept)
    # activations in 8 bits are within a step, 2^-6 of their block's largest value, and everything in 16 bits within 2^-8 of itself;
    # their errors are independent, and a few dozen roundings lie between input and gradient
    assert float((out.loss.double() - loss).norm() / loss.norm()) <= 2.0 ** -6
    for key in net.names:
        got = net._grad(*key).double()
        assert float((got - want[key]).norm() / want[key].norm()) <= 2.0 ** -4, key
    net.net.close()


def test_the_language_model_runs():
    from paper_2008_01425_b200 import sgd_experiment as sgd

    curve = sgd.run_language(6, 2, n_workers=6, length=20, words=200)
    assert [c[0] for c in curve] == [0, 2, 4, 6] and all(math.isfinite(v) for c in curve for v in c)
    assert curve[-1][2] < 0.05                         # the workers see different data and stay together
