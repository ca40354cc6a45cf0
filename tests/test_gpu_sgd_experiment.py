"""The training operators and the gossip round together: one step's gradients against 64-bit
automatic differentiation of the same network, and a short run that learns."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _reference(net, x, target):
    """Gradients of 0.5 sum diff^2 / (tokens width) per worker, in 64 bits, from the 16-bit weights the step uses."""
    params = []
    for k in range(net.blocks):
        w1, b1, w2, b2, gain = net._params(k)
        params.append([v.double().clone().requires_grad_(True) for v in (w1, b1, w2, b2, gain)])
    h = x.double()
    for w1, b1, w2, b2, gain in params:
        n = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-5) * gain[:, None]
        u = torch.nn.functional.gelu(n @ w1.transpose(1, 2) + b1[:, None], approximate="tanh")
        h = h + u @ w2.transpose(1, 2) + b2[:, None]
    (0.5 * (h - target.double()).square().sum() / (x.shape[1] * x.shape[2])).backward()
    return [[v.grad for v in p] for p in params]


def test_a_step_has_the_gradients_of_the_network():
    from paper_2008_01425_b200 import sgd_experiment as sgd

    net = sgd.ResidualNet(n_workers=4, width=96, hidden=200, blocks=2, seed=3)
    x, target = sgd.data(net, 150, 96, seed=5)
    want = _reference(net, x, target)
    out, kept = net.forward(x)
    net.backward(((out.float() - target.float()) / (150 * 96)).to(net.dtype), kept)
    for k in range(net.blocks):
        for i, w in enumerate(want[k]):
            got = net.net.gradient_layer(net.grads, 5 * k + i).double().reshape(w.shape)
            # activations in 8 bits are within a step, 2^-6 of their block's largest value, and everything in 16 bits within
            # 2^-8 of itself; their errors are independent, and a dozen roundings lie between input and gradient
            assert float((got - w).norm() / w.norm()) <= 2.0 ** -5, (k, sgd.NAMES[i])
    net.net.close()


def test_the_ring_learns():
    from paper_2008_01425_b200 import sgd_experiment as sgd

    curve = sgd.run(60, 20, width=64, tokens=128, n_workers=6)
    errors = [c[1] for c in curve]
    assert all(b < a for a, b in zip(errors, errors[1:])) and errors[-1] < 0.5 * errors[0]
    assert curve[-1][2] < 0.05                     # the workers see different data and stay together


def test_the_step_stays_on_the_current_stream(monkeypatch):
    """Inside another current stream everything of a step, the view of the parameters included, is enqueued there."""
    from paper_2008_01425_b200 import binding as pg
    from paper_2008_01425_b200 import sgd_experiment as sgd

    nets = [sgd.ResidualNet(n_workers=4, width=64, hidden=96, blocks=1, seed=3) for _ in range(2)]
    batches = [sgd.data(nets[0], 40, 64, seed=k) for k in range(3)]
    for x, target in batches:
        nets[0].step(x, target, eta=0.5)
    s, seen = torch.cuda.Stream(), []
    inner = pg.PowerGossip.pg_params_device
    monkeypatch.setattr(pg.PowerGossip, "pg_params_device",
                        lambda self, worker, layer, stream=None: seen.append(stream) or inner(self, worker, layer, stream))
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)                      # a step that left the stream would overtake the others
        for x, target in batches:
            nets[1].step(x, target, eta=0.5)
    assert seen and all(getattr(v, "cuda_stream", v) == s.cuda_stream for v in seen)
    torch.cuda.synchronize()
    for layer in range(len(nets[0].net.layer_shapes)):
        assert torch.equal(nets[0].net.params_layer(layer), nets[1].net.params_layer(layer))
    for n in nets:
        n.net.close()
