"""The sequence operators (include/pg_training.h: layer norm, causal convolution, selective scan, distillation loss) against their formulas
in 64 bits.

Tolerances.  u = 2^-24 is half a step of fp32 at and above 1; results in 16 bits are within half a step of the type besides (check()).
A sum of n numbers in fp32, in any order, is within n u of the sum of their sizes; exp, logarithm, reciprocal and root are good to 8 u of
their result and to what their argument's own error makes of it.  Where errors feed on one another (states along a sequence) the bound is
carried along with the 64-bit computation, step by step.
"""
import math

import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_training import BF, HF, U, check, check8, eight, gen, make8, rand, strided  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2008_01425_b200 import build as pg_build

    pg_build.build()


@pytest.fixture(scope="module")
def tr():
    from paper_2008_01425_b200 import training

    yield training
    assert training.pg_training_status() == 0


def sig(v):
    return torch.sigmoid(v)


# ---------------------------------------------------------------- layer norm
def norm_reference(x, r, gain, bias, eps):
    """(sum, mean, root, y) and how far mean and y may be off."""
    s = x.double() + (0.0 if r is None else r.double())
    n = s.shape[-1]
    mean = s.mean(-1, keepdim=True)
    d = s - mean
    var = d.square().mean(-1, keepdim=True)
    root = (var + float(torch.tensor(eps, dtype=torch.float32))) ** -0.5
    y = d * root * gain.double()[:, None] + bias.double()[:, None]
    off = (n + 4) * U * s.abs().mean(-1, keepdim=True)                     # of the mean
    rel = (n + 32) * U + off.square() * root.square()                     # of the root: sum of squares, and the mean's error squared
    slack = gain.double().abs()[:, None] * root * (off + 4 * U * s.abs()) + (y - bias.double()[:, None]).abs() * rel + 4 * U * y.abs()
    return s, mean, root, y, off, rel, slack


@pytest.mark.parametrize("shape,pad", [((1, 1, 1), 0), ((2, 3, 7), 1), ((3, 5, 64), 0), ((2, 9, 147), 1), ((2, 70, 650), 0), ((1, 33, 1024), 8),
                                       ((2, 5, 1029), 3), ((1, 3, 4612), 0), ((1, 2, 9000), 1), ((2, 2, 16384), 0)])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("residual,with8", [(False, False), (True, False), (True, True)])
def test_layer_norm(tr, shape, pad, dtype, residual, with8):
    b, t, n = shape
    g = gen(n + t)
    x = strided((rand(g, *shape) + 3.0).to(dtype), pad)
    r = strided(rand(g, *shape).to(dtype), pad) if residual else None
    gain, bias = rand(g, b, n), rand(g, b, n)
    out = tr.pg_add_layer_norm(x, gain, bias, residual=r, eps=1e-5, eight_bit=with8, save_h8=with8)
    s, mean, root, y, off, rel, slack = norm_reference(x, r, gain, bias, 1e-5)
    check(out.mean, mean[..., 0], off[..., 0])
    check(out.rstd, root[..., 0], (root * rel)[..., 0])
    if residual:
        check(out.h, s, U * s.abs(), dtype)
    else:
        assert out.h is x
    if with8:
        check8(out.y8, y, slack, dtype)
        assert torch.equal(out.y, tr.pg_checkpoint_read(out.y8))
        held = tr.pg_checkpoint_write(out.h)
        assert torch.equal(held.values, out.h8.values) and torch.equal(held.scales, out.h8.scales)
    else:
        check(out.y, y, slack, dtype)


def norm_grad_reference(dy, h, mean, rstd, gain, dh):
    dy, h, r, k = dy.double(), h.double(), rstd.double()[..., None], gain.double()[:, None]
    n, t = h.shape[-1], h.shape[-2]
    unit = (h - mean.double()[..., None]) * r
    a = dy * k
    m1, m2 = a.mean(-1, keepdim=True), (a * unit).mean(-1, keepdim=True)
    dx = r * (a - m1 - unit * m2) + (0.0 if dh is None else dh.double())
    eu = 4 * U * ((h.abs() + mean.double()[..., None].abs()) * r)          # of the unit
    m1_off, m2_off = (n + 4) * U * a.abs().mean(-1, keepdim=True), ((n + 6) * U * (a * unit).abs() + a.abs() * eu).mean(-1, keepdim=True)
    slack = r * (m1_off + unit.abs() * m2_off + eu * m2.abs() + 8 * U * (a.abs() + m1.abs() + (unit * m2).abs())) + 4 * U * dx.abs()
    if dh is not None:
        slack = slack + 4 * U * dh.double().abs()
    dgain, dgain_slack = (dy * unit).sum(1), ((t + 6) * U * (dy * unit).abs() + dy.abs() * eu).sum(1)
    return dx, slack, dgain, dgain_slack, dy.sum(1), (t + 2) * U * dy.abs().sum(1)


@pytest.mark.parametrize("shape,pad", [((1, 1, 1), 0), ((2, 3, 7), 1), ((3, 50, 64), 0), ((2, 90, 147), 1), ((2, 70, 650), 0), ((2, 300, 256), 8),
                                       ((2, 5, 1029), 3), ((1, 30, 4612), 0), ((1, 5, 9000), 1), ((1, 3, 16384), 0)])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dh,from8", [(False, False), (True, False), (True, True)])
def test_layer_norm_gradient(tr, shape, pad, dtype, dh, from8):
    b, t, n = shape
    g = gen(n * 3 + t)
    h = (rand(g, *shape) + 0.5).to(dtype)
    held = make8(tr, h, dtype) if from8 else strided(h, pad)
    if from8:
        h = eight(h, dtype)[2].to(dtype)
    dy, more = strided(rand(g, *shape).to(dtype), pad), strided(rand(g, *shape).to(dtype), pad) if dh else None
    mean = h.float().mean(-1)
    rstd = (h.float().var(-1, correction=0) + 1e-5).rsqrt()
    gain = rand(g, b, n)
    into, into_b = rand(g, b, n), rand(g, b, n)
    before, before_b = into.double(), into_b.double()
    dx, dgain, dbias = tr.pg_add_layer_norm_grad(dy, held, mean, rstd, gain, dh=more, gain_grad=into, bias_grad=into_b, accumulate=True)
    want, slack, wg, sg, wb, sb = norm_grad_reference(dy, h, mean, rstd, gain, more)
    check(dx, want, slack, dtype)
    check(dgain, before + wg, sg + 4 * U * (before.abs() + wg.abs()))
    check(dbias, before_b + wb, sb + 4 * U * (before_b.abs() + wb.abs()))
    again = tr.pg_add_layer_norm_grad(dy, held, mean, rstd, gain, dh=more)
    check(again[1], wg, sg)
    check(again[2], wb, sb)


@pytest.mark.parametrize("scale", [1e36, 1e25, 1e-18, 1e-30])
def test_layer_norm_of_rows_whose_squares_leave_fp32(tr, scale):
    g = gen(3)
    x = (rand(g, 2, 4, 700).double().clamp(-2, 2) * scale).to(BF)
    out = tr.pg_add_layer_norm(x, eps=0.0)
    one = torch.ones(2, 700, device="cuda")
    _, mean, root, y, off, rel, slack = norm_reference(x, None, one, one * 0, 0.0)
    check(out.y, y, slack, BF)
    check(out.mean, mean[..., 0], off[..., 0] + 2.0 ** -149)
    check(out.rstd, root[..., 0], (root * rel)[..., 0] + 2.0 ** -149)


def test_layer_norm_keeps_what_is_not_finite_in_its_row(tr):
    x = rand(gen(4), 2, 6, 300).to(HF)
    x[0, 1, 7], x[1, 2, 299] = float("nan"), float("inf")
    y = tr.pg_add_layer_norm(x).y
    bad = torch.isnan(y).any(-1)
    assert bad.nonzero().tolist() == [[0, 1], [1, 2]] and torch.isnan(y[0, 1]).all() and torch.isnan(y[1, 2]).all()


# ---------------------------------------------------------------- convolution
def there(lengths, length, seqs, b):
    """(workers, sequences, length, 1), the tokens that are there."""
    if lengths is None:
        return torch.ones(b, seqs, length, 1, dtype=torch.bool, device="cuda")
    return (torch.arange(length, device="cuda") < lengths[..., None]).unsqueeze(-1)


def conv_reference(x, weight, bias, seqs, lengths, state, act):
    b, t, n = x.shape
    length, taps = t // seqs, weight.shape[-1]
    is_there = there(lengths, length, seqs, b)
    xs = torch.where(is_there, x.double().reshape(b, seqs, length, n), torch.zeros((), dtype=torch.float64, device="cuda"))
    first = torch.zeros(b, seqs, taps - 1, n, dtype=torch.float64, device="cuda") if state is None else state.double()
    line = torch.cat([first, xs], 2)
    z = sum(line[:, :, j:j + length] * weight.double()[:, None, None, :, j] for j in range(taps)) + bias.double()[:, None, None]
    size = sum((line[:, :, j:j + length] * weight.double()[:, None, None, :, j]).abs() for j in range(taps)) + bias.double().abs()[:, None, None]
    off = (taps + 2) * U * size
    y = z * sig(z) if act == "silu" else z
    return line, z, off, y, 1.1 * off + 32 * U * y.abs(), is_there


CONV = [((1, 1, 1, 1), 2, 0), ((2, 3, 5, 7), 3, 1), ((2, 1, 70, 64), 4, 0), ((3, 4, 9, 65), 4, 1), ((1, 2, 200, 130), 2, 8), ((8, 4, 1, 300), 4, 0), ((1, 1, 1030, 33), 3, 3),
        ((2, 2, 2, 96), 4, 0)]


@pytest.mark.parametrize("shape,taps,pad", CONV)
@pytest.mark.parametrize("dtype,act,carried,ragged", [(BF, "silu", True, True), (HF, "silu", False, True), (BF, "none", True, False), (HF, "none", False, False)])
def test_causal_conv(tr, shape, taps, pad, dtype, act, carried, ragged):
    b, s, length, n = shape
    g = gen(n + length)
    x = strided(rand(g, b, s * length, n).to(dtype), pad)
    weight, bias = rand(g, b, n, taps), rand(g, b, n)
    state = rand(g, b, s, taps - 1, n).to(dtype) if carried else None
    lengths = torch.randint(0, length + 1, (b, s), device="cuda", generator=g).to(torch.int32) if ragged else None
    line, z, _, y, slack, is_there = conv_reference(x, weight, bias, s, lengths, state, act)
    got, last = tr.pg_causal_conv(x, weight, bias, activation=act, sequences=s, lengths=lengths, state=state, state_out=True)
    zero = torch.zeros_like(y)
    check(got, torch.where(is_there, y, zero).reshape(b, -1, n), torch.where(is_there, slack, zero).reshape(b, -1, n), dtype)
    ends = is_there.sum(2)[..., 0]
    want = torch.stack([torch.stack([line[i, k, ends[i, k]:ends[i, k] + taps - 1] for k in range(s)]) for i in range(b)])
    assert torch.equal(last.double(), want)
    if carried:                                        # and with the state in place
        again, same = tr.pg_causal_conv(x, weight, bias, activation=act, sequences=s, lengths=lengths, state=state, state_out=state)
        assert same is state and torch.equal(again, got) and torch.equal(state, last)


def conv_grad_reference(dy, x, weight, bias, seqs, lengths, state, act):
    b, t, n = x.shape
    length, taps = t // seqs, weight.shape[-1]
    line, z, off, _, _, is_there = conv_reference(x, weight, bias, seqs, lengths, state, act)
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    gy = torch.where(is_there, dy.double().reshape(b, seqs, length, n), zero)
    p = sig(z)
    dz = gy * (p * (1 + z * (1 - p))) if act == "silu" else gy
    ez = gy.abs() * (0.6 * off + 40 * U * (1 + z.abs() * p * (1 - p))) if act == "silu" else gy * 0
    w = weight.double()
    dline, eline = torch.zeros_like(line), torch.zeros_like(line)
    dw, ew = torch.empty_like(w), torch.empty_like(w)
    for j in range(taps):
        wj = w[:, None, None, :, j]
        dline[:, :, j:j + length] += dz * wj
        eline[:, :, j:j + length] += wj.abs() * ez + (taps + 2) * U * (dz * wj).abs()
        xj = line[:, :, j:j + length]
        dw[..., j] = (dz * xj).sum((1, 2))
        ew[..., j] = (ez * xj.abs() + (t + 4) * U * (dz * xj).abs()).sum((1, 2))
    dx = torch.where(is_there, dline[:, :, taps - 1:], zero).reshape(b, t, n)
    return dx, eline[:, :, taps - 1:].reshape(b, t, n), dw, ew, dz.sum((1, 2)), (ez + (t + 4) * U * dz.abs()).sum((1, 2))


@pytest.mark.parametrize("shape,taps,pad", CONV)
@pytest.mark.parametrize("dtype,act,carried,ragged", [(BF, "silu", True, True), (HF, "silu", False, False), (BF, "none", False, True)])
def test_causal_conv_gradient(tr, shape, taps, pad, dtype, act, carried, ragged):
    b, s, length, n = shape
    g = gen(n * 5 + length)
    x, dy = strided(rand(g, b, s * length, n).to(dtype), pad), strided(rand(g, b, s * length, n).to(dtype), pad)
    weight, bias = rand(g, b, n, taps), rand(g, b, n)
    state = rand(g, b, s, taps - 1, n).to(dtype) if carried else None
    lengths = torch.randint(0, length + 1, (b, s), device="cuda", generator=g).to(torch.int32) if ragged else None
    dx, ex, dw, ew, db, eb = conv_grad_reference(dy, x, weight, bias, s, lengths, state, act)
    got = tr.pg_causal_conv_grad(dy, x, weight, bias, activation=act, sequences=s, lengths=lengths, state=state)
    check(got[0], dx, ex, dtype)
    check(got[1], dw, ew)
    check(got[2], db, eb)
    wg, bg = rand(g, b, n, taps), rand(g, b, n)
    more = tr.pg_causal_conv_grad(dy, x, weight, bias, activation=act, sequences=s, lengths=lengths, state=state, weight_grad=wg.clone(), bias_grad=bg.clone(),
                                  accumulate=True)
    check(more[1], wg.double() + dw, ew + 4 * U * (wg.double().abs() + dw.abs()))
    check(more[2], bg.double() + db, eb + 4 * U * (bg.double().abs() + db.abs()))


# ---------------------------------------------------------------- scan
def scan_inputs(g, b, s, length, n, m, dtype, gate, carried, ragged, pad):
    t = s * length
    c = {"u": strided(rand(g, b, t, n).to(dtype), pad), "delta": strided(rand(g, b, t, n, scale=1.5).to(dtype), pad),
         "a": -torch.exp(rand(g, b, n, m, scale=0.7)), "b": strided(rand(g, b, t, m).to(dtype), pad), "c": strided(rand(g, b, t, m).to(dtype), pad),
         "skip": rand(g, b, n), "delta_bias": rand(g, b, n) - 2.0, "z": strided(rand(g, b, t, n).to(dtype), pad) if gate else None}
    more = {"sequences": s, "lengths": torch.randint(0, length + 1, (b, s), device="cuda", generator=g).to(torch.int32) if ragged else None,
            "state": rand(g, b, s, n, m) if carried else None}
    return c, more


def scan_forward(c, more, chunk):
    """64-bit states of all tokens with their bounds.  chunk: the longest sum of steps the states' decay may be computed from."""
    b, t, n = c["u"].shape
    s = more["sequences"]
    length, m = t // s, c["a"].shape[-1]
    wide = lambda v, k: v.double().reshape(b, s, length, k)
    u, bb, cc = wide(c["u"], n), wide(c["b"], m), wide(c["c"], m)
    raw = wide(c["delta"], n) + c["delta_bias"].double()[:, None, None]
    is_there = there(more["lengths"], length, s, b)
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    raw, u, bb, cc = (torch.where(is_there, v, zero) for v in (raw, u, bb, cc))
    step = torch.where(is_there, torch.nn.functional.softplus(raw, threshold=700.0), zero)
    e_step = step * 24 * U + U * raw.abs() * sig(raw)
    a = c["a"].double()[:, None]
    h = [torch.zeros(b, s, n, m, dtype=torch.float64, device="cuda") if more["state"] is None else more["state"].double()]
    e = [torch.zeros_like(h[0])]
    keeps, e_keeps = [], []
    for k in range(length):
        keep = torch.exp(step[:, :, k, :, None] * a)
        e_keep = keep * ((16 + chunk) * U * (step[:, :, k, :, None] * a).abs() + e_step[:, :, k, :, None] * a.abs() + 8 * U * (step[:, :, k, :, None] > 0))
        drive = (step * u)[:, :, k, :, None] * bb[:, :, k, None, :]
        e_drive = drive.abs() * 4 * U + (e_step * u.abs())[:, :, k, :, None] * bb[:, :, k, None, :].abs()
        e.append(keep * e[-1] + e_keep * (h[-1].abs() + e[-1]) + e_drive + 2 * U * (keep * h[-1]).abs())
        h.append(keep * h[-1] + drive)
        keeps.append(keep)
        e_keeps.append(e_keep)
    return {"u": u, "b": bb, "c": cc, "raw": raw, "step": step, "e_step": e_step, "h": h, "e": e, "keep": keeps, "e_keep": e_keeps, "there": is_there}


def scan_output(c, more, f):
    b, t, n = c["u"].shape
    length, m = len(f["keep"]), c["a"].shape[-1]
    inner = torch.stack([(f["h"][k + 1] * f["c"][:, :, k, None, :]).sum(-1) for k in range(length)], 2)
    off = torch.stack([(f["e"][k + 1] * f["c"][:, :, k, None, :].abs() + (m + 4) * U * (f["h"][k + 1] * f["c"][:, :, k, None, :]).abs()).sum(-1) for k in range(length)], 2)
    direct = c["skip"].double()[:, None, None] * f["u"]
    y, off = inner + direct, off + 2 * U * direct.abs()
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    if c["z"] is not None:
        z = c["z"].double().reshape(b, -1, length, n)
        gate = z * sig(z)
        y, off = y * gate, off * gate.abs() + 32 * U * (y * gate).abs()
    y, off = torch.where(f["there"], y, zero), torch.where(f["there"], off + 2 * U * y.abs(), zero)
    return inner, y.reshape(b, t, n), off.reshape(b, t, n)


SCAN = [((1, 1, 1, 1), 1, 0), ((2, 3, 5, 7), 16, 1), ((2, 1, 70, 64), 16, 0), ((1, 4, 17, 129), 8, 1), ((2, 2, 33, 40), 33, 8), ((8, 4, 1, 300), 16, 0), ((1, 1, 700, 33), 16, 3),
        ((1, 2, 300, 20), 64, 0), ((2, 1, 41, 130), 3, 1), ((1, 1, 2100, 5), 4, 0), ((1, 3, 16, 260), 17, 1)]


@pytest.mark.parametrize("shape,states,pad", SCAN)
@pytest.mark.parametrize("dtype,gate,carried,ragged", [(BF, True, True, True), (HF, False, False, False), (BF, False, True, False), (HF, True, False, True)])
def test_selective_scan(tr, shape, states, pad, dtype, gate, carried, ragged):
    b, s, length, n = shape
    c, more = scan_inputs(gen(n + length), b, s, length, n, states, dtype, gate, carried, ragged, pad)
    f = scan_forward(c, more, length)
    _, y, slack = scan_output(c, more, f)
    got, last = tr.pg_selective_scan(**c, **more, state_out=True)
    check(got, y, slack, dtype)
    check(last, f["h"][-1], f["e"][-1] + 2 * U * f["h"][-1].abs())
    if carried:                                        # and with the state in place
        held = more["state"].clone()
        again, same = tr.pg_selective_scan(**c, **{**more, "state": held}, state_out=held)
        assert same is held and torch.equal(again, got) and torch.equal(held, last)


def scan_grad_reference(c, more, dy, chunk):
    b, t, n = c["u"].shape
    s, m = more["sequences"], c["a"].shape[-1]
    length = t // s
    f = scan_forward(c, more, chunk)
    inner, _, _ = scan_output(c, more, f)
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    gy = torch.where(f["there"], dy.double().reshape(b, s, length, n), zero)
    skip, a, u, step, e_step = c["skip"].double()[:, None, None], c["a"].double()[:, None], f["u"], f["step"], f["e_step"]
    out, off = {}, {}
    e_inner = torch.stack([(f["e"][k + 1] * f["c"][:, :, k, None, :].abs() + (m + 4) * U * (f["h"][k + 1] * f["c"][:, :, k, None, :]).abs()).sum(-1) for k in range(length)], 2)
    dv, e_dv = gy, gy * 0
    if c["z"] is not None:
        z = torch.where(f["there"], c["z"].double().reshape(b, s, length, n), zero)
        p = sig(z)
        slope = p * (1 + z * (1 - p))
        full = inner + skip * u
        out["dz"] = gy * full * slope
        off["dz"] = gy.abs() * (slope.abs() * (e_inner + 4 * U * (inner.abs() + (skip * u).abs())) + 48 * U * full.abs() * (p + (z * p * (1 - p)).abs()))
        dv = gy * z * p
        e_dv = 32 * U * dv.abs()
    g = torch.zeros(b, s, n, m, dtype=torch.float64, device="cuda")          # what reaches h_t from behind it
    eg = torch.zeros_like(g)
    names = ("du", "ddelta", "db", "dc")
    for name, like in zip(names, (u, u, f["b"], f["c"])):
        out[name], off[name] = torch.zeros_like(like), torch.zeros_like(like)
    da, e_da = torch.zeros(b, n, m, dtype=torch.float64, device="cuda"), torch.zeros(b, n, m, dtype=torch.float64, device="cuda")
    chains = t + 4                                     # numbers in the longest sum over tokens
    for k in reversed(range(length)):
        bk, ck, h0, h1, keep = f["b"][:, :, k, None, :], f["c"][:, :, k, None, :], f["h"][k], f["h"][k + 1], f["keep"][k]
        e0, e1, e_keep = f["e"][k], f["e"][k + 1], f["e_keep"][k]
        v, ev = dv[:, :, k, :, None], e_dv[:, :, k, :, None]
        drive, e_drive = (step * u)[:, :, k, :, None], (e_step * u.abs() + 2 * U * (step * u).abs())[:, :, k, :, None]
        eg = eg + ev * ck.abs() + 2 * U * ((v * ck).abs() + g.abs())
        g = g + v * ck
        out["dc"][:, :, k], off["dc"][:, :, k] = (v * h1).sum(2), (ev * h1.abs() + v.abs() * e1 + (n + 4) * U * (v * h1).abs()).sum(2)
        out["db"][:, :, k], off["db"][:, :, k] = (g * drive).sum(2), (eg * drive.abs() + g.abs() * e_drive + (n + 4) * U * (g * drive).abs()).sum(2)
        to_drive, e_to = (g * bk).sum(-1), (eg * bk.abs() + (m + 4) * U * (g * bk).abs()).sum(-1)
        eg, g = eg * keep + e_keep * (g.abs() + eg) + 2 * U * (g * keep).abs(), g * keep
        d = g * h0
        ed = eg * h0.abs() + (g.abs() + eg) * e0 + 2 * U * d.abs()
        sk, esk, uk = step[:, :, k], e_step[:, :, k], u[:, :, k]
        out["du"][:, :, k] = to_drive * sk + skip[:, :, 0] * dv[:, :, k]
        off["du"][:, :, k] = e_to * sk + to_drive.abs() * esk + skip[:, :, 0].abs() * e_dv[:, :, k] + 4 * U * ((to_drive * sk).abs() + (skip[:, :, 0] * dv[:, :, k]).abs())
        slope = sig(f["raw"][:, :, k])
        to_step, e_step_sum = (d * a).sum(-1), (ed * a.abs() + (m + 8) * U * (d * a).abs()).sum(-1)
        total = to_drive * uk + to_step
        out["ddelta"][:, :, k] = total * slope
        off["ddelta"][:, :, k] = slope * (e_to * uk.abs() + e_step_sum + 64 * U * ((to_drive * uk).abs() + to_step.abs())) + total.abs() * esk
        da += (d * sk[..., None]).sum(1)
        e_da += (ed * sk[..., None] + d.abs() * esk[..., None] + chains * U * (d * sk[..., None]).abs()).sum(1)
    for name in names[:2] + (("dz",) if "dz" in out else ()):
        out[name], off[name] = (torch.where(f["there"], v, zero) for v in (out[name], off[name]))
    out["ddelta_bias"], off["ddelta_bias"] = out["ddelta"].sum((1, 2)), (off["ddelta"] + chains * U * out["ddelta"].abs()).sum((1, 2))
    out["dskip"], off["dskip"] = (dv * u).sum((1, 2)), (e_dv * u.abs() + chains * U * (dv * u).abs()).sum((1, 2))
    for name in names + (("dz",) if "dz" in out else ()):
        out[name], off[name] = out[name].reshape(b, t, -1), off[name].reshape(b, t, -1)
    out["da"], off["da"] = da, e_da
    return out, off


@pytest.mark.parametrize("shape,states,pad", SCAN)
@pytest.mark.parametrize("dtype,gate,carried,ragged", [(BF, True, True, True), (HF, False, False, False), (HF, True, False, True)])
def test_selective_scan_gradient(tr, shape, states, pad, dtype, gate, carried, ragged):
    b, s, length, n = shape
    g = gen(n * 7 + length)
    c, more = scan_inputs(g, b, s, length, n, states, dtype, gate, carried, ragged, pad)
    dy = strided(rand(g, b, s * length, n).to(dtype), pad)
    want, off = scan_grad_reference(c, more, dy, 64)
    into = [rand(g, b, n, states), rand(g, b, n), rand(g, b, n)]
    before = dict(zip(("da", "dskip", "ddelta_bias"), (v.double() for v in into)))
    got = tr.pg_selective_scan_grad(dy, **c, **more)
    for name in want:
        check(getattr(got, name), want[name], off[name] + 2 * U * want[name].abs(), None if name in before else dtype)
    more_got = tr.pg_selective_scan_grad(dy, **c, **more, a_grad=into[0], skip_grad=into[1], delta_bias_grad=into[2], accumulate=True)
    for name, old in before.items():
        check(getattr(more_got, name), old + want[name], off[name] + 4 * U * (old.abs() + want[name].abs()))
    assert (got.dz is None) == (not gate)


def test_steps_of_all_sizes(tr):
    """softplus from 1e-9 to 60, where it is tiny and where it is its argument: a state's first step shows it."""
    raw = torch.linspace(-20, 60, 400, device="cuda").reshape(1, 1, 400).to(BF)
    one = torch.ones(1, 1, 400, device="cuda", dtype=BF)
    b = torch.ones(1, 1, 1, device="cuda", dtype=BF)
    a = torch.full((1, 400, 1), -1e-6, device="cuda")
    _, state = tr.pg_selective_scan(one, raw, a, b, b, state_out=True)
    want = torch.nn.functional.softplus(raw.double(), threshold=700.0)[0, 0]
    check(state[0, 0, :, 0], want, 24 * U * want)
    g = tr.pg_selective_scan_grad(one, one, raw, a, b, b)
    slope = sig(raw.double())                          # ddelta = dy u b c sigmoid, and the decay's part, 1e-6 of a state that is zero
    check(g.ddelta[0, 0], slope[0, 0], 40 * U * slope[0, 0], BF)


# ---------------------------------------------------------------- loss
def loss_reference(x, ids, teacher, labels, tau, alpha, dloss):
    """64 bits, with bounds.  An entry's own row: workers x tokens are flattened."""
    x = x.double().flatten(0, -2)
    rows, n = x.shape
    lse1, lse = torch.logsumexp(x, -1), torch.logsumexp(x / tau, -1)
    chain = (n / 512 + 100) * U                        # of a sum of exponentials: no thread adds more than n / 512 + 36 numbers up in a row
    e1, e = chain + 8 * U * lse1.abs(), chain + 8 * U * lse.abs()
    soft, hard = alpha if ids is not None else 0.0, 1 - alpha if labels is not None else 0.0
    loss, off = torch.zeros(rows, dtype=torch.float64, device="cuda"), torch.zeros(rows, dtype=torch.float64, device="cuda")
    dx, slack = torch.zeros_like(x), torch.zeros_like(x)
    q, q1 = torch.exp(x / tau - lse[:, None]), torch.exp(x - lse1[:, None])
    g = None if dloss is None else dloss.double().flatten()[:, None]
    if soft:
        at, v = ids.long().flatten(0, -2), teacher.double().flatten(0, -2) / tau
        good = (at >= 0) & (at < n)
        v = torch.where(good, v, torch.full_like(v, -math.inf))
        at = torch.where(good, at, torch.zeros_like(at))
        some = (v > -math.inf).any(-1) | torch.isnan(v).any(-1)
        top = v.amax(-1, keepdim=True)
        logp = torch.where(some[:, None], v - torch.logsumexp(v, -1, keepdim=True), torch.full_like(v, -math.inf))
        p = torch.exp(logp)
        xt = torch.gather(x, 1, at) / tau
        logq = xt - lse[:, None]
        term = torch.where(p == 0, torch.zeros_like(p), p * (logp - logq))
        e_logp = (v.abs() + top.abs()) * 4 * U + 100 * U
        e_term = torch.where(p == 0, torch.zeros_like(p), p * (e_logp + e[:, None] + 8 * U * xt.abs()) + 300 * U * term.abs() + term.abs() * e_logp)
        loss, off = loss + soft * tau ** 2 * term.sum(-1), off + soft * tau ** 2 * (e_term.sum(-1) + (p.shape[1] + 16) * U * term.abs().sum(-1))
        if g is not None:
            use = torch.where(some, 1.0, 0.0)[:, None]
            d = (q * use).scatter_add(1, at, torch.where(good, -p, torch.zeros_like(p)))
            ed = (q * (e[:, None] + 8 * U * (x / tau).abs() + 64 * U)).nan_to_num(0.0).scatter_add(1, at, torch.where(good & (p != 0), p * (e_logp + 200 * U), torch.zeros_like(p)))
            dx, slack = dx + soft * tau * g * d, slack + soft * tau * g.abs() * ed
    if hard:
        y = labels.long().flatten()
        good = (y >= 0) & (y < n)
        xy = torch.gather(x, 1, torch.where(good, y, torch.zeros_like(y))[:, None])[:, 0]
        one = torch.where(good, lse1 - xy, torch.zeros_like(xy))
        loss, off = loss + hard * one, off + hard * torch.where(good, e1 + 8 * U * (lse1.abs() + xy.abs()), torch.zeros_like(xy))
        if g is not None:
            d = q1.clone()
            d[torch.arange(rows, device="cuda"), torch.where(good, y, torch.zeros_like(y))] -= 1.0
            ed = (q1 * (e1[:, None] + 8 * U * x.abs() + 64 * U)).nan_to_num(0.0)
            use = good[:, None].double()
            dx, slack = dx + hard * g * torch.where(good[:, None], d, torch.zeros_like(d)), slack + hard * g.abs() * (ed + 4 * U) * use
    lses = torch.stack([lse1 if hard else lse1 * 0, lse if soft else lse * 0], -1)
    return loss, off, lses, torch.stack([e1, e], -1), dx, slack + 8 * U * dx.abs()


def loss_inputs(g, b, t, n, k, dtype, labels, pad):
    x = strided(rand(g, b, t, n, scale=3.0).to(dtype), pad)
    ids = teacher = None
    if k:
        ids = torch.stack([torch.randperm(n, device="cuda", generator=g)[:k] for _ in range(b * t)]).reshape(b, t, k).to(torch.int32)
        teacher = rand(g, b, t, k, scale=3.0).to(dtype)
    y = torch.randint(0, n, (b, t), device="cuda", generator=g).to(torch.int32) if labels else None
    return x, ids, teacher, y


def check_loss(tr, x, ids, teacher, labels, tau, alpha, dloss, dtype):
    shape = x.shape
    loss, off, lse, e_lse, dx, slack = loss_reference(x, ids, teacher, labels, tau, alpha, dloss)
    loss, off, lse = loss.float().double(), off + U * loss.abs(), lse.float().double()       # (beyond fp32's range they are infinite)
    e_lse = e_lse + U * lse.abs().nan_to_num(posinf=0.0)
    kw = dict(ids=ids, teacher=teacher, labels=labels, temperature=tau, alpha=alpha)
    only = tr.pg_distillation_loss(x, **kw)
    assert only.dlogits is None
    one = tr.pg_distillation_loss(x, dloss=dloss, **kw)
    for r in (only, one):
        check(r.loss, loss.reshape(shape[:-1]), off.reshape(shape[:-1]))
        check(r.lse, lse.reshape(*shape[:-1], 2), e_lse.reshape(*shape[:-1], 2))
    check(one.dlogits, dx.reshape(shape), slack.reshape(shape), dtype)
    back = tr.pg_distillation_loss_grad(dloss, x, one.lse, **kw)
    held = (lse.abs().amax(-1) < 1e7).reshape(shape[:-1])                 # an lse whose own step is above 1 says nothing about a row's probabilities
    check(back[held], dx.reshape(shape)[held], slack.reshape(shape)[held], dtype)
    return one


@pytest.mark.parametrize("shape,k,pad", [((1, 1, 1), 1, 0), ((2, 3, 7), 3, 1), ((3, 5, 64), 8, 0), ((2, 4, 1000), 16, 8), ((2, 3, 1029), 33, 1), ((1, 9, 4099), 64, 0),
                                         ((2, 5, 28001), 32, 0), ((1, 3, 50000), 1, 8), ((1, 2, 120001), 5, 1), ((1, 700, 3000), 4, 0), ((1, 2, 2000), 1024, 0)])
@pytest.mark.parametrize("dtype,tau", [(BF, 1.0), (HF, 2.0), (BF, 4.0), (HF, 1.7)])
@pytest.mark.parametrize("alpha", [0.0, 0.3, 1.0])
def test_distillation_loss(tr, shape, k, pad, dtype, tau, alpha):
    b, t, n = shape
    g = gen(n + k)
    x, ids, teacher, labels = loss_inputs(g, b, t, n, k, dtype, alpha < 1.0, pad)
    dloss = rand(g, b, t)
    check_loss(tr, x, ids if alpha else None, teacher if alpha else None, labels, tau, alpha, dloss, dtype)


@pytest.mark.parametrize("n,k,pad", [(60, 3, 0), (1029, 5, 1), (4099, 0, 8)])
@pytest.mark.parametrize("dtype,tau", [(BF, 2.0), (HF, 1.7), (BF, 1.0)])
def test_distillation_loss_of_many_rows(tr, n, k, pad, dtype, tau):
    """Rows enough for every warp of the GPU."""
    g = gen(n)
    x = strided(rand(g, 2, 2300, n, scale=3.0).to(dtype), pad)
    ids = torch.randint(-1, n + 1, (2, 2300, k), device="cuda", generator=g).to(torch.int32) if k else None
    teacher = rand(g, 2, 2300, k).to(dtype) if k else None
    labels = torch.randint(-1, n, (2, 2300), device="cuda", generator=g).to(torch.int32)
    check_loss(tr, x, ids, teacher, labels, tau, 0.4 if k else 0.0, rand(g, 2, 2300), dtype)


@pytest.mark.parametrize("n", [50, 3000, 30001, 110000])
@pytest.mark.parametrize("tau", [1.0, 2.0, 0.7])
def test_lists_labels_and_masks_at_their_ends(tr, n, tau):
    g = gen(n)
    x, ids, teacher, labels = loss_inputs(g, 2, 6, n, 8, BF, True, 0)
    ids[0, 0, 3:] = -1                                  # a shorter list
    ids[0, 1] = torch.tensor([-1, n, n + 5, 2 ** 31 - 1, -2 ** 31, -7, n, n], device="cuda")        # an empty one
    ids[0, 2, 4:] = ids[0, 2, :4]                       # every class twice
    ids[0, 3] = ids[0, 3, 0]                            # one class eight times
    teacher[0, 4, 2:5] = -math.inf                      # entries that cannot be
    teacher[0, 5] = -math.inf                           # none that can
    labels[0, :3] = torch.tensor([-100, n, -1], device="cuda")
    labels[1, 0] = ids[1, 0, 0]                         # the label is listed
    labels[1, 1], ids[1, 1, 0], ids[1, 1, 1:] = n - 1, n - 1, torch.arange(7, device="cuda")
    x[1, 2, ::2] = torch.finfo(BF).min                  # masked by the type's lowest value, and by -inf
    x[1, 3, 1::2] = -math.inf
    ids[1, 3] = ids[1, 3] // 2 * 2 % (n // 2 * 2)
    labels[1, 3] = 2
    x[1, 4, :-1] = -math.inf                            # a single class is left
    ids[1, 4] = n - 1
    labels[1, 4] = n - 1
    x[1, 5] = -3e38                                     # all alike, far from zero
    check_loss(tr, x, ids, teacher, labels, tau, 0.4, rand(g, 2, 6), BF)


def test_what_is_not_finite_in_a_row_of_logits(tr):
    g = gen(8)
    x, ids, teacher, labels = loss_inputs(g, 1, 6, 900, 4, HF, True, 0)
    clean = tr.pg_distillation_loss(x, ids, teacher, labels, 2.0, 0.5, dloss=torch.ones(1, 6, device="cuda"))
    y = x.clone()
    y[0, 1, 17], y[0, 3, 400], y[0, 4] = math.nan, math.inf, -math.inf
    t = teacher.clone()
    t[0, 5, 2] = math.nan
    r = tr.pg_distillation_loss(y, ids, t, labels, 2.0, 0.5, dloss=torch.ones(1, 6, device="cuda"))
    assert torch.isnan(r.loss[0]).tolist() == [False, True, False, True, True, True]
    for k in (0, 2):
        assert r.loss[0, k] == clean.loss[0, k] and torch.equal(r.dlogits[0, k], clean.dlogits[0, k])
    assert all(bool(torch.isnan(r.dlogits[0, k]).all()) for k in (1, 3, 4))
    z = x.clone()                                       # a class of the list that the student rules out: the loss is infinite, its slope is not
    z[0, 0, ids[0, 0, 0].item()] = -math.inf
    r = tr.pg_distillation_loss(z, ids, teacher, None, 2.0, 1.0, dloss=torch.ones(1, 6, device="cuda"))
    assert math.isinf(r.loss[0, 0]) and torch.isfinite(r.dlogits[0, 0]).all()


@pytest.mark.parametrize("n", [300, 5000, 28000, 110001])
def test_the_gradient_in_place_of_the_logits(tr, n):
    g = gen(n)
    x, ids, teacher, labels = loss_inputs(g, 3, 40, n, 6, BF, True, 3)
    dloss, kw = rand(g, 3, 40), dict(ids=ids, teacher=teacher, labels=labels, temperature=2.0, alpha=0.5)
    want = tr.pg_distillation_loss(x, dloss=dloss, **kw)
    back = tr.pg_distillation_loss_grad(dloss, x, want.lse, **kw)
    y, z = x.clone(memory_format=torch.preserve_format), strided(x.clone(), 3)
    got = tr.pg_distillation_loss(z, dloss=dloss, out=z, **kw)
    assert got.dlogits is z and torch.equal(z, want.dlogits) and torch.equal(got.loss, want.loss) and torch.equal(got.lse, want.lse)
    z = strided(y, 3)
    assert torch.equal(tr.pg_distillation_loss_grad(dloss, z, want.lse, out=z, **kw), back)


def test_a_loss_of_no_terms(tr):
    x = rand(gen(1), 2, 3, 70).to(BF)
    r = tr.pg_distillation_loss(x, dloss=torch.ones(2, 3, device="cuda"))
    assert not r.loss.any() and not r.lse.any() and not r.dlogits.any()


# ---------------------------------------------------------------- differences
def directional(f, at, d, eps):
    up = [v + eps * w for v, w in zip(at, d)]
    down = [v - eps * w for v, w in zip(at, d)]
    return float((f(*up) - f(*down)) / (2 * eps))


def within(got, d, diff, size):
    """Sum of got * d against a difference quotient: half a step of 16 bits per entry, and `size`, the differences' own error."""
    total = sum(float((a.double() * w).sum()) for a, w in zip(got, d))
    slack = sum(float(((a.double() * w).abs() * (2.0 ** -8 if a.dtype == BF else 2.0 ** -18)).sum()) for a, w in zip(got, d))
    assert abs(total - diff) <= slack + size, (total, diff, slack)


def test_gradients_against_differences(tr):
    g = gen(31)
    wide = lambda *v: [a.double() for a in v]
    direction = lambda *v: [rand(g, *a.shape).double() for a in v]
    # layer norm
    x, gain, bias, dy = rand(g, 2, 5, 40).to(BF), rand(g, 2, 40), rand(g, 2, 40), rand(g, 2, 5, 40).to(BF)
    n = tr.pg_add_layer_norm(x, gain, bias)
    got = tr.pg_add_layer_norm_grad(dy, x, n.mean, n.rstd, gain)

    def norm(x, k, o):
        c = x - x.mean(-1, keepdim=True)
        return ((c / torch.sqrt(c.square().mean(-1, keepdim=True) + 1e-5) * k[:, None] + o[:, None]) * dy.double()).sum()

    at, d = wide(x, gain, bias), direction(x, gain, bias)
    within(got, d, directional(norm, at, d, 1e-5), 1e-4)
    # convolution
    x, w, o, dy = rand(g, 2, 12, 9).to(BF), rand(g, 2, 9, 4), rand(g, 2, 9), rand(g, 2, 12, 9).to(BF)
    got = tr.pg_causal_conv_grad(dy, x, w, o, sequences=3)

    def conv(x, w, o):
        line = torch.nn.functional.pad(x.reshape(2, 3, 4, 9), (0, 0, 3, 0))
        z = sum(line[:, :, j:j + 4] * w[:, None, None, :, j] for j in range(4)) + o[:, None, None]
        return (z * sig(z) * dy.double().reshape(2, 3, 4, 9)).sum()

    at, d = wide(x, w, o), direction(x, w, o)
    within(got, d, directional(conv, at, d, 1e-5), 1e-4)
    # scan
    c, more = scan_inputs(g, 2, 2, 7, 6, 5, BF, True, True, False, 0)
    dy = rand(g, 2, 14, 6).to(BF)
    r = tr.pg_selective_scan_grad(dy, **c, **more)
    names = ("u", "delta", "a", "b", "c", "skip", "delta_bias", "z")

    def scan(*v):
        q = dict(zip(names, v))
        step = torch.nn.functional.softplus(q["delta"] + q["delta_bias"][:, None]).reshape(2, 2, 7, 6)
        sp = lambda t: t.reshape(2, 2, 7, -1)
        h, rows = more["state"].double(), []
        for k in range(7):
            h = torch.exp(step[:, :, k, :, None] * q["a"][:, None]) * h + (step * sp(q["u"]))[:, :, k, :, None] * sp(q["b"])[:, :, k, None, :]
            rows.append((h * sp(q["c"])[:, :, k, None, :]).sum(-1))
        y = torch.stack(rows, 2) + q["skip"][:, None, None] * sp(q["u"])
        return (y * sp(q["z"]) * sig(sp(q["z"])) * dy.double().reshape(2, 2, 7, 6)).sum()

    at = wide(*(c[k] for k in names))
    got = [getattr(r, "d" + k) for k in names]
    for i in range(len(names)):                        # one input at a time
        d = [torch.zeros_like(v) for v in at]
        d[i] = rand(g, *at[i].shape).double()
        within(got, d, directional(scan, at, d, 1e-5), 1e-4)
    # loss
    x, ids, teacher, labels = loss_inputs(g, 2, 3, 50, 6, BF, True, 0)
    dloss = rand(g, 2, 3)
    got = tr.pg_distillation_loss(x, ids, teacher, labels, 1.7, 0.4, dloss=dloss).dlogits

    def loss(x):
        p = torch.softmax(teacher.double() / 1.7, -1)
        logq = torch.log_softmax(x / 1.7, -1).gather(-1, ids.long())
        ce = -torch.log_softmax(x, -1).gather(-1, labels.long()[..., None])[..., 0]
        return ((0.4 * 1.7 ** 2 * (p * (p.log() - logq)).sum(-1) + 0.6 * ce) * dloss.double()).sum()

    at, d = wide(x), direction(x)
    within([got], d, directional(loss, at, d, 1e-5), 1e-4)


# ---------------------------------------------------------------- the calls
def everything(tr, g, b=3, s=2, length=37, n=70, dtype=BF, stream=None):
    """One call of each operator; all outputs."""
    t = s * length
    x, r, dy = (rand(g, b, t, n).to(dtype) for _ in range(3))
    gain, bias = rand(g, b, n), rand(g, b, n)
    w, state = rand(g, b, n, 4), rand(g, b, s, 3, n).to(dtype)
    lengths = torch.randint(0, length + 1, (b, s), device="cuda", generator=g).to(torch.int32)
    c, more = scan_inputs(g, b, s, length, n, 16, dtype, True, True, True, 1)
    logits, ids, teacher, labels = loss_inputs(g, b, t, 900, 5, dtype, True, 1)
    dloss = rand(g, b, t)

    def run():
        k = dict(stream=stream)
        m = tr.pg_add_layer_norm(x, gain, bias, residual=r, eight_bit=True, save_h8=True, **k)
        out = [m.h, m.y, m.mean, m.rstd, m.y8.values, m.h8.scales, *tr.pg_add_layer_norm_grad(dy, m.h, m.mean, m.rstd, gain, **k)]
        out += tr.pg_causal_conv(x, w, bias, sequences=s, lengths=lengths, state=state, state_out=True, **k)
        out += tr.pg_causal_conv_grad(dy, x, w, bias, sequences=s, lengths=lengths, state=state, **k)
        out += tr.pg_selective_scan(**c, **more, state_out=True, **k)
        out += tr.pg_selective_scan_grad(dy, **c, **more, **k)
        kw = dict(ids=ids, teacher=teacher, labels=labels, temperature=2.0, alpha=0.5)
        q = tr.pg_distillation_loss(logits, dloss=dloss, **kw, **k)
        return out + [*q, tr.pg_distillation_loss_grad(dloss, logits, q.lse, **kw, **k)]

    return run


def test_sequence_results_repeat_bit_for_bit(tr):
    run = everything(tr, gen(1))
    first = run()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, run()))


def test_another_stream_and_two_at_once(tr):
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    runs = [everything(tr, gen(2), stream=k) for k in (None, s, t)]
    want = runs[0]()
    torch.cuda.synchronize()
    got = [[f() for f in runs[1:]] for _ in range(3)]
    torch.cuda.synchronize()
    for pair in got:
        for out in pair:
            assert all(torch.equal(a, b) for a, b in zip(want, out))


def test_captured_and_replayed(tr):
    """Two graphs, each with its own workspaces, replayed at once; an eager run in between."""
    run = [everything(tr, gen(k), n=66 + k) for k in (3, 4)]
    want = [f() for f in run]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for f in run:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(f())
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(3):
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
        eager = run[0]()
        torch.cuda.synchronize()
        for w, o in zip(want, outs):
            assert all(torch.equal(a, b) for a, b in zip(w, o))
        assert all(torch.equal(a, b) for a, b in zip(want[0], eager))


def test_no_tokens_no_sequences_and_no_workers(tr):
    for b, s, length in ((2, 3, 0), (2, 0, 0), (0, 2, 5)):
        t, n = s * length, 24
        x = torch.zeros(b, t, n, dtype=BF, device="cuda")
        f = torch.ones(b, n, device="cuda")
        m = tr.pg_add_layer_norm(x, f, f, residual=x)
        assert m.y.shape == x.shape
        dx, dg, db = tr.pg_add_layer_norm_grad(x, x, m.mean, m.rstd, f)
        assert not dg.any() and not db.any()
        w, state = torch.ones(b, n, 3, device="cuda"), torch.ones(b, s, 2, n, dtype=BF, device="cuda")
        y, last = tr.pg_causal_conv(x, w, f, sequences=s, state=state, state_out=True)
        assert y.shape == x.shape and (length > 0 or torch.equal(last, state))
        dx, dw, db = tr.pg_causal_conv_grad(x, x, w, f, sequences=s)
        assert not dw.any() and not db.any()
        a, bc, h = -torch.ones(b, n, 16, device="cuda"), torch.zeros(b, t, 16, dtype=BF, device="cuda"), torch.ones(b, s, n, 16, device="cuda")
        y, last = tr.pg_selective_scan(x, x, a, bc, bc, sequences=s, state=h, state_out=True)
        assert y.shape == x.shape and (length > 0 or torch.equal(last, h))
        g = tr.pg_selective_scan_grad(x, x, x, a, bc, bc, sequences=s)
        assert not g.da.any() and not g.dskip.any() and not g.ddelta_bias.any()
        assert tr.pg_distillation_loss(x, labels=torch.zeros(b, t, dtype=torch.int32, device="cuda"), alpha=0.0).loss.shape == (b, t)


def test_what_is_behind_a_sequence_is_not_used(tr):
    """NaN and infinities behind the ends of sequences: as zeros there; lengths outside of 0 to length count as those."""
    g = gen(9)
    b, s, length, n = 2, 4, 45, 50
    c, more = scan_inputs(g, b, s, length, n, 16, BF, True, True, False, 0)
    dy = rand(g, b, s * length, n).to(BF)
    w, bias = rand(g, b, n, 4), rand(g, b, n)
    lengths = torch.tensor([[0, 1, 20, 45], [45, 44, 3, 16]], dtype=torch.int32, device="cuda")
    beyond = ~there(lengths, length, s, b).reshape(b, s * length, 1)
    dirty = lambda v: torch.where(beyond, torch.full_like(v, math.nan), v)
    odd = torch.where(lengths == 0, -5, torch.where(lengths == 45, 2 ** 31 - 1, lengths)).to(torch.int32)
    names = ("u", "delta", "b", "c", "z")
    bad = {**c, **{k: dirty(c[k]) for k in names}}
    for f, args in ((lambda q, d, n_: list(tr.pg_selective_scan(**q, **{**more, "lengths": n_}, state_out=True)), ()),
                    (lambda q, d, n_: list(tr.pg_selective_scan_grad(d, **q, **{**more, "lengths": n_})), ()),
                    (lambda q, d, n_: list(tr.pg_causal_conv(q["u"], w, bias, sequences=s, lengths=n_, state_out=True)), ()),
                    (lambda q, d, n_: list(tr.pg_causal_conv_grad(d, q["u"], w, bias, sequences=s, lengths=n_)), ())):
        want, got = f(c, dy, lengths), f(bad, dirty(dy), odd)
        for p, q in zip(want, got):
            assert torch.equal(p, q)
            if p.shape[:2] == (b, s * length):
                assert not p[beyond.expand_as(p)].any()


def test_shared_operands_and_a_single_worker(tr):
    g = gen(10)
    b, s, length, n = 3, 2, 20, 33
    c, more = scan_inputs(g, 1, s, length, n, 16, HF, True, False, False, 0)
    wide = {k: v.expand(b, *v.shape[1:]) for k, v in c.items()}
    one = {k: v[0] for k, v in c.items()}
    want = tr.pg_selective_scan(**c, **more)
    assert torch.equal(tr.pg_selective_scan(**wide, **more), want.expand(b, -1, -1))
    assert torch.equal(tr.pg_selective_scan(**one, **more), want[0])
    w, bias = rand(g, 1, n, 4), rand(g, 1, n)
    y = tr.pg_causal_conv(c["u"], w, bias, sequences=s)
    assert torch.equal(tr.pg_causal_conv(wide["u"], w.expand(b, -1, -1), bias[0], sequences=s), y.expand(b, -1, -1))
    assert torch.equal(tr.pg_causal_conv(one["u"], w[0], bias[0], sequences=s), y[0])
    m = tr.pg_add_layer_norm(c["u"], bias, bias)
    assert torch.equal(tr.pg_add_layer_norm(wide["u"], bias[0], bias[0]).y, m.y.expand(b, -1, -1))
    x, ids, teacher, labels = loss_inputs(g, 1, 5, 200, 4, HF, True, 0)
    r = tr.pg_distillation_loss(x, ids, teacher, labels, 2.0, 0.5, dloss=torch.ones(1, 5, device="cuda"))
    q = tr.pg_distillation_loss(x[0], ids[0], teacher[0], labels[0], 2.0, 0.5, dloss=torch.ones(5, device="cuda"))
    assert torch.equal(r.loss[0], q.loss) and torch.equal(r.dlogits[0], q.dlogits)


def test_a_sequence_in_pieces_is_the_sequence(tr):
    """States carried from call to call: token by token, and in uneven pieces, by the tolerances of the whole."""
    g = gen(12)
    c, more = scan_inputs(g, 2, 1, 23, 40, 16, BF, True, False, False, 0)
    f = scan_forward(c, more, 23)
    _, y, slack = scan_output(c, more, f)
    w, bias = rand(g, 2, 40, 4), rand(g, 2, 40)
    conv = tr.pg_causal_conv(c["u"], w, bias)
    for cuts in ([1] * 23, [5, 1, 9, 8]):
        state, held, at = torch.zeros(2, 1, 40, 16, device="cuda"), torch.zeros(2, 1, 3, 40, dtype=BF, device="cuda"), 0
        for k in cuts:
            part = {q: v[:, at:at + k] if q in ("u", "delta", "b", "c", "z") else v for q, v in c.items()}
            got, _ = tr.pg_selective_scan(**part, state=state, state_out=state)
            check(got, y[:, at:at + k], slack[:, at:at + k] + 2 * U * y[:, at:at + k].abs(), BF)
            part, _ = tr.pg_causal_conv(c["u"][:, at:at + k], w, bias, state=held, state_out=held)
            assert torch.equal(part, conv[:, at:at + k])
            at += k
        check(state, f["h"][-1], f["e"][-1] + 2 * U * f["h"][-1].abs())


def test_sequence_offsets_beyond_32_bits(tr):
    """Rows that start more than 2^31 elements into their matrix."""
    n, t = 28001, 80000
    x = torch.zeros(1, t, n, dtype=BF, device="cuda")
    x[0, -1] = rand(gen(5), n).to(BF)
    label = torch.full((1, t), 7, dtype=torch.int32, device="cuda")
    r = tr.pg_distillation_loss(x, labels=label, alpha=0.0, dloss=torch.ones(1, t, device="cuda"), out=x.clone())
    want = loss_reference(x[:, -1:], None, None, label[:, -1:], 1.0, 0.0, torch.ones(1, 1, device="cuda"))
    check(r.loss[:, -1:], want[0][None], want[1][None])
    check(r.dlogits[:, -1:], want[4][None], want[5][None], BF)
    assert abs(float(r.loss[0, 0]) - math.log(n)) < 1e-4


def test_long_sequences_of_wide_rows(tr):
    """A chunked scan and a convolution whose matrices have more than 2^31 elements: the last tokens, from the states before them."""
    n, t = 2048, 1 << 20
    u = torch.zeros(1, t, n, dtype=BF, device="cuda")
    u[0, -50:] = rand(gen(6), 50, n).to(BF)
    w = rand(gen(7), 1, n, 4)
    y = tr.pg_causal_conv(u, w)
    assert torch.equal(y[:, -53:], tr.pg_causal_conv(u[:, -53:].contiguous(), w))
    assert not y[:, :-50].any()
    bc = torch.ones(1, t, 1, dtype=BF, device="cuda")
    a = -torch.ones(1, n, 1, device="cuda")
    y, last = tr.pg_selective_scan(u, u, a, bc, bc, state_out=True, out=y)
    part = {"u": u[:, -50:].contiguous(), "delta": u[:, -50:].contiguous(), "a": a, "b": bc[:, -50:], "c": bc[:, -50:], "skip": torch.zeros(1, n, device="cuda"),
            "delta_bias": torch.zeros(1, n, device="cuda"), "z": None}
    more = {"sequences": 1, "lengths": None, "state": None}
    f = scan_forward(part, more, 4096)
    _, want, slack = scan_output(part, more, f)
    check(y[:, -50:], want, slack, BF)
    check(last, f["h"][-1], f["e"][-1] + 2 * U * f["h"][-1].abs())
    assert not y[:, :-50].any()


def test_refusals_of_the_sequence_binding(tr):
    x, f = torch.zeros(2, 6, 8, dtype=BF, device="cuda"), torch.zeros(2, 8, device="cuda")
    w, a, bc = torch.zeros(2, 8, 4, device="cuda"), torch.zeros(2, 8, 16, device="cuda"), torch.zeros(2, 6, 16, dtype=BF, device="cuda")
    ids, top = torch.zeros(2, 6, 3, dtype=torch.int32, device="cuda"), torch.zeros(2, 6, 3, dtype=BF, device="cuda")
    stat = torch.zeros(2, 6, device="cuda")
    from paper_2008_01425_b200 import binding as pg

    for f_ in (lambda: tr.pg_add_layer_norm(x, f[:, :7]), lambda: tr.pg_add_layer_norm(x, f, f.double()), lambda: tr.pg_add_layer_norm(x.transpose(1, 2)),
               lambda: tr.pg_add_layer_norm_grad(x, x, stat[:, :5], stat), lambda: tr.pg_add_layer_norm_grad(x, x, stat, stat, accumulate=True),
               lambda: tr.pg_causal_conv(x, w, sequences=4), lambda: tr.pg_causal_conv(x, w, sequences=True), lambda: tr.pg_causal_conv(x, w[..., :1]),
               lambda: tr.pg_causal_conv(x, w, activation="tanh"), lambda: tr.pg_causal_conv(x, w, lengths=torch.zeros(2, 1, device="cuda")),
               lambda: tr.pg_causal_conv(x, w, state=torch.zeros(2, 1, 2, 8, dtype=BF, device="cuda")), lambda: tr.pg_causal_conv_grad(x, x, w, accumulate=True),
               lambda: tr.pg_selective_scan(x, x, a, bc[..., :15], bc), lambda: tr.pg_selective_scan(x, x, torch.zeros(2, 8, 65, device="cuda"), bc, bc),
               lambda: tr.pg_selective_scan(x, x, a, bc, bc, state=torch.zeros(2, 1, 16, 8, device="cuda")), lambda: tr.pg_selective_scan(x, x.half(), a, bc, bc),
               lambda: tr.pg_selective_scan_grad(x, x, x, a, bc, bc, accumulate=True), lambda: tr.pg_distillation_loss(x, ids),
               lambda: tr.pg_distillation_loss(x, ids.long(), top), lambda: tr.pg_distillation_loss(x, ids, top[..., :2]), lambda: tr.pg_distillation_loss(x, out=x),
               lambda: tr.pg_distillation_loss(x, labels=torch.zeros(2, 6, dtype=torch.int64, device="cuda")),
               lambda: tr.pg_distillation_loss_grad(stat, x, stat), lambda: tr.pg_distillation_loss(x.cpu())):
        with pytest.raises(ValueError):
            f_()
    for f_ in (lambda: tr.pg_distillation_loss(x, ids, top, temperature=0.0), lambda: tr.pg_distillation_loss(x, ids, top, alpha=1.5),
               lambda: tr.pg_distillation_loss_grad(stat, x, None, ids, top), lambda: tr.pg_causal_conv(x, w, activation="gelu"),
               lambda: tr.pg_add_layer_norm(x, eps=-1.0), lambda: tr.pg_selective_scan(x, x, a, bc, bc, out=x[:1].expand(2, -1, -1))):
        with pytest.raises(pg.PowerGossipError) as e:
            f_()
        assert e.value.status == pg.PG_ERR_INVALID
    wide = torch.zeros(1, 2, 2000, dtype=BF, device="cuda")
    with pytest.raises(pg.PowerGossipError) as e:
        tr.pg_distillation_loss(wide, torch.zeros(1, 2, 1025, dtype=torch.int32, device="cuda"), torch.zeros(1, 2, 1025, dtype=BF, device="cuda"))
    assert e.value.status == pg.PG_ERR_TOO_LARGE


def test_more_states_than_a_grid_has_rows(tr):
    """A chunked gradient of 8.96 million states per sequence: a channel's gradients are those it has on its own."""
    n, m, t = 140000, 64, 41
    c, more = scan_inputs(gen(11), 1, 1, t, n, m, BF, False, False, False, 0)
    dy = rand(gen(12), 1, t, n).to(BF)
    got = tr.pg_selective_scan_grad(dy, **c, **more)
    last = slice(n - 16, n)
    part = {k: v[..., last].contiguous() if k in ("u", "delta", "skip", "delta_bias") else v[:, last].contiguous() if k == "a" else v for k, v in c.items()}
    want = tr.pg_selective_scan_grad(dy[..., last].contiguous(), **part, **more)
    assert torch.equal(got.du[..., last], want.du) and torch.equal(got.ddelta[..., last], want.ddelta)
