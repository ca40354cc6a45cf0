"""The training operators (include/pg_training.h) against their formulas in 64 bits.

Tolerances.  u = 2^-24 is half a step of fp32 at and above 1.  A sum of K products in fp32, in any order and with
every partial sum cut off instead of rounded, is within 2 u K sum|products| of the exact one.  A result
stored in 16 bits is within half a step of the type: 2^-8 (bf16, 7 bits after the point) or 2^-11 (fp16,
10 bits) of the power of two at or below it, never less than half the type's smallest step.  exp, reciprocal and reciprocal square root are good to a few
units; 32 u of the result covers them.  A value in 8 bits is within half a step of its block,
or a whole one where it is clamped at 127 (the largest may lie between 127 and 128 steps), and the
step is at most 2^-6 of the block's largest value, or the least step the form has.
"""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF, HF = torch.bfloat16, torch.float16
HALF_STEP = {BF: 2.0 ** -8, HF: 2.0 ** -11}
TINY = {BF: 2.0 ** -134, HF: 2.0 ** -25}
LEAST = {BF: -126, HF: -24}


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2008_01425_b200 import build as pg_build

    pg_build.build()


@pytest.fixture(scope="module")
def tr():
    from paper_2008_01425_b200 import training

    yield training
    assert training.pg_training_status() == 0


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rand(g, *shape, scale=1.0):
    return torch.randn(*shape, device="cuda", generator=g) * scale


def strided(t, pad):
    """The same values with rows `pad` elements longer in memory, and the padding NaN."""
    if not pad:
        return t
    big = torch.full((*t.shape[:-1], t.shape[-1] + pad), float("nan"), dtype=t.dtype, device=t.device)
    big[..., :t.shape[-1]] = t
    return big[..., :t.shape[-1]]


def check(got, want, slack, dtype=None):
    """|got - want| <= slack + half a step of the type; NaN exactly where expected."""
    got = got.double()
    assert got.shape == want.shape
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    limit = slack
    if dtype:
        below = torch.exp2(torch.floor(torch.log2((want.abs() + slack).clamp(min=2.0 ** -300))))
        limit = slack + torch.nan_to_num(below) * HALF_STEP[dtype] + TINY[dtype]
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf])
    err = torch.where(torch.isnan(want) | inf, torch.zeros_like(want), (got - want).abs() - limit)
    assert err.numel() == 0 or float(err.max()) <= 0.0, "off by %.3e more than allowed" % float(err.max())


def blocks_of(v):
    cols = v.shape[-1]
    n = -(-cols // 32)
    return torch.nn.functional.pad(v, (0, n * 32 - cols)).unflatten(-1, (n, 32))


def eight(v, dtype):
    """(q, scale byte, value) of the 8-bit form, by its definition."""
    b = blocks_of(v.double())
    top = b.abs().amax(-1)
    e = torch.where(top > 0, torch.floor(torch.log2(top.clamp(min=2.0 ** -400))) - 6, torch.full_like(top, -1000.0))
    e = e.clamp(min=LEAST[dtype])
    q = torch.round(b * torch.exp2(-e)[..., None]).clamp(-127, 127)
    bad = ~torch.isfinite(top)
    val = torch.where(bad[..., None], torch.full_like(q, float("nan")), q * torch.exp2(e)[..., None])
    byte = torch.where(bad, torch.full_like(e, 255.0), e + 127)
    return q.flatten(-2)[..., :v.shape[-1]], byte, val.flatten(-2)[..., :v.shape[-1]]


def stored8(c):
    """Values a Checkpoint8 stands for, in 64 bits."""
    s = torch.where(c.scales == 255, torch.full_like(c.scales, 0, dtype=torch.float64) + float("nan"),
                    torch.exp2(c.scales.double() - 127))
    return c.values.double() * s.repeat_interleave(32, dim=-1)[..., :c.values.shape[-1]]


def check8(c, want, slack, dtype):
    """An 8-bit result against the exact values it was rounded from."""
    top = (blocks_of(want.abs() + slack)).amax(-1)
    step = torch.maximum(top * 2.0 ** -6, torch.full_like(top, 2.0 ** LEAST[dtype]))
    limit = slack + step.repeat_interleave(32, dim=-1)[..., :want.shape[-1]]
    got = stored8(c)
    bad = ~torch.isfinite(blocks_of(want)).all(-1)
    bad = bad.repeat_interleave(32, dim=-1)[..., :want.shape[-1]]
    assert torch.equal(torch.isnan(got), bad)
    err = torch.where(bad, torch.zeros_like(got), (got - want).abs() - limit)
    assert err.numel() == 0 or float(err.max()) <= 0.0, "off by %.3e more than allowed" % float(err.max())


def make8(tr, v, dtype):
    """A Checkpoint8 made by the definition, with rows padded by garbage."""
    q, byte, _ = eight(v, dtype)
    cols = v.shape[-1]
    held = torch.full((*v.shape[:-1], -(-cols // 16) * 16 + 16), 77, dtype=torch.int8, device=v.device)
    held[..., :cols] = torch.nan_to_num(q).to(torch.int8)
    return tr.Checkpoint8(held[..., :cols], byte.to(torch.uint8), dtype)


def act(z, kind):
    if kind == "relu":
        return torch.where(z > 0, z, z * 0)
    if kind == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z) if kind == "silu" else z


def act_slope(z, kind):
    if kind == "relu":
        return (z > 0).double()
    if kind == "gelu":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if kind == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


# ------------------------------------------------------------------ norm
NORM_SHAPES = [(1, 1, 1), (3, 1, 650), (2, 5, 31), (2, 7, 33), (4, 9, 64), (1, 130, 257), (2, 33, 1000), (3, 17, 1023), (2, 9, 1024),
               (1, 5, 1025), (2, 3, 2600), (1, 3, 4608), (1, 2, 8200), (1, 2, 16384)]


@pytest.mark.parametrize("shape", NORM_SHAPES)
@pytest.mark.parametrize("dtype,pad,residual,with8", [(BF, 0, True, True), (HF, 3, True, False), (BF, 8, False, True), (HF, 2, False, False)])
def test_norm(tr, shape, dtype, pad, residual, with8):
    g = gen(hash(shape) % 1000)
    b, t, n = shape
    x = strided(rand(g, b, t, n, scale=2.0).to(dtype), pad)
    r = strided(rand(g, b, t, n).to(dtype), pad + 1) if residual else None
    gain = 1 + 0.3 * rand(g, b, n)
    out = tr.pg_add_rms_norm(x, gain, residual=r, eps=1e-5, eight_bit=with8, save_h8=with8)
    s = x.double() + (r.double() if residual else 0.0)
    root = ((s * s).mean(-1) + 1e-5) ** -0.5
    # the sum rounds once (u), the mean n times 2 u at most
    slack_root = root * (n + 40) * 2 * U
    check(out.rstd, root, slack_root)
    if residual:
        check(out.h, s, s.abs() * U, dtype)
    y = s * root[..., None] * gain.double()[:, None]
    slack = y.abs() * (n + 40) * 2 * U
    if with8:
        check8(out.y8, y, slack, dtype)
        check8(out.h8, s, s.abs() * U, dtype)
        assert torch.equal(out.y.double(), stored8(out.y8))
    else:
        check(out.y, y, slack, dtype)


@pytest.mark.parametrize("shape", NORM_SHAPES)
@pytest.mark.parametrize("dtype,pad,dh,from8", [(BF, 0, True, False), (HF, 3, False, True), (BF, 8, True, True), (HF, 2, False, False)])
def test_norm_gradient(tr, shape, dtype, pad, dh, from8):
    g = gen(hash(shape) % 1000 + 1)
    b, t, n = shape
    h = rand(g, b, t, n, scale=2.0).to(dtype)
    root = ((h.double() ** 2).mean(-1) + 1e-5) ** -0.5
    dy = strided(rand(g, b, t, n).to(dtype), pad)
    add = strided(rand(g, b, t, n).to(dtype), pad + 1) if dh else None
    gain = 1 + 0.3 * rand(g, b, n)
    first = rand(g, b, n)
    kept = make8(tr, h.float(), dtype) if from8 else strided(h, pad)
    hv = stored8(kept) if from8 else h.double()
    dgain = first.clone()
    dx, got = tr.pg_add_rms_norm_grad(dy, kept, root.float(), gain, dh=add, gain_grad=dgain, accumulate=True)
    assert got is dgain
    rs = root.float().double()[..., None]
    u = hv * rs
    a = dy.double() * gain.double()[:, None]
    dot = (a * u).mean(-1, keepdim=True)
    want = rs * (a - u * dot) + (add.double() if dh else 0.0)
    mag = rs * (a.abs() + u.abs() * (a * u).abs().mean(-1, keepdim=True)) + (add.double().abs() if dh else 0.0)
    check(dx, want, mag * (n + 16) * 2 * U, dtype)
    check(dgain, first.double() + (dy.double() * u).sum(1), (first.abs().double() + (dy.double() * u).abs().sum(1)) * (t + 16) * 2 * U)
    dx2, dg2 = tr.pg_add_rms_norm_grad(dy, kept, root.float(), gain, dh=add)
    assert torch.equal(dx2, dx)
    check(dg2, (dy.double() * u).sum(1), (dy.double() * u).abs().sum(1) * (t + 16) * 2 * U)


def test_norm_gradient_against_differences(tr):
    """<dx, d> against central differences of the 64-bit forward pass along random directions."""
    g = gen(5)
    b, t, n = 2, 3, 96
    x = rand(g, b, t, n).to(BF)
    gain = 1 + 0.3 * rand(g, b, n)
    c = rand(g, b, t, n).to(BF)

    def loss(v, k):
        return (c.double() * v * (((v * v).mean(-1, keepdim=True) + 1e-5) ** -0.5) * k[:, None]).sum()

    rstd = tr.pg_add_rms_norm(x, gain).rstd
    dx, dg = tr.pg_add_rms_norm_grad(c, x, rstd, gain)
    eps = 1e-4
    for k in range(4):
        d = rand(g, b, t, n).double()
        diff = (loss(x.double() + eps * d, gain.double()) - loss(x.double() - eps * d, gain.double())) / (2 * eps)
        # every entry of dx is within half a bf16 step; the differences' own error is eps^2 times a third derivative of order n
        assert abs(float((dx.double() * d).sum() - diff)) <= float((dx.double() * d).abs().sum()) * 2.0 ** -8 + 1e-6 * n * b * t
        e = rand(g, b, n).double()
        diff = (loss(x.double(), gain.double() + eps * e) - loss(x.double(), gain.double() - eps * e)) / (2 * eps)
        assert abs(float((dg.double() * e).sum() - diff)) <= float((dg.double() * e).abs().sum()) * 1e-5 + 1e-6


# ------------------------------------------------------------------ products
PRODUCT_SHAPES = [(1, 1, 1, 1), (2, 1, 650, 260), (3, 5, 16, 16), (2, 33, 147, 65), (1, 64, 64, 128), (2, 130, 72, 136), (1, 257, 200, 129),
                  (5, 40, 650, 96), (1, 300, 512, 520), (2, 16, 1024, 256), (1, 1040, 64, 24), (3, 129, 136, 384), (1, 2, 4608, 512),
                  (40, 3, 24, 40), (1, 600, 1032, 1288), (2, 513, 328, 2600),
                  # enough tiles for pairs of blocks, in one, two or all of the products
                  (5, 300, 650, 1000), (40, 257, 136, 72), (20, 200, 520, 700), (38, 129, 64, 33), (19, 385, 257, 513), (37, 7, 300, 200)]


@pytest.mark.parametrize("shape", PRODUCT_SHAPES)
@pytest.mark.parametrize("dtype,pad,activation,residual,save", [(BF, 0, "gelu", True, True), (HF, 1, "relu", False, False), (BF, 8, "silu", False, True),
                                                                  (HF, 0, "none", True, False)])
def test_linear(tr, shape, dtype, pad, activation, residual, save):
    g = gen(hash(shape) % 1000 + 2)
    b, t, k, n = shape
    x = strided(rand(g, b, t, k).to(dtype), pad)
    w = strided(rand(g, b, n, k, scale=k ** -0.5).to(dtype), pad)
    bias = rand(g, b, n)
    r = strided(rand(g, b, t, n).to(dtype), pad) if residual else None
    got = tr.pg_linear(x, w, bias, residual=r, activation=activation, save_z=save)
    y, z8 = got if save else (got, None)
    z = x.double() @ w.double().transpose(1, 2) + bias.double()[:, None]
    slack = (x.double().abs() @ w.double().abs().transpose(1, 2) + bias.double().abs()[:, None]) * (k + 2) * 2 * U
    if save:
        check8(z8, z, slack, dtype)
    want = act(z, activation)
    slack = 1.13 * slack + z.abs() * 32 * U      # no activation here is steeper than 1.13
    if residual:
        want = want + r.double()
        slack = slack + want.abs() * U
    check(y, want, slack, dtype)


@pytest.mark.parametrize("n", list(range(257, 300, 3)) + [264, 272, 288])
@pytest.mark.parametrize("dtype,pad", [(BF, 0), (HF, 1), (BF, 8), (HF, 5)])
def test_ends_of_residual_rows(tr, n, dtype, pad):
    """Residual rows that start and end anywhere in a 16-byte piece, through the path with tokens as lanes; the residual
    ends with its allocation."""
    g = gen(n)
    b, t, k = 19, 257, 24
    x, w = rand(g, b, t, k).to(dtype), rand(g, b, n, k, scale=k ** -0.5).to(dtype)
    r = strided(rand(g, b, t, n).to(dtype), pad)
    y = tr.pg_linear(x, w, residual=r)
    z = x.double() @ w.double().transpose(1, 2)
    slack = (x.double().abs() @ w.double().abs().transpose(1, 2)) * (k + 2) * 2 * U
    check(y, z + r.double(), slack + (z + r.double()).abs() * U, dtype)


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("k", [7, 5120, 5128, 10240, 20480, 20488])
@pytest.mark.parametrize("dtype,pad", [(BF, 0), (HF, 1), (BF, 2)])
def test_few_tokens_at_the_limits_of_their_path(tr, tokens, k, dtype, pad):
    g = gen(tokens * k)
    b, n = 2, 45
    x, w = strided(rand(g, b, tokens, k).to(dtype), pad), strided(rand(g, b, n, k, scale=k ** -0.5).to(dtype), pad)
    bias, r = rand(g, b, n), rand(g, b, tokens, n).to(dtype)
    y, z8 = tr.pg_linear(x, w, bias, residual=r, activation="silu", save_z=True)
    z = x.double() @ w.double().transpose(1, 2) + bias.double()[:, None]
    slack = (x.double().abs() @ w.double().abs().transpose(1, 2) + bias.double().abs()[:, None]) * (k + 2) * 2 * U
    check8(z8, z, slack, dtype)
    want = act(z, "silu") + r.double()
    check(y, want, 1.13 * slack + z.abs() * 32 * U + want.abs() * U, dtype)


@pytest.mark.parametrize("shape", PRODUCT_SHAPES)
@pytest.mark.parametrize("dtype,pad,residual", [(BF, 0, True), (HF, 1, False), (BF, 8, False)])
def test_input_gradient(tr, shape, dtype, pad, residual):
    g = gen(hash(shape) % 1000 + 3)
    b, t, k, n = shape
    dz = strided(rand(g, b, t, n).to(dtype), pad)
    w = strided(rand(g, b, n, k, scale=n ** -0.5).to(dtype), pad)
    r = strided(rand(g, b, t, k).to(dtype), pad) if residual else None
    dx = tr.pg_linear_input_grad(dz, w, residual=r)
    want = dz.double() @ w.double() + (r.double() if residual else 0.0)
    slack = (dz.double().abs() @ w.double().abs() + (r.double().abs() if residual else 0.0)) * (n + 2) * 2 * U
    check(dx, want, slack, dtype)


@pytest.mark.parametrize("shape", PRODUCT_SHAPES)
@pytest.mark.parametrize("dtype,pad,from8,accumulate", [(BF, 0, True, False), (HF, 1, False, True), (BF, 8, False, False), (HF, 0, True, True)])
def test_weight_gradient(tr, shape, dtype, pad, from8, accumulate):
    g = gen(hash(shape) % 1000 + 4)
    b, t, k, n = shape
    dz = strided(rand(g, b, t, n).to(dtype), pad)
    x = rand(g, b, t, k).to(dtype)
    kept = make8(tr, x.float(), dtype) if from8 else strided(x, pad)
    xv = stored8(kept) if from8 else x.double()
    first = rand(g, b, n, k)
    out = torch.full((b, n, k + 3), 5.0, device="cuda")
    out[..., :k] = first
    dw = tr.pg_linear_weight_grad(dz, kept, out=out[..., :k], accumulate=accumulate)
    want = dz.double().transpose(1, 2) @ xv + (first.double() if accumulate else 0.0)
    slack = (dz.double().abs().transpose(1, 2) @ xv.abs() + (first.double().abs() if accumulate else 0.0)) * (t + 2) * 2 * U
    check(dw, want, slack)
    assert bool((out[..., k:] == 5.0).all())            # nothing beside the rows is written


@pytest.mark.parametrize("shape", [(1, 8192, 128, 64), (1, 40000, 96, 70), (20, 4096, 512, 264), (1, 5000, 1200, 1030)])
@pytest.mark.parametrize("from8", [False, True])
def test_long_sums_keep_fp32(tr, shape, from8):
    """A weight gradient over many tokens is as exact as a sum in fp32 with rounding: a few units of
    its size, not one cut-off unit per token.  Split over blocks, in chunks, and both."""
    g = gen(11)
    b, t, k, n = shape
    dz, x = rand(g, b, t, n).to(BF), rand(g, b, t, k).to(BF)
    kept = make8(tr, x.float(), BF) if from8 else x
    xv = stored8(kept) if from8 else x.double()
    want = dz.double().transpose(1, 2) @ xv
    got = tr.pg_linear_weight_grad(dz, kept)
    rel = float((got.double() - want).norm() / want.norm())
    assert rel <= 1e-6, rel
    twice = tr.pg_linear_weight_grad(dz, kept, out=got.clone(), accumulate=True)
    assert float((twice.double() - 2 * want).norm() / want.norm()) <= 3e-6


def test_linear_gradients_against_differences(tr):
    """Both gradients of a layer with activation, against central differences of its 64-bit forward pass."""
    g = gen(6)
    b, t, k, n = 2, 20, 48, 72
    x, w, bias = rand(g, b, t, k).to(BF), rand(g, b, n, k, scale=k ** -0.5).to(BF), rand(g, b, n)
    c = rand(g, b, t, n).to(BF)
    for kind in ("gelu", "silu"):
        _, z8 = tr.pg_linear(x, w, bias, activation=kind, save_z=True)
        dz, db = tr.pg_activation_grad(c, z8, kind)
        dx, dw = tr.pg_linear_input_grad(dz, w), tr.pg_linear_weight_grad(dz, x)

        def loss(xx, ww, bb):
            return (c.double() * act(xx @ ww.transpose(1, 2) + bb[:, None], kind)).sum()

        at = (x.double(), w.double(), bias.double())
        z = at[0] @ at[1].transpose(1, 2) + at[2][:, None]
        # z8 is within a step (2^-6 of the block's largest |z|, at most 2^-6 max|z|) of z and no slope here changes faster
        # than 1.6 per unit of z (|gelu''| <= 1.6/sqrt(2 pi) * 2, |silu''| <= 0.5); dz is then rounded to bf16
        dz_err = c.double().abs() * 1.6 * 2.0 ** -6 * float(z.abs().max()) + dz.double().abs() * 2.0 ** -8
        eps = 1e-5
        for i, (got, size) in enumerate(((dx, dz_err @ at[1].abs()), (dw, dz_err.transpose(1, 2) @ at[0].abs()), (db, dz_err.sum(1)))):
            d = rand(g, *got.shape).double()
            up = [v + eps * d if j == i else v for j, v in enumerate(at)]
            dn = [v - eps * d if j == i else v for j, v in enumerate(at)]
            diff = (loss(*up) - loss(*dn)) / (2 * eps)
            # independent errors of the entries: their root of squares, with a factor 4, and not their sum
            limit = 4 * float(((size + got.double().abs() * 2.0 ** -8) * d).norm()) + 1e-5
            assert abs(float((got.double() * d).sum() - diff)) <= limit


# ------------------------------------------------------------------ activation gradient
@pytest.mark.parametrize("shape", [(1, 1, 1), (2, 1, 650), (3, 9, 33), (1, 1000, 64), (2, 300, 257), (4, 65, 2600), (1, 5000, 31), (2, 40, 1024)])
@pytest.mark.parametrize("activation,dtype,pad", [("gelu", BF, 0), ("silu", HF, 1), ("relu", BF, 2), ("none", HF, 8)])
def test_activation_gradient(tr, shape, activation, dtype, pad):
    g = gen(hash(shape) % 1000 + 5)
    b, t, n = shape
    dy = strided(rand(g, b, t, n).to(dtype), pad)
    z8 = make8(tr, rand(g, b, t, n, scale=2.0), dtype)
    first = rand(g, b, n)
    db = first.clone()
    dz, _ = tr.pg_activation_grad(dy, z8, activation, bias_grad=db, accumulate=True)
    want = dy.double() * act_slope(stored8(z8), activation)
    slack = dy.double().abs() * 64 * U * (1 + stored8(z8).abs())
    check(dz, want, slack, dtype)
    check(db, first.double() + want.sum(1), slack.sum(1) + (first.double().abs() + want.abs().sum(1)) * (t + 10) * 2 * U)
    if activation == "none":
        plain, db2 = tr.pg_activation_grad(dy, None, "none")
        assert torch.equal(plain, dz)
        check(db2, want.sum(1), want.abs().sum(1) * (t + 10) * 2 * U)


def test_slopes_far_from_zero(tr):
    for dtype, most in ((BF, 3e38), (HF, 6e4)):
        z = torch.tensor([-most, -1e4, -100.0, -20.0, 0.0, 20.0, 100.0, 1e4, most], device="cuda").reshape(-1, 1).repeat(1, 32)
        z8 = tr.pg_checkpoint_write(z.to(dtype))
        dy = torch.ones(9, 32, device="cuda", dtype=dtype)
        for kind in ("relu", "gelu", "silu"):
            dz, _ = tr.pg_activation_grad(dy, z8, kind)
            want = torch.tensor([0, 0, 0, 0, 0.0 if kind == "relu" else 0.5, 1, 1, 1, 1], device="cuda").reshape(-1, 1)
            assert float((dz.float() - want).abs().max()) <= 1e-6, kind


# ------------------------------------------------------------------ 8-bit form
@pytest.mark.parametrize("shape", [(1, 1), (3, 31), (2, 32), (5, 33), (7, 650), (4, 1024), (3, 28000)])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("pad", [0, 1, 2, 8])
def test_checkpoint_is_bit_exact(tr, shape, dtype, pad):
    g = gen(hash(shape) % 1000 + 6)
    x = rand(g, *shape) * torch.exp(3 * rand(g, shape[0], 1))
    x[:, ::5] = 0.0
    if shape[1] > 40:
        x[0, 32:64] = 0.0                                         # a block of zeros
        x[-1, 3] = float("nan")
        x[0, 0] = float("inf")
        x[0, 64:80] = 2.0 ** -130 if dtype == BF else 2.0 ** -24    # under the least step, and one of it
        x[0, 100] = -float("inf") if shape[1] > 200 else 1.0
    x = x.to(dtype)
    x8 = tr.pg_checkpoint_write(strided(x, pad))
    q, byte, val = eight(x, dtype)
    fine = torch.isfinite(val)
    assert torch.equal(x8.scales.double(), byte)
    assert torch.equal(x8.values.double()[fine], q[fine])
    back = tr.pg_checkpoint_read(x8)
    assert back.dtype == dtype and torch.equal(torch.isnan(back), ~fine)
    assert torch.equal(back.double()[fine], val[fine])
    again = tr.pg_checkpoint_read(tr.pg_checkpoint_write(back), out=strided(back.clone(), pad))
    assert torch.equal(again[fine], back[fine])                   # what the form stands for is in it exactly


def test_every_eight_bit_value_reads_back(tr):
    """All 255 values under all scales, through the reader, the weight gradient and the activation gradient."""
    for dtype, scales in ((BF, list(range(1, 249)) + [255]), (HF, list(range(103, 137)) + [255])):
        q = torch.arange(-127, 128, device="cuda")
        q = torch.cat([q, q[:1]]).to(torch.int8).repeat(len(scales), 1)                       # 256 columns
        s = torch.tensor(scales, device="cuda", dtype=torch.uint8)[:, None].repeat(1, 8)
        x8 = tr.Checkpoint8(q, s, dtype)
        val = stored8(x8)
        back = tr.pg_checkpoint_read(x8).double()
        assert torch.equal(back[:-1], val[:-1]) and bool(torch.isnan(back[-1]).all())
        one = torch.zeros(len(scales) - 1, len(scales) - 1, device="cuda", dtype=dtype).fill_diagonal_(1.0)
        dw = tr.pg_linear_weight_grad(one, tr.Checkpoint8(q[:-1], s[:-1], dtype))
        assert torch.equal(dw.double(), val[:-1])


# ------------------------------------------------------------------ edges
def test_no_tokens_and_no_workers(tr):
    for b, t in ((2, 0), (0, 4)):
        x, w = torch.empty(b, t, 24, device="cuda", dtype=BF), torch.ones(b, 40, 24, device="cuda", dtype=BF)
        y, z8 = tr.pg_linear(x, w, torch.ones(b, 40, device="cuda"), activation="gelu", save_z=True)
        assert y.shape == (b, t, 40) and z8.values.shape == (b, t, 40)
        assert tr.pg_linear_input_grad(y, w).shape == (b, t, 24)
        dw = tr.pg_linear_weight_grad(y, x)
        assert dw.shape == (b, 40, 24) and float(dw.abs().sum()) == 0.0
        assert float(tr.pg_linear_weight_grad(y, tr.pg_checkpoint_write(x)).abs().sum()) == 0.0
        kept = torch.ones(b, 40, 24, device="cuda")
        assert bool((tr.pg_linear_weight_grad(y, x, out=kept, accumulate=True) == 1).all())
        n = tr.pg_add_rms_norm(x, torch.ones(b, 24, device="cuda"), residual=x, eight_bit=True)
        dx, dg = tr.pg_add_rms_norm_grad(x, n.h, n.rstd, None)
        assert dx.shape == x.shape and float(dg.abs().sum()) == 0.0
        dz, db = tr.pg_activation_grad(y, z8, "gelu")
        assert dz.shape == y.shape and float(db.abs().sum()) == 0.0
        assert tr.pg_checkpoint_read(z8).shape == y.shape


def test_what_is_not_finite_stays_where_it_is(tr):
    g = gen(7)
    b, t, k, n = 2, 70, 96, 160
    x, w = rand(g, b, t, k).to(BF), rand(g, b, n, k, scale=0.1).to(BF)
    x[0, 3, 5] = float("nan")
    x[1, 64, 0] = float("inf")
    y, z8 = tr.pg_linear(x, w, activation="none", save_z=True)
    bad = torch.zeros(b, t, dtype=torch.bool, device="cuda")
    bad[0, 3] = bad[1, 64] = True
    assert torch.equal(~torch.isfinite(y).all(-1), bad) and torch.equal((~torch.isfinite(y)).any(-1), bad)
    assert torch.equal(torch.isnan(tr.pg_checkpoint_read(z8)).any(-1), bad)
    assert torch.equal(torch.isnan(tr.pg_add_rms_norm(x).y).any(-1), bad)
    dw = tr.pg_linear_weight_grad(torch.ones(b, t, n, device="cuda", dtype=BF), x)
    assert torch.equal((~torch.isfinite(dw)).all(1), (~torch.isfinite(x)).any(1))
    dw = tr.pg_linear_weight_grad(torch.ones(b, t, n, device="cuda", dtype=BF), tr.pg_checkpoint_write(x))
    hit = torch.zeros(b, k, dtype=torch.bool, device="cuda")
    hit[0, :32] = hit[1, :32] = True                                       # the whole block of 32
    assert torch.equal(torch.isnan(dw).all(1), hit)


def test_shared_operands_and_single_worker(tr):
    g = gen(8)
    x, w = rand(g, 3, 20, 64).to(BF), rand(g, 1, 48, 64).to(BF)
    y = tr.pg_linear(x, w.expand(3, 48, 64), activation="relu")
    for i in range(3):
        assert torch.equal(tr.pg_linear(x[i], w[0], activation="relu"), y[i])
    dx = tr.pg_linear_input_grad(y, w.expand(3, 48, 64))
    assert torch.equal(dx[1], tr.pg_linear_input_grad(y[1], w[0]))
    n = tr.pg_add_rms_norm(x, torch.ones(64, device="cuda"))
    assert torch.equal(n.y[2], tr.pg_add_rms_norm(x[2]).y)


def test_results_repeat_bit_for_bit(tr):
    g = gen(9)
    x, dz = rand(g, 1, 900, 200).to(BF), rand(g, 1, 900, 264).to(BF)
    z8 = tr.pg_checkpoint_write(dz)
    runs = [(tr.pg_linear_weight_grad(dz, x), tr.pg_activation_grad(dz, z8, "gelu")[1],
             tr.pg_add_rms_norm_grad(x, x, torch.ones(1, 900, device="cuda"))[1], tr.pg_linear(x, dz.transpose(1, 2)[..., :200].contiguous()))
            for _ in range(3)]
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))


def test_in_place_outputs(tr):
    g = gen(10)
    x, r = rand(g, 2, 30, 136).to(BF), rand(g, 2, 30, 136).to(BF)
    w = rand(g, 2, 136, 136, scale=0.1).to(BF)
    want = tr.pg_linear(x, w, residual=r)
    assert torch.equal(tr.pg_linear(x, w, residual=r, out=r), want)
    z8 = tr.pg_checkpoint_write(x)
    want, _ = tr.pg_activation_grad(r, z8, "silu")
    assert torch.equal(tr.pg_activation_grad(r, z8, "silu", out=r)[0], want)
    n = tr.pg_add_rms_norm(x)
    want, _ = tr.pg_add_rms_norm_grad(r, x, n.rstd, dh=w[:, :30])
    assert torch.equal(tr.pg_add_rms_norm_grad(r, x, n.rstd, dh=w[:, :30], out=r)[0], want)


def test_another_stream(tr):
    g = gen(12)
    x, w = rand(g, 4, 256, 512).to(BF), rand(g, 4, 512, 512, scale=0.05).to(BF)
    want = tr.pg_linear(x, w, activation="gelu")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = tr.pg_linear(x, w, activation="gelu", stream=s)
    raw = tr.pg_linear(x, w, activation="gelu", stream=s.cuda_stream)
    with torch.cuda.stream(s):
        inside = tr.pg_linear(x, w, activation="gelu")
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(raw, want) and torch.equal(inside, want)


def test_offsets_beyond_32_bits(tr):
    """Rows and workers that lie further apart than 2^31 elements."""
    base = torch.zeros((1 << 31) + (1 << 20), dtype=BF, device="cuda")
    g = gen(13)
    far = torch.as_strided(base, (2, 8, 64), ((1 << 31) + 64, 128, 1))
    far.copy_(rand(g, 2, 8, 64).to(BF))
    near = far.contiguous()
    w = rand(g, 2, 64, 64, scale=0.1).to(BF)
    assert torch.equal(tr.pg_linear(far, w), tr.pg_linear(near, w))
    assert torch.equal(tr.pg_linear_weight_grad(far, near), tr.pg_linear_weight_grad(near, near))
    assert torch.equal(tr.pg_add_rms_norm(far).y, tr.pg_add_rms_norm(near).y)
    rows = torch.as_strided(base, (2, 64), ((1 << 31) + 8, 1))
    rows.copy_(near[:, 0])
    c = tr.pg_checkpoint_write(rows)
    assert torch.equal(c.values, tr.pg_checkpoint_write(near[:, 0].contiguous()).values)
    out = torch.as_strided(base, (2, 64), ((1 << 31) + 8, 1), 4096)
    tr.pg_checkpoint_read(c, out=out)
    assert torch.equal(out, tr.pg_checkpoint_read(c))


# ------------------------------------------------------------------ refusals
def test_refusals_of_the_binding(tr):
    x, w = torch.zeros(2, 4, 16, device="cuda", dtype=BF), torch.zeros(2, 8, 16, device="cuda", dtype=BF)
    for bad in (lambda: tr.pg_linear(x.cpu(), w), lambda: tr.pg_linear(x.float(), w), lambda: tr.pg_linear(x, w.half()),
                lambda: tr.pg_linear(x, w[:1]), lambda: tr.pg_linear(x, w[..., :8]), lambda: tr.pg_linear(x, w.transpose(1, 2)),
                lambda: tr.pg_linear(x, w, activation="tanh"), lambda: tr.pg_linear(x, w, bias=torch.zeros(8, device="cuda", dtype=BF)),
                lambda: tr.pg_linear_weight_grad(x, x, accumulate=True), lambda: tr.pg_linear_input_grad(x, w),
                lambda: tr.pg_add_rms_norm(x, torch.zeros(3, 16, device="cuda")), lambda: tr.pg_checkpoint_read(x),
                lambda: tr.pg_activation_grad(x, tr.pg_checkpoint_write(x.half()), "relu")):
        with pytest.raises(ValueError):
            bad()


def test_refusals_of_the_library(tr):
    from paper_2008_01425_b200 import binding as pg

    x, w = torch.zeros(2, 4, 16, device="cuda", dtype=BF), torch.zeros(2, 8, 16, device="cuda", dtype=BF)
    y = torch.full((2, 4, 8), 3.0, device="cuda", dtype=BF)
    host = torch.zeros(2, 4, 16, dtype=BF)
    lib = pg.load_library()

    def linear(xp=x.data_ptr(), ld=16, stride=64, out_stride=32, dtype=0, act=0, tokens=4, n_in=16, yp=y.data_ptr(), out_ld=8):
        a = tr.pg_linear_args(dtype, act, 2, tokens, n_in, 8, tr.pg_matrix(xp, ld, stride), tr.pg_matrix(w.data_ptr(), 16, 128), None, 0,
                              tr.pg_matrix(None, 0, 0), tr.pg_matrix(yp, out_ld, out_stride), tr.pg_matrix8(None, None, 0, 0, 0, 0))
        return lib.pg_linear(ctypes.byref(a), None, 0, None)

    assert linear(yp=torch.empty_like(y).data_ptr()) == pg.PG_OK
    for bad in (dict(xp=None), dict(xp=host.data_ptr()), dict(xp=x.data_ptr() + 1), dict(ld=15), dict(stride=-1), dict(out_stride=16),
                dict(dtype=2), dict(act=4), dict(act=-1), dict(tokens=-1), dict(n_in=0), dict(yp=None), dict(out_ld=7), dict(out_stride=0)):
        assert linear(**bad) == pg.PG_ERR_INVALID, bad
    # a weight gradient's rows that are not 16-byte aligned go through the workspace, so there has to be one
    dw = torch.full((2, 8, 16), 3.0, device="cuda")
    a = tr.pg_weight_grad_args(0, 2, 4, 16, 8, 0, tr.pg_matrix(y.data_ptr(), 8, 32), tr.pg_matrix(x.data_ptr() + 2, 16, 64),
                               tr.pg_matrix8(None, None, 0, 0, 0, 0), tr.pg_matrix(dw.data_ptr(), 16, 128))
    need = ctypes.c_size_t(0)
    assert lib.pg_linear_weight_grad_workspace_bytes(ctypes.byref(a), ctypes.byref(need)) == pg.PG_OK and need.value >= 2 * 4 * 16 * 2
    assert lib.pg_linear_weight_grad(ctypes.byref(a), None, 0, None) == pg.PG_ERR_WORKSPACE
    assert lib.pg_linear_weight_grad(ctypes.byref(a), x.data_ptr(), need.value - 1, None) == pg.PG_ERR_WORKSPACE
    torch.cuda.synchronize()
    assert bool((dw == 3.0).all())
    c8 = tr.pg_checkpoint_write(x)
    a = tr.pg_checkpoint_args(0, 2, 4, 16, tr.pg_matrix(x.data_ptr(), 16, 64),
                              tr.pg_matrix8(c8.values.data_ptr(), c8.scales.data_ptr(), 24, 96, 1, 4))
    assert lib.pg_checkpoint_write(ctypes.byref(a), None) == pg.PG_ERR_INVALID        # ld not a multiple of 16
    a = tr.pg_norm_grad_args(0, 2, 4, 16, 0, tr.pg_matrix(x.data_ptr(), 16, 64), tr.pg_matrix(None, 16, 0),
                             tr.pg_matrix8(None, None, 16, 0, 1, 0), None, None, 0, tr.pg_matrix(None, 16, 0),
                             tr.pg_matrix(x.data_ptr(), 16, 64), None, 0)
    assert lib.pg_add_rms_norm_grad(ctypes.byref(a), None, 0, None) == pg.PG_ERR_INVALID   # neither h nor h8
    big = torch.zeros(1, 1, 16392, device="cuda", dtype=BF)
    with pytest.raises(pg.PowerGossipError) as e:
        tr.pg_add_rms_norm(big)
    assert e.value.status == pg.PG_ERR_TOO_LARGE
    torch.cuda.synchronize()
    assert bool((y == 3.0).all())


def test_refusal_of_a_norm_gradient_that_is_too_wide(tr):
    from paper_2008_01425_b200 import binding as pg

    x, rstd = torch.zeros(1, 2, 16392, device="cuda", dtype=BF), torch.ones(1, 2, device="cuda")
    with pytest.raises(pg.PowerGossipError) as e:
        tr.pg_add_rms_norm_grad(x, x, rstd)
    assert e.value.status == pg.PG_ERR_TOO_LARGE


@pytest.mark.parametrize("shape", [(64, 512, 512, 512), (32, 700, 650, 2600), (20, 4096, 512, 264), (37, 65, 300, 200)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_weight_gradients_of_many_tiles_repeat_bit_for_bit(tr, shape, dtype):
    """Enough tiles for every block to take several: x widened from 8 bits beside the products, and pairs of blocks."""
    g = gen(21)
    b, t, k, n = shape
    dz, x8 = rand(g, b, t, n).to(dtype), tr.pg_checkpoint_write(rand(g, b, t, k).to(dtype))
    first = tr.pg_linear_weight_grad(dz, x8)
    for _ in range(8):
        assert torch.equal(tr.pg_linear_weight_grad(dz, x8), first)
    # the same products from the 16-bit values x8 stands for: the operands are equal, only the chunks of a sum differ
    x = tr.pg_checkpoint_read(x8)
    size = (dz[0].double().abs().transpose(0, 1) @ x[0].double().abs())
    from16 = tr.pg_linear_weight_grad(dz, x)
    assert float(((first[0] - from16[0]).double().abs() / size).max()) <= 2 * (t + 2) * 2 * U
    for _ in range(8):
        assert torch.equal(tr.pg_linear_weight_grad(dz, x), from16)


def test_a_wait_that_runs_out_is_reported_once(tr):
    from paper_2008_01425_b200 import binding as pg

    assert tr.pg_training_status() == pg.PG_OK
    assert tr.pg_selftest_training_timeout() == pg.PG_ERR_TIMEOUT
    assert tr.pg_training_status() == pg.PG_OK               # told once; the GPU goes on
    s = torch.cuda.Stream()
    assert tr.pg_selftest_training_timeout(stream=s) == pg.PG_ERR_TIMEOUT
    x, w = torch.ones(1, 4, 64, device="cuda", dtype=BF), torch.ones(1, 32, 64, device="cuda", dtype=BF)
    assert bool((tr.pg_linear(x, w) == 64).all()) and tr.pg_training_status() == pg.PG_OK


@pytest.mark.parametrize("raw", [False, True])
def test_memory_of_calls_on_another_stream(tr, raw):
    """Results do not lie in memory that the current stream still writes, and inputs that are let go are not
    reused under the call."""
    g = gen(14)
    x, w = rand(g, 4, 250, 515).to(BF), rand(g, 4, 520, 515, scale=0.05).to(BF)     # rows that need a workspace
    want = tr.pg_linear(x, w, activation="gelu")
    grads = tr.pg_linear_weight_grad(want, x)
    s = torch.cuda.Stream()
    stream = s.cuda_stream if raw else s
    torch.cuda.synchronize()
    for _ in range(3):
        held = [torch.empty_strided(want.shape, want.stride(), dtype=BF, device="cuda"), torch.empty_like(grads),
                torch.empty(16 << 20, dtype=torch.uint8, device="cuda")]
        mine = [t.untyped_storage().data_ptr() for t in held]
        torch.cuda._sleep(20_000_000)                     # some ten milliseconds
        for t in held:
            t.fill_(1)
        del held, t
        y = tr.pg_linear(x, w, activation="gelu", stream=stream)
        dw = tr.pg_linear_weight_grad(want, x, stream=stream)
        assert y.untyped_storage().data_ptr() not in mine and dw.untyped_storage().data_ptr() not in mine
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(dw, grads)
    x2, w2 = x.clone(), w.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
    y = tr.pg_linear(x2, w2, activation="gelu", stream=stream)
    gone = [t.data_ptr() for t in (x2, w2)]
    del x2, w2
    over = [torch.full_like(x, float("nan")), torch.full_like(w, float("nan"))]
    assert not set(gone) & {t.data_ptr() for t in over}
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_the_default_stream_by_its_handle(tr):
    g = gen(15)
    x, w = rand(g, 2, 30, 64).to(BF), rand(g, 2, 48, 64).to(BF)
    want = tr.pg_linear(x, w)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = tr.pg_linear(x, w, stream=0)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("n", [1, 650, 1000, 1100, 4608, 16384])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
@pytest.mark.parametrize("residual,with8", [(False, False), (True, True)])
def test_norms_of_rows_whose_squares_leave_fp32(tr, n, eps, residual, with8):
    """bf16 reaches from 2^-133 to 2^128; the squares' sum does not fit fp32 at either end, the result always does."""
    g = gen(n)
    sizes = [3e38, 1e37, 2e19, 1e18, 1.0, 1e-12, 1e-18, 1e-20, 1e-30, 1e-36]
    v = (rand(g, 1, len(sizes), n) * 0.2).clamp(-0.99, 0.99)
    v[..., 0] = 0.5
    x = (v.double() * torch.tensor(sizes, device="cuda").double()[:, None]).to(BF)
    r = (x * 0.25) if residual else None
    x = x * 0.75 if residual else x
    gain = 1 + 0.3 * rand(g, 1, n)
    out = tr.pg_add_rms_norm(x, gain, residual=r, eps=eps, eight_bit=with8)
    s = x.double() + (r.double() if residual else 0.0)
    root = ((s * s).mean(-1) + float(torch.tensor(eps, dtype=torch.float32))) ** -0.5
    # as for other rows; a root below fp32's smallest normal number is held in steps of 2^-149, and so are sums of numbers that small
    check(out.rstd, root, root * (n + 40) * 2 * U + 2.0 ** -149)
    y = s * root[..., None] * gain.double()[:, None]
    slack = y.abs() * (n + 40) * 2 * U + 2.0 ** -149 * root[..., None] * gain.double()[:, None].abs()
    if with8:
        check8(out.y8, y, slack, BF)
    else:
        check(out.y, y, slack, BF)


@pytest.mark.parametrize("shape", [(3, 17, 33), (2, 33, 650), (2, 9, 1024), (1, 3, 4608), (1, 2, 16384)])
@pytest.mark.parametrize("dtype,pad", [(BF, 0), (HF, 1)])
def test_the_norms_checkpoint_is_that_of_its_stored_sum(tr, shape, dtype, pad):
    g = gen(hash(shape) % 1000 + 7)
    x, r = strided(rand(g, *shape, scale=2.0).to(dtype), pad), strided(rand(g, *shape).to(dtype), pad)
    if dtype == HF:
        x[0, 0, 0] = r[0, 0, 0] = 6e4                    # the sum has no place in fp16
    out = tr.pg_add_rms_norm(x, residual=r, save_h8=True)
    want = tr.pg_checkpoint_write(out.h)
    fine = want.scales != 255                            # a block that is not finite has no values
    assert torch.equal(out.h8.scales, want.scales)
    fine = fine.repeat_interleave(32, dim=-1)[..., :shape[-1]]
    assert torch.equal(out.h8.values[fine], want.values[fine])


@pytest.mark.parametrize("tokens", [512, 768, 769, 1024, 1025, 1500, 2048, 8192])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("from8", [False, True])
@pytest.mark.parametrize("sizes", [False, True])
def test_weight_gradients_are_within_a_millionth(tr, tokens, dtype, from8, sizes):
    """Of the gradient's size, for both types, at and beside the lengths at which a sum is put together from parts, for tokens
    alike and for tokens that differ in size; by enough workers for the parts not to be split over blocks, and by one."""
    g = gen(tokens)
    for b in (20, 1):
        def make(cols, scale):
            v = rand(g, b, tokens, cols, scale=scale)
            return (v * torch.exp(0.5 * rand(g, b, tokens, 1)) * torch.exp(0.5 * rand(g, 1, 1, cols)) if sizes else v).to(dtype)

        dz, x = make(512, 0.05), make(512, 1.0)
        kept = tr.pg_checkpoint_write(x) if from8 else x
        xv = stored8(kept) if from8 else x.double()
        want = dz.double().transpose(1, 2) @ xv
        assert float((tr.pg_linear_weight_grad(dz, kept).double() - want).norm() / want.norm()) <= 1e-6


def scale_bytes(top, dtype):
    """floor(log2(top)) - 6 with its bias, from the exponent itself: log2 of a power of two may come out under it."""
    e = torch.where(top > 0, torch.frexp(top)[1] - 7, torch.full_like(top, -1000).int())
    return e.clamp(min=LEAST[dtype]) + 127


def check8_half(c, want, slack, dtype):
    """An 8-bit result is the rounded one: within half a step of its block, of a whole one only where 127 is the limit, and the
    step is the one that a largest value within its slack has."""
    cols = want.shape[-1]
    step = torch.exp2(c.scales.double() - 127).repeat_interleave(32, dim=-1)[..., :cols]
    top, err = blocks_of(want).abs().amax(-1), blocks_of(slack).amax(-1)
    assert bool((c.scales >= scale_bytes(top - err, dtype)).all()) and bool((c.scales <= scale_bytes(top + err, dtype)).all())
    limit = slack + step * torch.where(c.values.abs() == 127, 1.0, 0.5)
    over = (stored8(c) - want).abs() - limit
    assert float(over.max()) <= 0.0, "off by %.3e more than allowed" % float(over.max())


@pytest.mark.parametrize("shape", [(3, 17, 33), (2, 33, 650), (2, 9, 1024), (1, 3, 4608)])
@pytest.mark.parametrize("dtype,pad", [(BF, 0), (HF, 1)])
def test_the_norms_8_bit_result_is_rounded_to_nearest(tr, shape, dtype, pad):
    g = gen(hash(shape) % 1000 + 8)
    b, t, n = shape
    x, gain = strided(rand(g, b, t, n, scale=2.0).to(dtype), pad), 1 + 0.3 * rand(g, b, n)
    out = tr.pg_add_rms_norm(x, gain, eight_bit=True)
    s = x.double()
    y = s * ((s * s).mean(-1, keepdim=True) + 1e-5) ** -0.5 * gain.double()[:, None]
    check8_half(out.y8, y, y.abs() * (n + 40) * 2 * U, dtype)


@pytest.mark.parametrize("shape", [(2, 1, 650, 260), (2, 33, 147, 65), (1, 64, 64, 128), (1, 257, 200, 129), (20, 200, 520, 700), (19, 385, 257, 513)])
@pytest.mark.parametrize("dtype,pad", [(BF, 0), (HF, 1)])
def test_the_layers_8_bit_result_is_rounded_to_nearest(tr, shape, dtype, pad):
    """One token, features as lanes, tokens as lanes; the slack is the exact sum's, so small integers have none."""
    g = gen(hash(shape) % 1000 + 9)
    b, t, k, n = shape
    x = strided(torch.randint(-4, 5, (b, t, k), device="cuda", generator=g).to(dtype), pad)
    w = strided((torch.randint(-4, 5, (b, n, k), device="cuda", generator=g) / 8).to(dtype), pad)
    bias = torch.randint(-40, 41, (b, n), device="cuda", generator=g) / 8.0
    _, z8 = tr.pg_linear(x, w, bias, save_z=True)
    z = x.double() @ w.double().transpose(1, 2) + bias.double()[:, None]       # multiples of 1/8 below 2^14: exact in fp32
    check8_half(z8, z, torch.zeros_like(z), dtype)
    byte = scale_bytes(blocks_of(z).abs().amax(-1), dtype)
    q = torch.round(blocks_of(z) * torch.exp2(127.0 - byte.double())[..., None]).clamp(-127, 127).flatten(-2)[..., :n]
    assert torch.equal(z8.scales.int(), byte) and torch.equal(z8.values.double(), q)


@pytest.mark.parametrize("tokens", [1, 2, 4, 5])
@pytest.mark.parametrize("k", [7, 63, 650, 5120, 5128, 10240, 20480, 20488])
@pytest.mark.parametrize("dtype,pad", [(BF, 0), (HF, 1), (BF, 2)])
def test_the_last_products_of_long_rows_count(tr, tokens, k, dtype, pad):
    """Only the last values of k are not zero, and small integers: any that is left out changes the sum, which is exact."""
    g = gen(tokens + k)
    for tail in (1, 3, 8, 16):
        x, w = torch.zeros(2, tokens, k, device="cuda"), torch.zeros(2, 45, k, device="cuda")
        x[..., -tail:] = torch.randint(1, 4, x[..., -tail:].shape, device="cuda", generator=g).float()
        w[..., -tail:] = torch.randint(1, 4, w[..., -tail:].shape, device="cuda", generator=g).float()
        y = tr.pg_linear(strided(x.to(dtype), pad), strided(w.to(dtype), pad))
        assert torch.equal(y.double(), x.double() @ w.double().transpose(1, 2))           # at most 144: exact in 16 bits
