"""Cases of the training operators: what one worker's residual block needs around a gossip round.

The library simulates the decentralized training of many workers on one GPU, so every operator
takes a leading axis of workers, each with weights of its own:

  norm             residual addition, root-mean-square norm, output in 8 bits with scales
  norm_grad        its backward pass, from the sum as it was stored or from its 8-bit checkpoint
  linear           x W^T + bias, activation, residual; the pre-activation kept as an 8-bit checkpoint
  input_grad       dz W, the gradient of the residual path added
  weight_grad      dz^T x into fp32, x a 16-bit tensor or an 8-bit checkpoint
  activation_grad  dy * act'(z) and the bias gradient, z an 8-bit checkpoint
  checkpoint       a 16-bit tensor to its 8-bit form and back

8-bit form: blocks of 32 values along a row share one power of two 2^e, e = floor(log2(max |v|)) - 6,
and every value is kept as q = round(v / 2^e) in -127..127.  e is held with a bias of 127, is at
least -126 (-24 for fp16, whose own step that is), and 255 marks a block that held a NaN or an
infinity: all of it reads back as NaN.
"""
import math

import torch

own = False

BLOCK = 32
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
MOST_FLOPS = 2.0 * 64 * 2048 * 1024 * 1024     # the largest listed products
MOST_BYTES = 9.0e8
EPS = 1e-5


def listed():
    def case(name, op, workers, tokens, inner, outer=0, dtype="bf16", activation="none", residual=False, eight=False):
        return {"name": name, "op": op, "workers": workers, "tokens": tokens, "inner": inner, "outer": outer, "dtype": dtype,
                "activation": activation, "residual": residual, "eight": eight}

    return [
        # one token per worker while a model answers: latency of a single small call
        case("norm_token", "norm", 8, 1, 650, residual=True),
        # 32 workers of the 650-wide language model, 20 sequences of 35 tokens each
        case("norm_lstm", "norm", 32, 700, 650, residual=True, eight=True),
        # 64 workers of the torus, 1024-wide blocks, backward with the residual stream's gradient
        case("norm_grad_torus", "norm_grad", 64, 1024, 1024, residual=True),
        # one token per worker through the widening layer: every worker's weights are read for one row
        case("linear_token", "linear", 32, 1, 650, 2600, activation="gelu"),
        # the same layer in a training step: activation, and the pre-activation kept in 8 bits
        case("linear_lstm", "linear", 32, 700, 650, 2600, activation="gelu", eight=True),
        # the largest: square layers of 64 workers on 2048 tokens each, with the residual path
        case("linear_torus", "linear", 64, 2048, 1024, 1024, activation="silu", residual=True),
        # a first layer on 3 x 7 x 7 patches: rows of 147 values are not 16-byte aligned, nothing is a tile
        case("linear_ragged", "linear", 8, 1037, 147, 65, dtype="fp16", activation="relu"),
        # gradient through the widening layer, back to 650 columns
        case("input_grad_lstm", "input_grad", 32, 700, 650, 2600, residual=True),
        # weight gradients from 8-bit activations, language-model layer and torus layer
        case("weight_grad_lstm", "weight_grad", 32, 700, 650, 2600, eight=True),
        case("weight_grad_torus", "weight_grad", 64, 2048, 1024, 1024, eight=True),
        # activation's backward pass from the 8-bit pre-activation, with the bias gradient
        case("activation_grad_lstm", "activation_grad", 32, 700, 2600, activation="gelu", eight=True),
        # checkpoint of a small layer of the 16-worker ring, written and read back
        case("checkpoint_ring", "checkpoint", 16, 128, 512, dtype="fp16", eight=True),
    ]


def draw(rng):
    """One more case: sizes spread over their logarithms, about half of the widths odd or ragged."""
    def size(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def width():
        n = size(16, 4608)
        return n if rng.random() < 0.5 else max(16, n // 8 * 8)

    while True:
        op = rng.choice(["norm", "norm_grad", "linear", "linear", "input_grad", "weight_grad", "activation_grad", "checkpoint"])
        product = op in ("linear", "input_grad", "weight_grad")
        case = {"op": op, "workers": size(1, 64), "tokens": size(1, 4096), "inner": width(), "outer": width() if product else 0,
                "dtype": rng.choice(["bf16", "bf16", "fp16"]), "activation": "none", "residual": False, "eight": False}
        if op in ("linear", "activation_grad"):
            case["activation"] = rng.choice(["none", "relu", "gelu", "silu"])
        if op in ("norm", "norm_grad", "linear", "input_grad"):
            case["residual"] = rng.random() < 0.5
        case["eight"] = op in ("activation_grad", "checkpoint") or (op != "input_grad" and rng.random() < 0.5)
        w = work(case)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return case


def work(case):
    """Every input read once and every output written once; two operations for a product's multiply and add."""
    op, b, t, k, n = case["op"], case["workers"], case["tokens"], case["inner"], case["outer"]
    eight = 1.0 + 1.0 / BLOCK
    row = float(b) * t * k
    if op == "norm":
        return {"bytes": row * (2 * (4 if case["residual"] else 2) + (eight if case["eight"] else 0)) + 4.0 * b * (k + t), "flops": 6 * row}
    if op == "norm_grad":
        return {"bytes": row * (4 + (eight if case["eight"] else 2) + (2 if case["residual"] else 0)) + 4.0 * b * (2 * k + t), "flops": 10 * row}
    if op == "activation_grad":
        return {"bytes": row * (4 + eight) + 4.0 * b * k, "flops": 16 * row}
    if op == "checkpoint":
        return {"bytes": row * (2 + 2 * eight + 2), "flops": 4 * row}
    flops = 2.0 * b * t * k * n
    x, y, w = float(b) * t * k, float(b) * t * n, float(b) * k * n
    if op == "linear":
        return {"bytes": 2 * (x + w) + y * (2 + (2 if case["residual"] else 0) + (eight if case["eight"] else 0)) + 4.0 * b * n, "flops": flops}
    if op == "input_grad":
        return {"bytes": 2 * (y + w) + x * (2 + (2 if case["residual"] else 0)), "flops": flops}
    return {"bytes": 2 * y + x * (eight if case["eight"] else 2) + 4 * w, "flops": flops}


# ---------------------------------------------------------------- inputs
def _eight_parts(v, least):
    """(q, biased exponent) of the 8-bit form of fp32 values; q has rows padded to 16 bytes."""
    cols = v.shape[-1]
    blocks = -(-cols // BLOCK)
    p = torch.nn.functional.pad(v, (0, blocks * BLOCK - cols)).unflatten(-1, (blocks, BLOCK))
    top = p.abs().amax(-1)
    e = (torch.frexp(top)[1] - 7).clamp(min=least)
    e = torch.where(top > 0, e, torch.full_like(e, least))
    q = torch.round(torch.ldexp(p, -e.unsqueeze(-1))).clamp(-127, 127)
    q = q.flatten(-2)[..., :cols].to(torch.int8)
    held = torch.zeros(*v.shape[:-1], -(-cols // 16) * 16, dtype=torch.int8, device=v.device)
    held[..., :cols] = q
    return held[..., :cols], (e + 127).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 13)
    b, t, k, n, dt = case["workers"], case["tokens"], case["inner"], case["outer"], DTYPES[case["dtype"]]
    least = -24 if case["dtype"] == "fp16" else -126

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, device="cuda", generator=g) * scale

    def tokens(cols, scale=1.0):     # tokens differ in size, and a few features are large, as activations are
        v = normal(b, t, cols, scale=scale) * torch.exp(0.5 * normal(b, t, 1))
        return v * torch.exp(0.5 * normal(1, 1, cols))

    s = {"case": dict(case), "dt": dt, "least": least}
    op = case["op"]
    if op in ("norm", "norm_grad"):
        s["gain"] = 1.0 + 0.1 * normal(b, k)
    if op == "norm":
        s["x"] = tokens(k).to(dt)
        s["residual"] = tokens(k).to(dt) if case["residual"] else None
    elif op == "norm_grad":
        h = tokens(k)
        s["rstd"] = torch.rsqrt(h.square().mean(-1) + EPS)
        if case["eight"]:
            s["h_q"], s["h_e"] = _eight_parts(h.to(dt).float(), least)
        else:
            s["h"] = h.to(dt)
        s["dy"] = tokens(k, 0.05).to(dt)
        s["dh"] = tokens(k, 0.05).to(dt) if case["residual"] else None
    elif op == "linear":
        s["x"] = tokens(k).to(dt)
        s["weight"] = normal(b, n, k, scale=k ** -0.5).to(dt)
        s["bias"] = normal(b, n, scale=0.1)
        s["residual"] = tokens(n).to(dt) if case["residual"] else None
    elif op == "input_grad":
        s["dz"] = tokens(n, 0.05).to(dt)
        s["weight"] = normal(b, n, k, scale=k ** -0.5).to(dt)
        s["dres"] = tokens(k, 0.05).to(dt) if case["residual"] else None
    elif op == "weight_grad":
        s["dz"] = tokens(n, 0.05).to(dt)
        x = tokens(k).to(dt)
        if case["eight"]:
            s["x_q"], s["x_e"] = _eight_parts(x.float(), least)
        else:
            s["x"] = x
    elif op == "activation_grad":
        s["dy"] = tokens(k, 0.05).to(dt)
        s["z_q"], s["z_e"] = _eight_parts(tokens(k), least)
    else:
        s["x"] = tokens(k).to(dt)
    return s


# ---------------------------------------------------------------- plain forms
def _values(q, e):
    """fp32 values of an 8-bit form."""
    cols = q.shape[-1]
    scale = torch.exp2(e.float() - 127.0)
    scale = torch.where(e == 255, torch.full_like(scale, float("nan")), scale)
    return q.float() * scale.repeat_interleave(BLOCK, dim=-1)[..., :cols]


def _rounded(v, least):
    """fp32 values of the 8-bit form of v, with blocks that are not finite read back as NaN."""
    cols = v.shape[-1]
    blocks = -(-cols // BLOCK)
    p = torch.nn.functional.pad(v, (0, blocks * BLOCK - cols)).unflatten(-1, (blocks, BLOCK))
    top = p.abs().amax(-1, keepdim=True)
    e = (torch.frexp(top)[1] - 7).clamp(min=least)
    e = torch.where(top > 0, e, torch.full_like(e, least))
    q = torch.ldexp(torch.round(torch.ldexp(p, -e)).clamp(-127, 127), e)
    return torch.where(torch.isfinite(top), q, torch.full_like(q, float("nan"))).flatten(-2)[..., :cols]


def _act(z, kind):
    if kind == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if kind == "gelu":
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z / (1 + torch.exp(-z)) if kind == "silu" else z


def _act_grad(z, kind):
    if kind == "relu":
        return (z > 0).float()
    if kind == "gelu":
        c = math.sqrt(2 / math.pi)
        s = 1 / (1 + torch.exp(-2 * c * (z + 0.044715 * z * z * z)))
        return s + z * s * (1 - s) * 2 * c * (1 + 3 * 0.044715 * z * z)
    if kind == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _plain(s):
    case, dt, least = s["case"], s["dt"], s["least"]
    op = case["op"]
    if op == "norm":
        h = s["x"].float()
        if s["residual"] is not None:
            h = h + s["residual"].float()
        rstd = torch.rsqrt((h * h).mean(-1) + EPS)
        y = h * rstd.unsqueeze(-1) * s["gain"].unsqueeze(1)
        y = (_rounded(y, least) if case["eight"] else y).to(dt)
        return {"h": h.to(dt), "y": y, "rstd": rstd} if case["residual"] else {"y": y, "rstd": rstd}
    if op == "norm_grad":
        h = _values(s["h_q"], s["h_e"]) if case["eight"] else s["h"].float()
        dy, rstd = s["dy"].float(), s["rstd"].unsqueeze(-1)
        unit = h * rstd
        a = dy * s["gain"].unsqueeze(1)
        dx = rstd * (a - unit * (a * unit).mean(-1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(dt), "dgain": (dy * unit).sum(1)}
    if op == "linear":
        z = torch.matmul(s["x"].float(), s["weight"].float().transpose(1, 2)) + s["bias"].unsqueeze(1)
        y = _act(z, case["activation"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return {"y": y.to(dt), "z": _rounded(z, least).to(dt)} if case["eight"] else {"y": y.to(dt)}
    if op == "input_grad":
        dx = torch.matmul(s["dz"].float(), s["weight"].float())
        if s["dres"] is not None:
            dx = dx + s["dres"].float()
        return {"dx": dx.to(dt)}
    if op == "weight_grad":
        x = _values(s["x_q"], s["x_e"]) if case["eight"] else s["x"].float()
        return {"dweight": torch.matmul(s["dz"].float().transpose(1, 2), x)}
    if op == "activation_grad":
        dz = s["dy"].float() * _act_grad(_values(s["z_q"], s["z_e"]), case["activation"])
        return {"dz": dz.to(dt), "dbias": dz.sum(1)}
    return {"x": _rounded(s["x"].float(), least).to(dt)}


# ---------------------------------------------------------------- the framework's calls
def _own(s):
    from paper_2008_01425_b200 import training as tr

    case, dt = s["case"], s["dt"]
    op = case["op"]
    if op == "norm":
        out = tr.pg_add_rms_norm(s["x"], s["gain"], residual=s["residual"], eps=EPS, eight_bit=case["eight"])
        return {"h": out.h, "y": out.y, "rstd": out.rstd} if case["residual"] else {"y": out.y, "rstd": out.rstd}
    if op == "norm_grad":
        h = tr.Checkpoint8(s["h_q"], s["h_e"], dt) if case["eight"] else s["h"]
        dx, dgain = tr.pg_add_rms_norm_grad(s["dy"], h, s["rstd"], s["gain"], dh=s["dh"])
        return {"dx": dx, "dgain": dgain}
    if op == "linear":
        if not case["eight"]:
            return {"y": tr.pg_linear(s["x"], s["weight"], s["bias"], activation=case["activation"], residual=s["residual"])}
        y, z8 = tr.pg_linear(s["x"], s["weight"], s["bias"], activation=case["activation"], residual=s["residual"], save_z=True)
        return {"y": y, "z": tr.pg_checkpoint_read(z8)}
    if op == "input_grad":
        return {"dx": tr.pg_linear_input_grad(s["dz"], s["weight"], residual=s["dres"])}
    if op == "weight_grad":
        x = tr.Checkpoint8(s["x_q"], s["x_e"], dt) if case["eight"] else s["x"]
        return {"dweight": tr.pg_linear_weight_grad(s["dz"], x)}
    if op == "activation_grad":
        dz, dbias = tr.pg_activation_grad(s["dy"], tr.Checkpoint8(s["z_q"], s["z_e"], dt), case["activation"])
        return {"dz": dz, "dbias": dbias}
    return {"x": tr.pg_checkpoint_read(tr.pg_checkpoint_write(s["x"]))}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    """The operators' definitions in 64 bits.  Outputs held in 16 or 8 bits are given before that rounding."""
    s = prepare(case, seed)
    wide = {key: v.double() for key, v in s.items() if isinstance(v, torch.Tensor)}

    def stored(q, e):
        group = torch.arange(q.shape[-1], device="cuda") // BLOCK
        return torch.ldexp(q, (e - 127)[..., group])

    def slope(z, kind):
        if kind == "gelu":
            c, a = math.sqrt(2 / math.pi), 0.044715
            th = torch.tanh(c * (z + a * z ** 3))
            return 0.5 * (1 + th) + 0.5 * z * (1 - th ** 2) * c * (1 + 3 * a * z ** 2)
        if kind == "silu":
            return torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
        return (z > 0).double() if kind == "relu" else torch.ones_like(z)

    op = case["op"]
    if op == "norm":
        h = wide["x"] + wide.get("residual", 0.0)
        root = ((h ** 2).sum(-1) / case["inner"] + EPS) ** -0.5
        y = torch.einsum("btk,bt,bk->btk", h, root, wide["gain"])
        return {"h": h, "y": y, "rstd": root} if case["residual"] else {"y": y, "rstd": root}
    if op == "norm_grad":
        h = stored(wide["h_q"], wide["h_e"]) if case["eight"] else wide["h"]
        r = wide["rstd"]
        a = torch.einsum("btk,bk->btk", wide["dy"], wide["gain"])
        dot = torch.einsum("btk,btk->bt", a, h) * r ** 3 / case["inner"]
        dx = a * r[..., None] - h * dot[..., None] + wide.get("dh", 0.0)
        return {"dx": dx, "dgain": torch.einsum("btk,btk,bt->bk", wide["dy"], h, r)}
    if op == "linear":
        z = torch.einsum("btk,bnk->btn", wide["x"], wide["weight"]) + wide["bias"][:, None]
        kind = case["activation"]
        if kind == "gelu":
            y = 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
        else:
            y = z * torch.sigmoid(z) if kind == "silu" else z.clamp(min=0) if kind == "relu" else z
        y = y + wide.get("residual", 0.0)
        return {"y": y, "z": z} if case["eight"] else {"y": y}
    if op == "input_grad":
        return {"dx": torch.einsum("btn,bnk->btk", wide["dz"], wide["weight"]) + wide.get("dres", 0.0)}
    if op == "weight_grad":
        x = stored(wide["x_q"], wide["x_e"]) if case["eight"] else wide["x"]
        return {"dweight": torch.einsum("btn,btk->bnk", wide["dz"], x)}
    if op == "activation_grad":
        dz = wide["dy"] * slope(stored(wide["z_q"], wide["z_e"]), case["activation"])
        return {"dz": dz, "dbias": dz.sum(1)}
    return {"x": wide["x"]}
