"""Cases of the sequence operators: what a worker's language model needs beside its residual blocks.

As with the other training operators a leading axis of workers comes first, each worker with weights
of its own; a worker's tokens are `sequences` sequences of `length` tokens, one after another.

  norm       residual addition and layer norm (with mean and bias), output in 8 bits with scales; its backward pass
  conv       short causal convolution of every channel with SiLU; its backward pass
  scan       selective state space scan
                 D_t = softplus(delta_t + delta_bias)
                 h_t = exp(D_t A) h_{t-1} + D_t u_t B_t,   y_t = (C_t . h_t + skip u_t) silu(z_t)
             for whole sequences, for single tokens behind the convolution, and its backward pass
  loss       alpha tau^2 KL(teacher's top logits || student) at temperature tau + (1 - alpha) cross entropy of labels;
             its backward pass, alone or in one pass with the loss
"""
import math

import torch

own = False

BLOCK = 32
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
MOST_BYTES = 2.6e9                              # of the largest listed case, the language model's loss
MOST_STATES = 32.0 * 700 * 1300 * 16            # and of the largest scan: tokens x channels x states
MOST_LENGTH = 8192
EPS = 1e-5


def listed():
    def case(name, op, workers, sequences, length, cols, direction="forward", dtype="bf16", **more):
        c = {"name": name, "op": op, "direction": direction, "workers": workers, "sequences": sequences, "length": length, "cols": cols,
             "dtype": dtype, "residual": False, "eight": False, "width": 4, "states": 16, "gate": True, "carried": False, "ragged": False,
             "top": 0, "labels": False, "temperature": 1.0, "alpha": 1.0}
        c.update(more)
        return c

    return [
        # one token per worker while a model answers: latency of a single small call
        case("norm_token", "norm", 8, 1, 1, 650, residual=True),
        # 32 workers of the 650-wide language model, 20 sequences of 35 tokens each, output kept in 8 bits
        case("norm_lstm", "norm", 32, 20, 35, 650, residual=True, eight=True),
        # 64 workers of the torus, 1024-wide blocks, backward with the residual stream's gradient
        case("norm_grad_torus", "norm", 64, 1, 1024, 1024, "backward", residual=True),
        # the language model's inner width of 1300 in a training step, state carried from batch to batch
        case("conv_lstm", "conv", 32, 20, 35, 1300, carried=True),
        # backward through long sequences of unequal length, widths that are no multiple of eight
        case("conv_grad_long", "conv", 4, 3, 2049, 1029, "backward", dtype="fp16", width=3, ragged=True),
        # single tokens while models answer: convolution and scan of 4 sequences of 8 workers, states read and written
        case("scan_token", "step", 8, 4, 1, 1300, carried=True),
        # the scan of the training step
        case("scan_lstm", "scan", 32, 20, 35, 1300, carried=True),
        # one long prompt of one model
        case("scan_prompt", "scan", 1, 1, 8192, 1300, dtype="fp16"),
        # backward through the training step's scan, sequences of unequal length
        case("scan_grad_lstm", "scan", 32, 20, 35, 1300, "backward", ragged=True),
        # the loss of one sequence per worker on 28000 words, with its gradient, from the 8 best of a teacher
        case("loss_small", "loss", 8, 1, 35, 28000, "both", dtype="fp16", top=8, temperature=1.5),
        # the loss alone of a whole batch (evaluation)
        case("loss_lstm", "loss", 32, 20, 35, 28000, top=32, labels=True, temperature=2.0, alpha=0.7),
        # the training step's loss and gradient, logits read once
        case("loss_both_lstm", "loss", 32, 20, 35, 28000, "both", top=32, labels=True, temperature=2.0, alpha=0.7),
    ]


def draw(rng):
    """One more case: sizes spread over their logarithms, about half of the widths odd or ragged."""
    def size(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def width(lo, hi):
        n = size(lo, hi)
        return n if rng.random() < 0.5 else max(8, n // 8 * 8)

    while True:
        op = rng.choice(["norm", "norm", "conv", "conv", "scan", "scan", "scan", "step", "loss", "loss", "loss"])
        case = {"op": op, "direction": "forward", "workers": size(1, 64), "sequences": size(1, 32), "length": size(1, MOST_LENGTH), "cols": 0,
                "dtype": rng.choice(["bf16", "bf16", "fp16"]), "residual": False, "eight": False, "width": rng.choice([2, 3, 4, 4]),
                "states": 16, "gate": False, "carried": False, "ragged": False, "top": 0, "labels": False, "temperature": 1.0, "alpha": 1.0}
        if op == "norm":
            case["cols"] = width(16, 4608)
            case["direction"] = rng.choice(["forward", "backward"])
            case["residual"], case["eight"] = rng.random() < 0.5, rng.random() < 0.5
        elif op == "loss":
            case["cols"] = width(64, 50000)
            case["direction"] = rng.choice(["forward", "backward", "both"])
            case["labels"] = rng.random() < 0.6
            case["top"] = 0 if case["labels"] and rng.random() < 0.2 else min(size(1, 64), case["cols"])
            case["temperature"] = rng.choice([1.0, 2.0, round(rng.uniform(0.5, 5.0), 2)])
            case["alpha"] = 0.0 if case["top"] == 0 else 1.0 if not case["labels"] else round(rng.uniform(0.1, 0.9), 2)
        else:
            case["cols"] = width(16, 4608)
            case["states"] = rng.choice([16, 16, 16, 8, 32, size(1, 64)])
            case["gate"], case["carried"] = rng.random() < 0.5, rng.random() < 0.5
            if op == "step":
                case["length"], case["carried"] = 1, True
            else:
                case["direction"] = rng.choice(["forward", "backward"])
                case["ragged"] = rng.random() < 0.4
        w = work(case)
        rows = float(case["workers"]) * case["sequences"] * case["length"]
        if w["bytes"] <= MOST_BYTES and (op != "scan" or rows * case["cols"] * case["states"] <= MOST_STATES) \
                and (op in ("scan", "step", "loss") or w["bytes"] <= MOST_BYTES / 3):
            return case


def work(case):
    """Every input read once and every output written once."""
    op, b, s, k = case["op"], case["workers"], case["sequences"], case["cols"]
    t = float(b) * s * case["length"]
    row = t * k
    back = case["direction"] == "backward"
    eight = 1.0 + 1.0 / BLOCK
    if op == "norm":
        if back:
            return {"bytes": row * (4 + (eight if case["eight"] else 2) + (2 if case["residual"] else 0)) + 4.0 * b * 3 * k + 8 * t, "flops": 13 * row}
        return {"bytes": row * (2 * (4 if case["residual"] else 2) + (eight if case["eight"] else 0)) + 4.0 * b * 2 * k + 8 * t, "flops": 9 * row}
    if op == "loss":
        top = t * case["top"] * 6 + t * (4 if case["labels"] else 0)
        one = 10 if case["alpha"] in (0.0, 1.0) else 18
        return {"bytes": row * (2 if case["direction"] == "forward" else 4) + top + 4 * t * (3 if case["direction"] == "forward" else 4), "flops": one * row}
    w, n = case["width"], case["states"]
    held = float(b) * s * k
    conv = {"bytes": row * (6 if back else 4) + 4.0 * b * k * (w + 1) * (2 if back else 1)
            + (2 * held * (w - 1) * (1 if back else 2) if case["carried"] else 0), "flops": row * (6 * w + 12 if back else 2 * w + 6)}
    if op == "conv":
        return conv
    gate = 2 if case["gate"] else 0
    scan = {"bytes": row * ((10 + 2 * gate) if back else 6 + gate) + t * n * 2 * (4 if back else 2) + 4.0 * b * k * (n + 2) * (2 if back else 1)
            + (4 * held * n * (1 if back else 2) if case["carried"] else 0), "flops": row * n * (22 if back else 8)}
    if op == "scan":
        return scan
    return {"bytes": conv["bytes"] + scan["bytes"] - row * 4, "flops": conv["flops"] + scan["flops"]}


# ---------------------------------------------------------------- inputs
def _eight_parts(v, least):
    """(q, biased exponent) of the 8-bit form of fp32 values: blocks of 32 share a power of two; q has rows padded to 16 bytes."""
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
    g.manual_seed(seed * 7919 + 29)
    b, seqs, length, k, dt = case["workers"], case["sequences"], case["length"], case["cols"], DTYPES[case["dtype"]]
    t, n, back = seqs * length, case["states"], case["direction"] == "backward"
    least = -24 if case["dtype"] == "fp16" else -126

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, device="cuda", generator=g) * scale

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=g)

    def tokens(cols, scale=1.0):     # tokens differ in size, and a few features are large, as activations are
        return normal(b, t, cols, scale=scale) * torch.exp(0.5 * normal(b, t, 1)) * torch.exp(0.5 * normal(1, 1, cols))

    s = {"case": dict(case), "dt": dt, "least": least, "lengths": None}
    op = case["op"]
    if op == "norm":
        s["gain"], s["bias"] = 1.0 + 0.1 * normal(b, k), normal(b, k, scale=0.1)
        x = tokens(k) + 0.5 * normal(b, 1, k)
        if not back:
            s["x"], s["residual"] = x.to(dt), tokens(k).to(dt) if case["residual"] else None
        else:
            s["mean"] = x.mean(-1)
            s["rstd"] = torch.rsqrt((x - s["mean"].unsqueeze(-1)).square().mean(-1) + EPS)
            if case["eight"]:
                s["h_q"], s["h_e"] = _eight_parts(x.to(dt).float(), least)
            else:
                s["h"] = x.to(dt)
            s["dy"] = tokens(k, 0.05).to(dt)
            s["dh"] = tokens(k, 0.05).to(dt) if case["residual"] else None
        return s
    if op == "loss":
        x = torch.empty(b, t, k, dtype=dt, device="cuda")
        ids = torch.empty(b, t, case["top"], dtype=torch.int32, device="cuda") if case["top"] else None
        teacher = torch.empty(b, t, case["top"], dtype=dt, device="cuda") if case["top"] else None
        common = normal(k, scale=1.5)              # frequent words; student and teacher agree in part
        for i in range(b):
            logits = common + normal(t, k, scale=2.0)
            x[i] = logits.to(dt)
            if case["top"]:
                # the best of a teacher: its distribution over the classes drawn anew near the student's best ones
                v, at = torch.topk(logits + normal(t, k), case["top"], dim=-1)
                ids[i], teacher[i] = at.to(torch.int32), (1.3 * v).to(dt)
        s.update(x=x, ids=ids, teacher=teacher)
        s["labels"] = None
        if case["labels"]:
            y = (uniform(b, t) ** 3 * k).long().clamp(max=k - 1).to(torch.int32)
            s["labels"] = torch.where(uniform(b, t) < 0.05, torch.full_like(y, -100), y)       # padding carries no label
        if case["direction"] != "forward":         # the mean over tokens, scaled up for fp16
            s["dloss"] = (0.5 + uniform(b, t)) * (1024.0 if case["dtype"] == "fp16" else 1.0 / t)
        if back:
            s["lse"] = torch.stack([torch.stack([torch.logsumexp(row, -1), torch.logsumexp(row / case["temperature"], -1)], -1)
                                    for row in (r.float() for r in x)])
        return s
    if case["ragged"]:
        s["lengths"] = torch.randint(0, length + 1, (b, seqs), device="cuda", generator=g).to(torch.int32)
    if op in ("conv", "step"):
        s["x"] = tokens(k).to(dt)
        s["weight"], s["conv_bias"] = normal(b, k, case["width"], scale=case["width"] ** -0.5), normal(b, k, scale=0.1)
        s["conv_state"] = normal(b, seqs, case["width"] - 1, k).to(dt) if case["carried"] else None
    if op in ("scan", "step"):
        # (a step's scan reads inputs of its own too: the convolution's results in 16 bits would be other inputs on each side)
        u = normal(b, t, k)
        s["u"] = (u * torch.sigmoid(u) * 2).to(dt)
        s["delta"] = normal(b, t, k, scale=0.5).to(dt)
        step = torch.exp(uniform(b, k) * (math.log(0.1) - math.log(0.001)) + math.log(0.001))
        s["delta_bias"] = step + torch.log(-torch.expm1(-step))
        s["a"] = -torch.arange(1, n + 1, device="cuda").float() * torch.exp(0.1 * normal(b, k, n))
        s["b"], s["c"] = normal(b, t, n).to(dt), normal(b, t, n).to(dt)
        s["skip"] = 1.0 + 0.1 * normal(b, k)
        s["z"] = normal(b, t, k).to(dt) if case["gate"] else None
        s["state"] = normal(b, seqs, k, n, scale=0.3) if case["carried"] else None
    if back:
        s["dy"] = tokens(k, 0.05).to(dt)
    return s


# ---------------------------------------------------------------- plain forms
def _values(q, e):
    """fp32 values of an 8-bit form."""
    scale = torch.exp2(e.float() - 127.0)
    scale = torch.where(e == 255, torch.full_like(scale, float("nan")), scale)
    return q.float() * scale.repeat_interleave(BLOCK, dim=-1)[..., :q.shape[-1]]


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


def _sigmoid(v):
    return 1 / (1 + torch.exp(-v))


def _softplus(v):
    return v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))


def _valid(s):
    """(workers, sequences, length, 1): tokens that are there; None if all are."""
    if s["lengths"] is None:
        return None
    at = torch.arange(s["case"]["length"], device="cuda")
    return (at < s["lengths"].unsqueeze(-1)).unsqueeze(-1)


def _split(v, case):
    return v.unflatten(1, (case["sequences"], case["length"]))


def _conv_parts(s):
    """Inputs with the state before them, (workers, sequences, width - 1 + length, channels), and what tokens are there."""
    case, valid = s["case"], _valid(s)
    x = _split(s["x"].float(), case)
    if valid is not None:
        x = torch.where(valid, x, torch.zeros_like(x))
    if s["conv_state"] is None:
        before = torch.zeros_like(x[:, :, :1]).repeat(1, 1, case["width"] - 1, 1)
    else:
        before = s["conv_state"].float()
    return torch.cat([before, x], 2), valid


def _conv_z(s, line):
    case = s["case"]
    z = s["conv_bias"][:, None, None, :]
    for j in range(case["width"]):
        z = z + line[:, :, j:j + case["length"]] * s["weight"][:, None, None, :, j]
    return z


def _conv(s):
    case, dt = s["case"], s["dt"]
    line, valid = _conv_parts(s)
    z = _conv_z(s, line)
    y = z * _sigmoid(z)
    if valid is not None:
        y = torch.where(valid, y, torch.zeros_like(y))
    y = y.flatten(1, 2).to(dt)
    if not case["carried"]:
        return {"y": y}
    if s["lengths"] is None:
        return {"y": y, "conv_state": line[:, :, case["length"]:].to(dt)}
    at = s["lengths"].long()[:, :, None] + torch.arange(case["width"] - 1, device="cuda")
    return {"y": y, "conv_state": torch.gather(line, 2, at[..., None].expand(-1, -1, -1, case["cols"])).to(dt)}


def _conv_grad(s):
    case, dt = s["case"], s["dt"]
    line, valid = _conv_parts(s)
    z = _conv_z(s, line)
    sig = _sigmoid(z)
    dz = _split(s["dy"].float(), case) * sig * (1 + z * (1 - sig))
    if valid is not None:
        dz = torch.where(valid, dz, torch.zeros_like(dz))
    w, length = case["width"], case["length"]
    dline = torch.zeros_like(line)
    dweight = torch.empty_like(s["weight"])
    for j in range(w):
        dline[:, :, j:j + length] += dz * s["weight"][:, None, None, :, j]
        dweight[:, :, j] = (dz * line[:, :, j:j + length]).sum((1, 2))
    dx = dline[:, :, w - 1:]
    if valid is not None:
        dx = torch.where(valid, dx, torch.zeros_like(dx))
    return {"dx": dx.flatten(1, 2).to(dt), "dweight": dweight, "dbias": dz.sum((1, 2))}


def _scan_inputs(s):
    case, u = s["case"], s["u"]
    delta = _softplus(_split(s["delta"].float(), case) + s["delta_bias"][:, None, None, :])
    return delta, _split(u.float(), case), _split(s["b"].float(), case), _split(s["c"].float(), case), s["a"][:, None]


def _scan(s):
    case, valid = s["case"], _valid(s)
    delta, u, b, c, a = _scan_inputs(s)
    h = s["state"] if s["state"] is not None else torch.zeros(case["workers"], case["sequences"], case["cols"], case["states"], device="cuda")
    y = torch.empty_like(u)
    if valid is not None:
        delta = torch.where(valid, delta, torch.zeros_like(delta))      # nothing decays and nothing is added behind the end
        u, b = torch.where(valid, u, torch.zeros_like(u)), torch.where(valid, b, torch.zeros_like(b))
    drive = delta * u
    for t in range(case["length"]):
        h = torch.exp(delta[:, :, t, :, None] * a) * h + drive[:, :, t, :, None] * b[:, :, t, None, :]
        y[:, :, t] = (h * c[:, :, t, None, :]).sum(-1)
    y = y + s["skip"][:, None, None, :] * u
    if s["z"] is not None:
        z = _split(s["z"].float(), case)
        y = y * z * _sigmoid(z)
    if valid is not None:
        y = torch.where(valid, y, torch.zeros_like(y))
    y = y.flatten(1, 2).to(s["dt"])
    return {"y": y, "state": h} if case["carried"] else {"y": y}


def _scan_grad(s):
    case, valid, dt = s["case"], _valid(s), s["dt"]
    delta, u, b, c, a = _scan_inputs(s)
    dy = _split(s["dy"].float(), case)
    if valid is not None:
        delta, u, dy = (torch.where(valid, v, torch.zeros_like(v)) for v in (delta, u, dy))
        b, c = torch.where(valid, b, torch.zeros_like(b)), torch.where(valid, c, torch.zeros_like(c))
    h = s["state"] if s["state"] is not None else torch.zeros(case["workers"], case["sequences"], case["cols"], case["states"], device="cuda")
    length = case["length"]
    held = torch.empty(length + 1, *h.shape, device="cuda")
    held[0] = h
    inner = torch.empty_like(u)
    drive = delta * u
    for t in range(length):
        held[t + 1] = torch.exp(delta[:, :, t, :, None] * a) * held[t] + drive[:, :, t, :, None] * b[:, :, t, None, :]
        inner[:, :, t] = (held[t + 1] * c[:, :, t, None, :]).sum(-1)
    out = {}
    if s["z"] is not None:
        z = _split(s["z"].float(), case)
        sig = _sigmoid(z)
        dz = dy * (inner + s["skip"][:, None, None, :] * u) * sig * (1 + z * (1 - sig))
        if valid is not None:
            dz = torch.where(valid, dz, torch.zeros_like(dz))
        out["dz"] = dz.flatten(1, 2).to(dt)
        dy = dy * z * sig
        if valid is not None:
            dy = torch.where(valid, dy, torch.zeros_like(dy))
    du = dy * s["skip"][:, None, None, :]
    ddelta, db, dc = torch.empty_like(u), torch.empty_like(b), torch.empty_like(c)
    da, dh = torch.zeros_like(s["a"]), torch.zeros_like(h)
    for t in reversed(range(length)):
        keep = torch.exp(delta[:, :, t, :, None] * a)
        dh = dh + dy[:, :, t, :, None] * c[:, :, t, None, :]
        dc[:, :, t] = (dy[:, :, t, :, None] * held[t + 1]).sum(2)
        db[:, :, t] = (dh * drive[:, :, t, :, None]).sum(2)
        to_drive = (dh * b[:, :, t, None, :]).sum(-1)
        decay = dh * held[t] * keep
        du[:, :, t] += to_drive * delta[:, :, t]
        ddelta[:, :, t] = to_drive * u[:, :, t] + (decay * a).sum(-1)
        da += (decay * delta[:, :, t, :, None]).sum(1)
        dh = dh * keep
    raw = ddelta * _sigmoid(_split(s["delta"].float(), case) + s["delta_bias"][:, None, None, :])
    dskip = (dy * u).sum((1, 2))
    if valid is not None:
        raw, du = (torch.where(valid, v, torch.zeros_like(v)) for v in (raw, du))
    out.update(du=du.flatten(1, 2).to(dt), ddelta=raw.flatten(1, 2).to(dt), da=da, db=db.flatten(1, 2).to(dt), dc=dc.flatten(1, 2).to(dt),
               dskip=dskip, ddelta_bias=raw.sum((1, 2)))
    return out


def _norm(s):
    case, dt = s["case"], s["dt"]
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    mean = h.mean(-1)
    c = h - mean.unsqueeze(-1)
    rstd = torch.rsqrt((c * c).mean(-1) + EPS)
    y = c * rstd.unsqueeze(-1) * s["gain"].unsqueeze(1) + s["bias"].unsqueeze(1)
    y = (_rounded(y, s["least"]) if case["eight"] else y).to(dt)
    out = {"y": y, "mean": mean, "rstd": rstd}
    if case["residual"]:
        out["h"] = h.to(dt)
    return out


def _norm_grad(s):
    case, dt = s["case"], s["dt"]
    h = _values(s["h_q"], s["h_e"]) if case["eight"] else s["h"].float()
    dy, rstd = s["dy"].float(), s["rstd"].unsqueeze(-1)
    unit = (h - s["mean"].unsqueeze(-1)) * rstd
    a = dy * s["gain"].unsqueeze(1)
    dx = rstd * (a - a.mean(-1, keepdim=True) - unit * (a * unit).mean(-1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(dt), "dgain": (dy * unit).sum(1), "dbias": dy.sum(1)}


def _loss(s):
    """A worker at a time: its logits in 32 bits."""
    case, dt = s["case"], s["dt"]
    tau, alpha = case["temperature"], case["alpha"]
    hard = 1.0 - alpha if case["labels"] else 0.0
    soft = alpha if case["top"] else 0.0
    losses, grads, lses = [], [], []
    for i in range(case["workers"]):
        x = s["x"][i].float()
        loss = torch.zeros(x.shape[0], device="cuda")
        lse = [loss, loss]                          # of x and of x / tau; 0 where the loss does not need it
        grad = None
        dloss = None if case["direction"] == "forward" else s["dloss"][i].unsqueeze(-1)
        if soft:
            cold = x / tau
            top = cold.amax(-1, keepdim=True)
            e = torch.exp(cold - top)
            total = e.sum(-1, keepdim=True)
            at, want = s["ids"][i].long(), s["teacher"][i].float() / tau
            want = want - want.amax(-1, keepdim=True)
            we = torch.exp(want)
            p = we / we.sum(-1, keepdim=True)
            logq = torch.gather(cold, 1, at) - top - torch.log(total)
            lse[1] = (top + torch.log(total)).squeeze(-1)
            loss = loss + soft * tau * tau * (p * (want - torch.log(we.sum(-1, keepdim=True)) - logq)).sum(-1)
            if dloss is not None:
                grad = (e / total).scatter_add(1, at, -p) * (soft * tau * dloss)
        if hard:
            top = x.amax(-1, keepdim=True)
            e = torch.exp(x - top)
            total = e.sum(-1, keepdim=True)
            y = s["labels"][i].long().unsqueeze(-1)
            there = (y >= 0).float()
            y = y.clamp(min=0)
            lse[0] = (top + torch.log(total)).squeeze(-1)
            loss = loss + hard * (there * (top + torch.log(total) - torch.gather(x, 1, y))).squeeze(-1)
            if dloss is not None:
                g = (e / total).scatter_add(1, y, -torch.ones_like(there)) * (hard * there * dloss)
                grad = g if grad is None else grad + g
        losses.append(loss)
        lses.append(torch.stack(lse, -1))
        if grad is not None:
            grads.append(grad.to(dt))
    out = {} if case["direction"] == "backward" else {"loss": torch.stack(losses), "lse": torch.stack(lses)}
    if grads:
        out["dlogits"] = torch.stack(grads)
    return out


def _plain(s):
    case = s["case"]
    back = case["direction"] == "backward"
    if case["op"] == "norm":
        return _norm_grad(s) if back else _norm(s)
    if case["op"] == "conv":
        return _conv_grad(s) if back else _conv(s)
    if case["op"] == "scan":
        return _scan_grad(s) if back else _scan(s)
    if case["op"] == "step":
        out = _conv(s)
        out["u"] = out.pop("y")
        return {**out, **_scan(s)}
    return _loss(s)


# ---------------------------------------------------------------- the framework's calls
def _own(s):
    from paper_2008_01425_b200 import training as tr

    case, dt = s["case"], s["dt"]
    back = case["direction"] == "backward"
    seqs = {"sequences": case["sequences"], "lengths": s["lengths"]}
    if case["op"] == "norm":
        if back:
            h = tr.Checkpoint8(s["h_q"], s["h_e"], dt) if case["eight"] else s["h"]
            dx, dgain, dbias = tr.pg_add_layer_norm_grad(s["dy"], h, s["mean"], s["rstd"], s["gain"], dh=s["dh"])
            return {"dx": dx, "dgain": dgain, "dbias": dbias}
        n = tr.pg_add_layer_norm(s["x"], s["gain"], s["bias"], residual=s["residual"], eps=EPS, eight_bit=case["eight"])
        out = {"y": n.y, "mean": n.mean, "rstd": n.rstd}
        if case["residual"]:
            out["h"] = n.h
        return out
    if case["op"] == "loss":
        top = {"ids": s["ids"], "teacher": s["teacher"], "labels": s["labels"], "temperature": case["temperature"], "alpha": case["alpha"]}
        if back:
            return {"dlogits": tr.pg_distillation_loss_grad(s["dloss"], s["x"], s["lse"], **top)}
        r = tr.pg_distillation_loss(s["x"], dloss=s.get("dloss"), **top)
        return {"loss": r.loss, "lse": r.lse} if case["direction"] == "forward" else {"loss": r.loss, "lse": r.lse, "dlogits": r.dlogits}
    if case["op"] == "conv" and back:
        dx, dweight, dbias = tr.pg_causal_conv_grad(s["dy"], s["x"], s["weight"], s["conv_bias"], state=s["conv_state"], **seqs)
        return {"dx": dx, "dweight": dweight, "dbias": dbias}
    out = {}
    if case["op"] in ("conv", "step"):
        u = tr.pg_causal_conv(s["x"], s["weight"], s["conv_bias"], state=s["conv_state"], state_out=case["carried"], **seqs)
        if case["carried"]:
            u, out["conv_state"] = u
        if case["op"] == "conv":
            return {"y": u, **out}
        out["u"] = u
    if back:
        g = tr.pg_selective_scan_grad(s["dy"], s["u"], s["delta"], s["a"], s["b"], s["c"], s["skip"], s["delta_bias"], s["z"], state=s["state"], **seqs)
        out = {"du": g.du, "ddelta": g.ddelta, "da": g.da, "db": g.db, "dc": g.dc, "dskip": g.dskip, "ddelta_bias": g.ddelta_bias}
        if s["z"] is not None:
            out["dz"] = g.dz
        return out
    y = tr.pg_selective_scan(s["u"], s["delta"], s["a"], s["b"], s["c"], s["skip"], s["delta_bias"], s["z"], state=s["state"],
                             state_out=case["carried"], **seqs)
    if case["carried"]:
        y, out["state"] = y
    return {"y": y, **out}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- 64 bits
def _exact_conv(w, case, lengths):
    """Definition by a sum over taps, differentiable; (y, last inputs)."""
    f = torch.nn.functional
    b, q, length, k, taps = case["workers"], case["sequences"], case["length"], case["cols"], case["width"]
    x = w["x"].reshape(b, q, length, k)
    if lengths is not None:
        x = x.masked_fill(torch.arange(length, device="cuda")[None, None, :, None] >= lengths[:, :, None, None], 0.0)
    held = w.get("conv_state")
    line = f.pad(x, (0, 0, taps - 1, 0)) if held is None else torch.cat([held, x], 2)
    z = torch.einsum("bqtkj,bkj->bqtk", line.unfold(2, taps, 1), w["weight"]) + w["conv_bias"][:, None, None]
    y = z * torch.sigmoid(z)
    if lengths is not None:
        y = y.masked_fill(torch.arange(length, device="cuda")[None, None, :, None] >= lengths[:, :, None, None], 0.0)
        ends = lengths.long()
    else:
        ends = torch.full((b, q), length, device="cuda")
    last = torch.stack([line[torch.arange(b, device="cuda")[:, None], torch.arange(q, device="cuda")[None], ends + j] for j in range(taps - 1)], 2)
    return y.reshape(b, q * length, k), last


def _exact_scan(w, case, lengths):
    """Definition token by token, differentiable; (y, state)."""
    b, q, length, k, n = case["workers"], case["sequences"], case["length"], case["cols"], case["states"]
    shape = (b, q, length)
    step = torch.nn.functional.softplus(w["delta"] + w["delta_bias"][:, None], threshold=700.0).reshape(*shape, k)
    u = w["u"].reshape(*shape, k)
    bb, cc = w["b"].reshape(*shape, n), w["c"].reshape(*shape, n)
    h = w["state"] if "state" in w else torch.zeros(b, q, k, n, dtype=torch.float64, device="cuda")
    rows = []
    for t in range(length):
        new = torch.exp(torch.einsum("bqk,bkn->bqkn", step[:, :, t], w["a"])) * h
        new = new + torch.einsum("bqk,bqk,bqn->bqkn", step[:, :, t], u[:, :, t], bb[:, :, t])
        if lengths is not None:
            new = torch.where((t < lengths)[:, :, None, None], new, h)
        h = new
        rows.append(torch.einsum("bqkn,bqn->bqk", h, cc[:, :, t]))
    y = torch.stack(rows, 2) + w["skip"][:, None, None] * u
    if "z" in w:
        y = y * torch.nn.functional.silu(w["z"].reshape(*shape, k))
    if lengths is not None:
        y = y.masked_fill(torch.arange(length, device="cuda")[None, None, :, None] >= lengths[:, :, None, None], 0.0)
    return y.reshape(b, q * length, k), h


def exact(case, seed):
    """The operators' definitions in 64 bits.  Outputs held in 16 or 8 bits are given before that rounding."""
    s = prepare(case, seed)
    op, back = case["op"], case["direction"] == "backward"
    if op == "loss":
        return _exact_loss(case, s)
    wide = {key: v.double() for key, v in s.items() if isinstance(v, torch.Tensor) and key != "lengths"}
    if op == "norm":
        if not back:
            h = wide["x"] + wide.get("residual", 0.0)
            var, mean = torch.var_mean(h, -1, correction=0)
            root = (var + EPS) ** -0.5
            y = torch.einsum("btk,bt,bk->btk", h - mean[..., None], root, wide["gain"]) + wide["bias"][:, None]
            if case["eight"]:                       # y holds the values of its 8-bit form: whole steps, a power of two for each 32
                group = torch.arange(case["cols"], device="cuda") // BLOCK
                tops = torch.stack([v.abs().amax(-1) for v in y.split(BLOCK, dim=-1)], -1)
                step = torch.exp2((torch.floor(torch.log2(tops.clamp(min=1e-300))) - 6).clamp(min=s["least"]))[..., group]
                y = (y / step).round().clamp(-127, 127) * step
            out = {"y": y, "mean": mean, "rstd": root}
            return {**out, "h": h} if case["residual"] else out
        if case["eight"]:
            group = torch.arange(case["cols"], device="cuda") // BLOCK
            h = torch.ldexp(wide["h_q"], (wide["h_e"] - 127)[..., group])
        else:
            h = wide["h"]
        r, k = wide["rstd"], case["cols"]
        c = h - wide["mean"][..., None]
        a = torch.einsum("btk,bk->btk", wide["dy"], wide["gain"])
        dx = (a - a.sum(-1, keepdim=True) / k) * r[..., None] - c * (torch.einsum("btk,btk->bt", a, c) * r ** 3 / k)[..., None]
        return {"dx": dx + wide.get("dh", 0.0), "dgain": torch.einsum("btk,btk,bt->bk", wide["dy"], c, r), "dbias": wide["dy"].sum(1)}
    lengths = s["lengths"]
    if not back:
        out = {}
        if op in ("conv", "step"):
            y, last = _exact_conv(wide, case, lengths)
            if case["carried"]:
                out["conv_state"] = last
            if op == "conv":
                return {"y": y, **out}
            out["u"] = y
        y, h = _exact_scan(wide, case, lengths)
        if case["carried"]:
            out["state"] = h
        return {"y": y, **out}
    names = {"conv": {"x": "dx", "weight": "dweight", "conv_bias": "dbias"},
             "scan": {"u": "du", "delta": "ddelta", "a": "da", "b": "db", "c": "dc", "skip": "dskip", "delta_bias": "ddelta_bias", "z": "dz"}}[op]
    names = {key: v for key, v in names.items() if key in wide}
    for key in names:
        wide[key].requires_grad_(True)
    y, _ = (_exact_conv if op == "conv" else _exact_scan)(wide, case, lengths)
    if lengths is not None:
        there = (torch.arange(case["length"], device="cuda") < lengths[..., None]).flatten(1)
        wide["dy"] = wide["dy"].masked_fill(~there[..., None], 0.0)
    grads = torch.autograd.grad(y, [wide[key] for key in names], wide["dy"])
    return {name: g.detach() for name, g in zip(names.values(), grads)}


def _exact_loss(case, s):
    tau, alpha = case["temperature"], case["alpha"]
    losses, grads, lses = [], [], []
    for i in range(case["workers"]):
        x = s["x"][i].double()
        loss, g = 0.0, 0.0
        lse = torch.zeros(len(x), 2, dtype=torch.float64, device="cuda")
        if case["top"]:
            at = s["ids"][i].long()
            logp = torch.log_softmax(s["teacher"][i].double() / tau, -1)
            logq = torch.log_softmax(x / tau, -1)
            lse[:, 1] = torch.logsumexp(x / tau, -1)
            loss = loss + alpha * tau ** 2 * (logp.exp() * (logp - logq.gather(1, at))).sum(-1)
            if case["direction"] != "forward":
                g = g + alpha * tau * logq.exp().scatter_add(1, at, -logp.exp())
        if case["labels"] and alpha < 1:
            y = s["labels"][i].long()
            logq = torch.log_softmax(x, -1)
            lse[:, 0] = torch.logsumexp(x, -1)
            there = y >= 0
            loss = loss - (1 - alpha) * torch.where(there, logq.gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
            if case["direction"] != "forward":
                q = logq.exp()
                q[torch.arange(len(y), device="cuda"), y.clamp(min=0)] -= 1.0
                g = g + (1 - alpha) * q * there[:, None]
        losses.append(loss)
        lses.append(lse)
        if case["direction"] != "forward":
            grads.append(g * s["dloss"][i].double()[:, None])
    out = {} if case["direction"] == "backward" else {"loss": torch.stack(losses), "lse": torch.stack(lses)}
    if grads:
        out["dlogits"] = torch.stack(grads)
    return out
