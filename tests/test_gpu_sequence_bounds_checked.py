"""The sequence operators in the bounds-checked build (-DPG_BOUNDS_CHECK): every address that their kernels compute is looked up in the
operands of the call.  Ragged widths, rows that start anywhere, one token to thousands, sequences without tokens, chunked scans, rows
of logits that shared memory does not hold: no access may lie outside, and the results must be the bits that the regular build gives."""
import json
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import hashlib, json, sys
sys.path.insert(0, %(root)r)
import torch
from paper_2008_01425_b200 import training as tr
from tests.test_gpu_sequence_bounds_checked import cases, outputs

out = {}
for case in cases():
    h = hashlib.sha256()
    for t in outputs(tr, *case):
        t = t.contiguous()
        h.update(t.view(torch.uint8).cpu().numpy().tobytes() if t.numel() else b"-")
    out[str(case)] = [tr.pg_training_status(), h.hexdigest()]
print("RESULT " + json.dumps(out))
"""

# workers, sequences, length, channels, states, classes
SHAPES = [(1, 1, 1, 1, 1, 1), (2, 3, 5, 7, 3, 33), (2, 1, 70, 64, 16, 1000), (3, 4, 9, 65, 8, 1029), (1, 2, 200, 130, 33, 4099), (8, 4, 1, 300, 16, 8200), (1, 1, 700, 33, 16, 28001),
          (2, 2, 41, 1300, 16, 9000), (1, 1, 2100, 5, 64, 300), (1, 3, 3, 257, 17, 110001)]


def cases():
    """(workers, sequences, length, channels, states, classes, pad of the rows, type)"""
    for i, shape in enumerate(SHAPES):
        for pad in (0, 1, 8):
            yield shape + (pad, "float16" if (i + pad) % 2 else "bfloat16")


def outputs(tr, b, s, length, n, m, classes, pad, dtype):
    """Everything that the operators make of one set of inputs.  Inputs and outputs end with their last row."""
    import torch

    dtype = getattr(torch, dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(b * 7 + s * 5 + length * 3 + n + pad)
    t = s * length

    def make(*shape, scale=1.0, kind=None):
        big = torch.zeros(*shape[:-1], shape[-1] + pad, device="cuda", dtype=kind or dtype)
        v = big[..., :shape[-1]]
        v.copy_(torch.randn(*shape, device="cuda", generator=g) * scale)
        return v

    def flat(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    x, r, gain, bias = make(b, t, n), make(b, t, n), flat(b, n), flat(b, n)
    norm = tr.pg_add_layer_norm(x, gain, bias, residual=r, eight_bit=True, save_h8=True, out=make(b, t, n))
    yield from (norm.h, norm.y, norm.mean, norm.rstd, norm.y8.values, norm.y8.scales, norm.h8.values, norm.h8.scales)
    for h in (norm.h, norm.h8):
        yield from tr.pg_add_layer_norm_grad(x, h, norm.mean, norm.rstd, gain, dh=r, out=make(b, t, n))
    lengths = torch.randint(0, length + 1, (b, s), device="cuda", generator=g).to(torch.int32)
    for taps, which in ((2, None), (3, lengths), (4, lengths)):
        w, state = make(b, n, taps, kind=torch.float32), flat(b, s, taps - 1, n).to(dtype)
        yield from tr.pg_causal_conv(x, w, bias, sequences=s, lengths=which, state=state, state_out=True, out=make(b, t, n))
        yield from tr.pg_causal_conv_grad(r, x, w, bias, sequences=s, lengths=which, state=state, out=make(b, t, n), weight_grad=make(b, n, taps, kind=torch.float32),
                                          bias_grad=flat(b, n), accumulate=True)
    a, bb, cc, z = -torch.exp(make(b, n, m, kind=torch.float32)), make(b, t, m), make(b, t, m), make(b, t, n)
    state = flat(b, s, n, m)
    for gate, held, which in ((z, state, lengths), (None, None, None)):
        y, last = tr.pg_selective_scan(x, r, a, bb, cc, gain, bias, gate, sequences=s, lengths=which, state=held, state_out=True, out=make(b, t, n))
        yield from (y, last)
        yield from (v for v in tr.pg_selective_scan_grad(z, x, r, a, bb, cc, gain, bias, gate, sequences=s, lengths=which, state=held) if v is not None)
    rows = min(t, 40)
    logits = make(b, rows, classes, scale=3.0)
    if n % 2:                                          # rows for every warp of the GPU, the last ones at the end of their allocation
        many = make(1, 4700, min(classes, 1500))
        yield tr.pg_distillation_loss(many, labels=torch.zeros(1, 4700, dtype=torch.int32, device="cuda"), alpha=0.0).loss
    ids = torch.randint(-1, classes + 1, (b, rows, 5), device="cuda", generator=g).to(torch.int32)
    labels = torch.randint(-1, classes + 1, (b, rows), device="cuda", generator=g).to(torch.int32)
    teacher, dloss = make(b, rows, 5), flat(b, rows)
    for tau, alpha in ((1.0, 0.5), (2.0, 0.5), (1.3, 0.5), (4.0, 1.0)):
        kw = dict(ids=ids, teacher=teacher, labels=labels, temperature=tau, alpha=alpha)
        yield tr.pg_distillation_loss(logits, **kw).loss
        q = tr.pg_distillation_loss(logits, dloss=dloss, **kw)
        yield from q
        yield tr.pg_distillation_loss(logits, dloss=dloss, out=make(b, rows, classes), **kw).dlogits
        yield tr.pg_distillation_loss_grad(dloss, logits, q.lse, out=make(b, rows, classes), **kw)


def _run_child(library):
    env = dict(os.environ)
    env.pop("PG_LIBRARY", None)
    if library:
        env["PG_LIBRARY"] = library
    r = subprocess.run([sys.executable, "-c", CHILD % {"root": ROOT}], cwd=ROOT, env=env, stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, timeout=600)
    text = r.stdout.decode()
    assert r.returncode == 0, text[-3000:]
    line = [l for l in text.splitlines() if l.startswith("RESULT ")][-1]
    return json.loads(line[len("RESULT "):])


def test_checked_sequence_kernels_stay_inside_their_operands():
    from paper_2008_01425_b200 import binding as pg
    from paper_2008_01425_b200 import build as pg_build

    got, want = _run_child(pg_build.build(checked=True)), _run_child(None)
    assert sorted(got) == sorted(want) and len(got) == 3 * len(SHAPES)
    for name in sorted(got):
        assert got[name][0] == pg.PG_OK, "%s: status %d in the checked build" % (name, got[name][0])
        assert want[name][0] == pg.PG_OK
        assert got[name][1] == want[name][1], "%s: the checked build gives other bits" % name
