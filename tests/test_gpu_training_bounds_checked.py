"""The training operators in the bounds-checked build (-DPG_BOUNDS_CHECK): every address that their kernels compute is looked
up in the operands of the call.  Ragged widths, rows that start anywhere, one token to thousands, single blocks, split sums and
pairs of blocks (with a second block behind the last row too): no access may lie outside, and the results must be the bits
that the regular build gives."""
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
from tests.test_gpu_training_bounds_checked import cases, outputs

out = {}
for case in cases():
    h = hashlib.sha256()
    for t in outputs(tr, *case):
        t = t.contiguous()
        h.update(t.view(torch.uint8).cpu().numpy().tobytes() if t.numel() else b"-")
    out[str(case)] = [tr.pg_training_status(), h.hexdigest()]
out["__probe__"] = [tr.pg_selftest_training_bounds(), ""]
print("RESULT " + json.dumps(out))
"""

SHAPES = [(1, 1, 1, 1), (2, 1, 650, 260), (3, 4, 147, 65), (2, 33, 147, 65), (2, 130, 72, 136), (5, 40, 650, 96), (1, 300, 512, 520),
          (1, 1040, 64, 24), (40, 3, 24, 40), (1, 2500, 200, 136), (2, 513, 328, 2600),
          # pairs of blocks; features in the first half of a last pair's 256, and in both
          (19, 385, 257, 513), (37, 7, 300, 200), (38, 129, 384, 33), (20, 200, 640, 700), (12, 1100, 896, 264), (5, 300, 650, 1000)]


def cases():
    """(workers, tokens, in, out, pad of the rows, type)"""
    for i, shape in enumerate(SHAPES):
        for pad in (0, 1, 8):
            yield shape + (pad, "float16" if (i + pad) % 2 else "bfloat16")
    for cols in (31, 1000, 1024, 2600, 4612, 9000, 16384):
        yield (2, 9, cols, 0, cols % 3, "bfloat16")


def outputs(tr, b, t, k, n, pad, dtype):
    """Everything that the operators make of one set of inputs.  Inputs and outputs end with their last row."""
    import torch

    dtype = getattr(torch, dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(b * 7 + t * 5 + k * 3 + n + pad)

    def make(*shape, scale=1.0, kind=None):
        big = torch.zeros(*shape[:-1], shape[-1] + pad, device="cuda", dtype=kind or dtype)
        v = big[..., :shape[-1]]
        v.copy_(torch.randn(*shape, device="cuda", generator=g) * scale)
        return v

    def flat(c):
        cols = c.values.shape[-1]
        return [torch.where((c.scales == 255).repeat_interleave(32, dim=-1)[..., :cols], 0, c.values), c.scales]

    x, r, gain = make(b, t, k), make(b, t, k), make(b, k, kind=torch.float32)
    norm = tr.pg_add_rms_norm(x, gain, residual=r, eight_bit=True, save_h8=True, out=make(b, t, k))
    yield from (norm.h, norm.y, norm.rstd, *flat(norm.y8), *flat(norm.h8))
    yield tr.pg_add_rms_norm(x).y
    for h in (norm.h, norm.h8):
        yield from tr.pg_add_rms_norm_grad(x, h, norm.rstd, gain, dh=r, out=make(b, t, k))
    x8 = tr.pg_checkpoint_write(x)
    yield from flat(x8)
    yield tr.pg_checkpoint_read(x8, out=make(b, t, k))
    for kind in ("none", "relu", "gelu", "silu"):
        yield from tr.pg_activation_grad(r, x8, kind, out=make(b, t, k))
    if n == 0:
        return
    w, bias = make(b, n, k, scale=k ** -0.5), make(b, n, kind=torch.float32)
    res = make(b, t, n)
    y, z8 = tr.pg_linear(x, w, bias, residual=res, activation="gelu", save_z=True)
    yield from (y, *flat(z8))
    yield tr.pg_linear(x, w, out=make(b, t, n))
    yield tr.pg_linear_input_grad(res, w, residual=x)
    yield tr.pg_linear_input_grad(res, w, out=make(b, t, k))
    for kept in (x, x8):
        yield tr.pg_linear_weight_grad(res, kept)
        yield tr.pg_linear_weight_grad(res, kept, out=make(b, n, k, kind=torch.float32), accumulate=True)


def _run_child(library):
    env = dict(os.environ)
    env.pop("PG_LIBRARY", None)
    if library:
        env["PG_LIBRARY"] = library
    r = subprocess.run([sys.executable, "-c", CHILD % {"root": ROOT}], cwd=ROOT, env=env, stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, timeout=900)
    text = r.stdout.decode()
    assert r.returncode == 0, text[-3000:]
    line = [l for l in text.splitlines() if l.startswith("RESULT ")][-1]
    return json.loads(line[len("RESULT "):])


def test_checked_training_kernels_stay_inside_their_operands():
    from paper_2008_01425_b200 import binding as pg
    from paper_2008_01425_b200 import build as pg_build

    got, want = _run_child(pg_build.build(checked=True)), _run_child(None)
    assert sorted(got) == sorted(want) and len(got) == 3 * len(SHAPES) + 8
    # the checks are really there: an address behind an operand is reported, one inside is not
    assert got.pop("__probe__")[0] == pg.PG_ERR_BOUNDS and want.pop("__probe__")[0] == pg.PG_OK
    for name in sorted(got):
        assert got[name][0] == pg.PG_OK, "%s: status %d in the checked build" % (name, got[name][0])
        assert want[name][0] == pg.PG_OK
        assert got[name][1] == want[name][1], "%s: the checked build gives other bits" % name
