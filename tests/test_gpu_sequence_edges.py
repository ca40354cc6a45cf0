"""The sequence operators where calls, tokens, rows and chunks end: against their formulas in 64 bits, by the tolerances of test_gpu_sequence.py, and
against calls that must give the same bits."""
import ctypes
import json
import math
import os
import subprocess
import sys
import threading

import pytest

torch = pytest.importorskip("torch")

from tests import test_gpu_sequence_bounds_checked as bounds  # noqa: E402
from tests.test_gpu_sequence import (check_loss, loss_inputs, norm_grad_reference, scan_forward, scan_grad_reference, scan_inputs,  # noqa: E402
                                     scan_output)
from tests.test_gpu_sequence import test_selective_scan as scan_case, test_selective_scan_gradient as scan_gradient_case  # noqa: E402
from tests.test_gpu_training import BF, HF, U, check, eight, gen, make8, rand, strided  # noqa: E402

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


# ---------------------------------------------------------------- calls from several host threads
def loss_of(tr, classes):
    x, ids, teacher, labels = loss_inputs(gen(classes), 1, 3, classes, 4, BF, True, 0)
    dloss = torch.ones(1, 3, device="cuda")
    return lambda: list(tr.pg_distillation_loss(x, ids, teacher, labels, 2.0, 0.5, dloss=dloss))


def scan_gradient_of(tr, length):
    g = gen(length)
    c, more = scan_inputs(g, 1, 2, length, 20, 16, BF, False, False, False, 0)
    dy = rand(g, 1, 2 * length, 20).to(BF)
    return lambda: list(tr.pg_selective_scan_grad(dy, **c, **more))[:-1]


def again(tr, monkeypatch, call):
    """The outputs of a call, and the C call by itself, on any stream, with the same outputs."""
    held = []

    def run(self, fn, args, size_fn=None):
        need = ctypes.c_size_t(0)
        if size_fn is not None:
            assert size_fn(ctypes.byref(args), ctypes.byref(need)) == 0
        scratch = torch.empty(need.value, dtype=torch.uint8, device="cuda")
        rest = () if size_fn is None else (scratch.data_ptr(), need.value)
        held.append((lambda stream: fn(ctypes.byref(args), *rest, stream), scratch, call))   # (and what it works on)
        assert held[-1][0](self.handle) == 0

    with monkeypatch.context() as m:
        m.setattr(tr._Call, "run", run)
        outputs = call()
    return outputs, held[0]


@pytest.mark.parametrize("make,sizes", [(loss_of, (28000, 50000)), (scan_gradient_of, (36, 50))])
def test_calls_of_two_sizes_from_several_host_threads(tr, monkeypatch, make, sizes):
    """The shared memory that a kernel may ask for belongs to the kernel and not to the call: a small call must not take it from a large one."""
    jobs = [again(tr, monkeypatch, make(tr, sizes[k % 2])) for k in range(4)]
    torch.cuda.synchronize()
    want = [[v.clone() for v in outputs] for outputs, _ in jobs]
    wrong, start = [], threading.Barrier(len(jobs))

    def run(k):
        stream = torch.cuda.Stream()
        call, handle = jobs[k][1][0], stream.cuda_stream
        start.wait()
        wrong.extend(status for status in [call(handle) for _ in range(2000)] if status)
        stream.synchronize()

    threads = [threading.Thread(target=run, args=(k,)) for k in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, "%d calls failed, the first with %d" % (len(wrong), wrong[0])
    for (outputs, _), w in zip(jobs, want):
        assert all(torch.equal(p, q) for p, q in zip(outputs, w))


# ---------------------------------------------------------------- loss
@pytest.mark.parametrize("n", [70, 3000, 30001, 110000])
@pytest.mark.parametrize("which", ["neither", "list at weight 0", "labels at weight 0"])
def test_the_gradient_of_a_loss_without_terms(tr, n, which):
    x, ids, teacher, labels = loss_inputs(gen(n), 1, 3, n, 4, HF, True, 0)
    x[0, 0, 5], x[0, 1, 7], x[0, 2] = 1000.0, math.nan, -math.inf
    kw = {"neither": {}, "list at weight 0": dict(ids=ids, teacher=teacher, alpha=0.0), "labels at weight 0": dict(labels=labels, alpha=1.0)}[which]
    ones = torch.ones(1, 3, device="cuda")
    r = tr.pg_distillation_loss(x, dloss=ones, **kw)
    assert not r.loss.any() and not r.lse.any() and not r.dlogits.any()
    assert not tr.pg_distillation_loss_grad(ones, x, r.lse, **kw).any()


@pytest.mark.parametrize("n", [50, 3000, 30001, 110000])
@pytest.mark.parametrize("tau", [1.0, 2.0, 1.7])
def test_rows_without_a_term_have_no_gradient(tr, n, tau):
    """Rows of padding: no label, an empty list or one of logits -inf, and any numbers as logits.  The rows around them stay as they are."""
    g = gen(n)
    x, ids, teacher, labels = loss_inputs(g, 2, 6, n, 8, BF, True, 0)
    ids[0, 1], ids[0, 4], teacher[1, 2], ids[1, 5] = -1, n, -math.inf, -7
    none = torch.zeros(2, 6, dtype=torch.bool, device="cuda")
    for row in ((0, 1), (0, 4), (1, 2), (1, 5)):
        labels[row], none[row] = -100, True
    dloss = rand(g, 2, 6)
    kw = dict(ids=ids, teacher=teacher, labels=labels, temperature=tau, alpha=0.4)
    clean = tr.pg_distillation_loss(x, dloss=dloss, **kw)
    assert not clean.loss[none].any() and not clean.dlogits[none].any()
    x[0, 1], x[0, 4, n // 2], x[1, 2], x[1, 5, 0] = math.nan, math.inf, -math.inf, 3e38
    for pad in (0, 1):
        out = strided(torch.ones_like(x), pad)
        r = tr.pg_distillation_loss(x, dloss=dloss, out=out, **kw)
        back = strided(torch.ones_like(x), pad)
        tr.pg_distillation_loss_grad(dloss, x, r.lse, out=back, **kw)
        assert not r.loss[none].any() and not out[none].any() and not back[none].any()
        assert torch.equal(r.loss[~none], clean.loss[~none]) and torch.equal(out[~none], clean.dlogits[~none])
    here = x.clone()
    tr.pg_distillation_loss(here, dloss=dloss, out=here, **kw)
    assert torch.equal(here, clean.dlogits)


@pytest.mark.parametrize("top", [127, 128, 129, 1024])
def test_lists_as_long_as_a_row_a_warp_has_room_for(tr, top):
    """Up to 128 entries the loss alone of many rows is computed by a warp each, whose lists fill a block's shared memory then."""
    x, ids, teacher, labels = loss_inputs(gen(top), 1, 4736, 1500, top, BF, True, 1)
    check_loss(tr, x, ids, teacher, labels, 2.0, 0.5, torch.ones(1, 4736, device="cuda"), BF)


# ---------------------------------------------------------------- scan
# (length of the sequence, tokens that are there)
@pytest.mark.parametrize("length,have", [(4, 4), (5, 5), (5, 4), (7, 6), (52, 51), (90, 90), (90, 31), (90, 61)])
@pytest.mark.parametrize("gate", [False, True])
def test_what_the_last_token_does_not_reach(tr, length, have, gate):
    """dA depends on neither the last token's u nor its b, and what the last token gives dB, du and ddelta does not depend on a, or only through
    the state before it: a NaN there leaves those as they are, bit for bit, wherever the last token lies in its group of tokens and chunk."""
    g = gen(length + have)
    n, m = 40, 16
    c, more = scan_inputs(g, 1, 1, length, n, m, BF, gate, True, False, 0)
    more["lengths"] = torch.tensor([[have]], dtype=torch.int32, device="cuda")
    dy = rand(g, 1, length, n).to(BF)
    want = tr.pg_selective_scan_grad(dy, **c, **more)
    assert all(torch.isfinite(v).all() for v in want if v is not None)
    other = [d for d in range(n) if d != 3]
    u = c["u"].clone()
    u[0, have - 1, 3] = math.nan
    got = tr.pg_selective_scan_grad(dy, **{**c, "u": u}, **more)
    assert torch.equal(got.da, want.da) and torch.equal(got.ddelta_bias[0, other], want.ddelta_bias[0, other])
    b = c["b"].clone()
    b[0, have - 1, 5] = math.inf
    got = tr.pg_selective_scan_grad(dy, **{**c, "b": b}, **more)
    assert torch.equal(got.da, want.da) and torch.equal(got.dskip, want.dskip)
    a = c["a"].clone()
    a[0, 3, 5] = math.nan
    got = tr.pg_selective_scan_grad(dy, **{**c, "a": a}, **more)
    assert torch.equal(got.du[0, have - 1], want.du[0, have - 1]) and torch.equal(got.db[0, have - 1], want.db[0, have - 1])
    assert torch.equal(got.da[0, other], want.da[0, other]) and torch.isnan(got.da[0, 3, 5])


@pytest.mark.parametrize("length,n,states", [(1, 20, 16), (2, 20, 3), (5, 20, 16), (53, 20, 17), (700, 33, 16)])
@pytest.mark.parametrize("ragged", [False, True])
def test_states_that_are_forgotten_at_once(tr, length, n, states, ragged):
    """a = -inf, or so large that a log2(e) is: exp(D a) = 0 for every token, and a sequence without tokens keeps its state."""
    g = gen(length)
    c, more = scan_inputs(g, 1, 3, length, n, states, BF, True, True, ragged, 0)
    if ragged:
        more["lengths"][0, 0] = 0
    dy = rand(g, 1, 3 * length, n).to(BF)
    some = torch.rand(c["a"].shape, device="cuda", generator=g) < 0.5
    c["a"] = torch.where(some, torch.full_like(c["a"], -1e30), c["a"])
    f = scan_forward(c, more, length)
    _, y, slack = scan_output(c, more, f)
    want, last = tr.pg_selective_scan(**c, **more, state_out=True)
    check(want, y, slack, BF)
    check(last, f["h"][-1], f["e"][-1] + 2 * U * f["h"][-1].abs())
    grads = tr.pg_selective_scan_grad(dy, **c, **more)
    for rate in (-math.inf, -3.4e38):
        c["a"] = torch.where(some, torch.full_like(c["a"], rate), c["a"])
        got, state = tr.pg_selective_scan(**c, **more, state_out=True)
        assert torch.equal(got, want) and torch.equal(state, last)
        for p, q in zip(tr.pg_selective_scan_grad(dy, **c, **more), grads):
            assert torch.equal(p, q)


def scan_gradient_needs(tr, b, length, n, m):
    """Bytes of workspace of the scan's gradient of one sequence a worker."""
    from paper_2008_01425_b200.binding import load_library

    args, size = tr.pg_scan_grad_args(0, b, 1, length, n, m), ctypes.c_size_t()
    assert load_library().pg_selective_scan_grad_workspace_bytes(ctypes.byref(args), ctypes.byref(size)) == 0
    return size.value


def gradient_is_chunked(tr, b, length, n, m):
    """Whether there is room for the states and carries of two chunks besides what grows with the tokens."""
    per_token = (scan_gradient_needs(tr, b, 33, n, m) - scan_gradient_needs(tr, b, 1, n, m)) / 32
    return scan_gradient_needs(tr, b, length, n, m) - scan_gradient_needs(tr, b, 1, n, m) - per_token * (length - 1) >= 16 * b * n * m


@pytest.mark.parametrize("n,states", [(5, 16), (33, 3), (20, 40)])
def test_growing_states_that_nothing_has_reached(tr, n, states):
    """a > 0: over a chunk exp of the sum of steps leaves fp32's range, but what is zero stays zero.  Inputs come with the last tokens, gradients
    with the first."""
    g = gen(n)
    length = 700
    c, more = scan_inputs(g, 1, 1, length, n, states, BF, False, False, False, 0)
    c["a"] = torch.rand(1, n, states, device="cuda", generator=g) + 0.5
    c["delta"] = torch.full_like(c["delta"], 5.0)
    c["delta_bias"] = torch.zeros_like(c["delta_bias"])
    c["u"][:, :-8] = 0
    dy = rand(g, 1, length, n).to(BF)
    dy[:, 8:] = 0
    f = scan_forward(c, more, length)
    _, y, slack = scan_output(c, more, f)
    got, last = tr.pg_selective_scan(**c, **more, state_out=True)
    check(got, y, slack, BF)
    check(last, f["h"][-1], f["e"][-1] + 2 * U * f["h"][-1].abs())
    assert gradient_is_chunked(tr, 1, length, n, states)
    want, off = scan_grad_reference(c, more, dy, 64)
    r = tr.pg_selective_scan_grad(dy, **c, **more)
    for name in want:
        check(getattr(r, name), want[name], off[name] + 2 * U * want[name].abs(), None if name in ("da", "dskip", "ddelta_bias") else BF)


# ---------------------------------------------------------------- layer norm
@pytest.mark.parametrize("n", [64, 650, 1029, 5000])
@pytest.mark.parametrize("from8", [False, True])
def test_layer_norm_gradient_where_differences_leave_fp32(tr, n, from8):
    """Rows near bf16's ends: an element may be further from the mean than fp32's largest number."""
    g = gen(n)
    b, t = 2, 9
    h = torch.full((b, t, n), -1.2e38, device="cuda")
    h[..., 1::7] = 3.2e38
    h[0, 0], h[0, 1] = -h[0, 0], rand(g, n)           # the other way round, and a row like others
    h = h.to(BF)
    held = make8(tr, h, BF) if from8 else h
    if from8:
        h = eight(h, BF)[2].to(BF)
    out = tr.pg_add_layer_norm(h, eps=0.0)
    dy, gain = rand(g, b, t, n).to(BF), rand(g, b, n)
    dx, dgain, dbias = tr.pg_add_layer_norm_grad(dy, held, out.mean, out.rstd, gain)
    want, slack, wg, sg, wb, sb = norm_grad_reference(dy, h, out.mean, out.rstd, gain, None)
    check(dx, want, slack + 2.0 ** -149, BF)
    check(dgain, wg, sg)
    check(dbias, wb, sb)


@pytest.mark.parametrize("n", [70, 650, 1029, 5000])
@pytest.mark.parametrize("power", [100, -100])
def test_norms_of_far_rows_are_those_of_near_ones(tr, n, power):
    """Rows whose squares leave fp32's range are scaled by a power of two, which rounds nothing: the same bits as of the rows at home."""
    x = rand(gen(n), 2, 6, n).to(BF)
    far = (x.double() * 2.0 ** power).to(BF)
    assert torch.equal(far.double(), x.double() * 2.0 ** power)
    for norm in (tr.pg_add_rms_norm, tr.pg_add_layer_norm):
        near, out = norm(x, eps=0.0), norm(far, eps=0.0)
        assert torch.equal(out.y, near.y) and torch.equal(out.rstd.double() * 2.0 ** power, near.rstd.double())
        if norm is tr.pg_add_layer_norm:
            assert torch.equal(out.mean.double(), near.mean.double() * 2.0 ** power)


@pytest.mark.parametrize("n", [2, 64, 650, 1029, 5000, 16384])
@pytest.mark.parametrize("eps", [1e-5, 1e-35])
def test_layer_norm_of_rows_of_equal_values(tr, n, eps):
    """Rows that a mask filled with bf16's lowest number, and others: y is the bias and rstd is eps ^ -1/2 (sums of equal 16-bit values are exact)."""
    g = gen(n)
    values = [torch.finfo(BF).min, torch.finfo(BF).max, 3e36, 1e10, 1.0, 1e-20, 0.0]
    x = torch.tensor(values, device="cuda").to(BF)[:, None].expand(-1, n).contiguous()
    gain, bias = rand(g, n), rand(g, n)
    out = tr.pg_add_layer_norm(x, gain, bias, eps=eps)
    root = torch.full((len(values),), float(torch.tensor(eps, dtype=torch.float32)), dtype=torch.float64, device="cuda") ** -0.5
    check(out.y, bias.double().expand_as(x), torch.zeros_like(x, dtype=torch.float64), BF)
    check(out.mean, x[:, 0].double(), 0 * root)
    check(out.rstd, root, 32 * U * root)
    dy = rand(g, len(values), n).to(BF)
    dx, dgain, dbias = tr.pg_add_layer_norm_grad(dy, x, out.mean, out.rstd, gain)
    want, slack = norm_grad_reference(dy[None], x[None], out.mean[None], out.rstd[None], gain[None], None)[:2]
    check(dx, want[0], slack[0], BF)
    assert not dgain.any()


# ---------------------------------------------------------------- convolution
@pytest.mark.parametrize("length,have", [(1, 1), (2, 2), (9, 9), (9, 5), (70, 64), (70, 65), (130, 130)])
@pytest.mark.parametrize("taps", [2, 3, 4])
def test_weights_of_tokens_behind_the_last_do_not_count(tr, length, have, taps):
    """dx of a token takes a weight for every token up to taps - 1 behind it that is there: an infinite one of another changes nothing."""
    g = gen(length + taps)
    n = 70
    x, dy, weight = rand(g, 1, length, n).to(BF), rand(g, 1, length, n).to(BF), rand(g, 1, n, taps)
    kw = dict(activation="none", lengths=torch.tensor([[have]], dtype=torch.int32, device="cuda"))
    want = tr.pg_causal_conv_grad(dy, x, weight, **kw)
    weight[0, ::2, 0] = math.inf                       # the oldest input's: of dx of tokens that have taps - 1 behind them
    got = tr.pg_causal_conv_grad(dy, x, weight, **kw)
    last = slice(max(0, have - taps + 1), length)
    assert torch.equal(got[0][:, last], want[0][:, last]) and torch.equal(got[0][..., 1::2], want[0][..., 1::2])
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    assert not torch.isfinite(got[0][0, :max(0, have - taps + 1), ::2]).any()


# ---------------------------------------------------------------- chunks, and 17 to 32 states
CHUNKS = [((1, 2, 52, 50), 16, 1), ((1, 2, 53, 50), 16, 0), ((2, 1, 73, 130), 8, 1), ((1, 2, 45, 40), 32, 0), ((1, 1, 300, 20), 24, 1), ((2, 1, 300, 33), 32, 0), ((1, 1, 1100, 9), 20, 0)]
KINDS = [(BF, True, True, True), (HF, False, False, False)]


@pytest.mark.parametrize("shape,states,pad", CHUNKS)
@pytest.mark.parametrize("dtype,gate,carried,ragged", KINDS)
def test_scan_at_the_ends_of_chunks(tr, shape, states, pad, dtype, gate, carried, ragged):
    scan_case(tr, shape, states, pad, dtype, gate, carried, ragged)


@pytest.mark.parametrize("shape,states,pad", CHUNKS)
@pytest.mark.parametrize("dtype,gate,carried,ragged", KINDS)
def test_scan_gradient_at_the_ends_of_chunks(tr, shape, states, pad, dtype, gate, carried, ragged):
    assert gradient_is_chunked(tr, 1, shape[2], shape[3], states) == (shape[2] > 52)
    scan_gradient_case(tr, shape, states, pad, dtype, gate, carried, ragged)


def test_chunks_of_more_states_than_a_grid_has_rows(tr):
    """8.96 million states per sequence, in chunks: a channel's gradients are those it has on its own."""
    n, m, t = 140000, 64, 73
    assert gradient_is_chunked(tr, 1, t, n, m) and gradient_is_chunked(tr, 1, t, 16, m)
    c, more = scan_inputs(gen(11), 1, 1, t, n, m, BF, False, False, False, 0)
    dy = rand(gen(12), 1, t, n).to(BF)
    got = tr.pg_selective_scan_grad(dy, **c, **more)
    for last in (slice(n - 16, n), slice(70000, 70016)):
        part = {k: v[..., last].contiguous() if k in ("u", "delta", "skip", "delta_bias") else v[:, last].contiguous() if k == "a" else v for k, v in c.items()}
        want = tr.pg_selective_scan_grad(dy[..., last].contiguous(), **part, **more)
        assert torch.equal(got.du[..., last], want.du) and torch.equal(got.ddelta[..., last], want.ddelta)


def test_what_is_behind_a_sequence_is_not_used_in_chunks(tr):
    g = gen(9)
    b, s, length, n, m = 2, 4, 90, 50, 24
    assert gradient_is_chunked(tr, 1, length, n, m)
    c, more = scan_inputs(g, b, s, length, n, m, BF, True, True, False, 0)
    dy = rand(g, b, s * length, n).to(BF)
    lengths = torch.tensor([[0, 1, 40, 90], [90, 89, 30, 61]], dtype=torch.int32, device="cuda")
    beyond = (torch.arange(length, device="cuda") >= lengths[..., None]).reshape(b, s * length, 1)
    dirty = lambda v: torch.where(beyond, torch.full_like(v, math.nan), v)
    bad = {**c, **{k: dirty(c[k]) for k in ("u", "delta", "b", "c", "z")}}
    kw = {**more, "lengths": lengths}
    for f in (lambda q, d: list(tr.pg_selective_scan(**q, **kw, state_out=True)), lambda q, d: list(tr.pg_selective_scan_grad(d, **q, **kw))):
        for p, q in zip(f(c, dy), f(bad, dirty(dy))):
            assert torch.isfinite(p).all() and torch.equal(p, q)
            if p.shape[:2] == (b, s * length):
                assert not p[beyond.expand_as(p)].any()


# ---------------------------------------------------------------- the bounds-checked build
# workers, sequences, length, channels, states, classes
MORE_SHAPES = [(1, 2, 52, 50, 16, 33), (1, 2, 53, 50, 16, 700), (2, 1, 73, 65, 8, 64), (1, 2, 45, 40, 24, 70), (2, 1, 300, 33, 32, 500), (1, 1, 130, 9, 20, 9001)]


def more_cases():
    for i, shape in enumerate(MORE_SHAPES):
        for pad in (0, 1):
            yield shape + (pad, "float16" if (i + pad) % 2 else "bfloat16")


def test_chunks_in_the_bounds_checked_build():
    """Chunked gradients and 17 to 32 states, as test_gpu_sequence_bounds_checked.py does with its shapes."""
    from paper_2008_01425_b200 import build as pg_build

    child = bounds.CHILD.replace("test_gpu_sequence_bounds_checked import cases", "test_gpu_sequence_edges import more_cases as cases").replace(
        "cases, outputs", "cases\nfrom tests.test_gpu_sequence_bounds_checked import outputs")
    results = []
    for library in (pg_build.build(checked=True), None):
        env = {k: v for k, v in os.environ.items() if k != "PG_LIBRARY"}
        if library:
            env["PG_LIBRARY"] = library
        r = subprocess.run([sys.executable, "-c", child % {"root": bounds.ROOT}], cwd=bounds.ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, timeout=600)
        text = r.stdout.decode()
        assert r.returncode == 0, text[-3000:]
        results.append(json.loads([l for l in text.splitlines() if l.startswith("RESULT ")][-1][len("RESULT "):]))
    got, want = results
    assert sorted(got) == sorted(want) and len(got) == 2 * len(MORE_SHAPES)
    for name in got:
        assert got[name][0] == want[name][0] == 0, "%s: status %d in the checked build" % (name, got[name][0])
        assert got[name][1] == want[name][1], "%s: the checked build gives other bits" % name
