"""The sequence operators (layer norm, causal convolution, selective scan, distillation loss) refuse bad arguments without a GPU."""
import ctypes

import pytest

from paper_2008_01425_b200 import binding as pg
from paper_2008_01425_b200 import build as pg_build

tr = pytest.importorskip("paper_2008_01425_b200.training")
CALLS = {"pg_add_layer_norm": tr.pg_layer_norm_args, "pg_add_layer_norm_grad": tr.pg_layer_norm_grad_args, "pg_causal_conv": tr.pg_conv_args,
         "pg_causal_conv_grad": tr.pg_conv_grad_args, "pg_selective_scan": tr.pg_scan_args, "pg_selective_scan_grad": tr.pg_scan_grad_args,
         "pg_distillation_loss": tr.pg_distillation_args, "pg_distillation_loss_grad": tr.pg_distillation_args}
WITH_WORKSPACE = ("pg_add_layer_norm_grad", "pg_causal_conv_grad", "pg_selective_scan", "pg_selective_scan_grad")


@pytest.fixture(scope="module")
def lib():
    pg_build.build()
    return pg.load_library()


def call(lib, name, args):
    p = None if args is None else ctypes.byref(args)
    return getattr(lib, name)(p, None, 0, None) if name in WITH_WORKSPACE else getattr(lib, name)(p, None)


def valid(name, **change):
    """Sizes that are fine, and no pointers."""
    a = CALLS[name]()
    for f, v in dict(dtype=0, activation=3, batch=1, tokens=4, sequences=2, length=4, cols=8, channels=8, width=4, states=16, classes=8, top=0,
                     temperature=1.0, alpha=1.0, eps=1e-5).items():
        if hasattr(a, f):
            setattr(a, f, v)
    for f, kind in CALLS[name]._fields_:
        if kind is tr.pg_matrix:
            getattr(a, f).ld = 64
    for f, v in change.items():
        setattr(a, f, v)
    return a


@pytest.mark.parametrize("name", sorted(CALLS))
def test_null_empty_and_pointerless_arguments_are_refused(lib, name):
    assert call(lib, name, None) == pg.PG_ERR_INVALID
    assert call(lib, name, CALLS[name]()) == pg.PG_ERR_INVALID            # zero widths
    assert call(lib, name, valid(name)) == pg.PG_ERR_INVALID              # no pointers
    if name in WITH_WORKSPACE:
        n = ctypes.c_size_t(7)
        query = getattr(lib, name + "_workspace_bytes")
        assert query(None, ctypes.byref(n)) == pg.PG_ERR_INVALID
        assert query(ctypes.byref(CALLS[name]()), ctypes.byref(n)) == pg.PG_ERR_INVALID
        assert query(ctypes.byref(valid(name)), None) == pg.PG_ERR_INVALID
        assert n.value == 7
        assert query(ctypes.byref(valid(name)), ctypes.byref(n)) == pg.PG_OK


@pytest.mark.parametrize("name", sorted(CALLS))
def test_sizes_out_of_range_are_refused(lib, name):
    bad = [dict(dtype=2), dict(dtype=-1), dict(batch=-1), dict(batch=70000)]
    fields = {f for f, _ in CALLS[name]._fields_}
    bad += [{f: v} for f, values in (("tokens", (-1,)), ("sequences", (-1,)), ("length", (-1,)), ("cols", (0, -3)), ("channels", (0, -3)), ("width", (0, 1, 5)),
                                     ("activation", (-1, 1, 2, 4)), ("states", (0, -1)), ("classes", (0,)), ("top", (-1,)),
                                     ("temperature", (0.0, -1.0, float("nan"), float("inf"), 1e-38)), ("alpha", (-0.1, 1.1, float("nan"))),
                                     ("eps", (-1.0, float("nan"), float("inf")))) if f in fields for v in values]
    bad += [dict(sequences=1 << 20, length=1 << 20)] if "sequences" in fields else []
    for change in bad:
        assert call(lib, name, valid(name, **change)) == pg.PG_ERR_INVALID, change


@pytest.mark.parametrize("name", sorted(CALLS))
def test_nothing_to_do_is_fine(lib, name):
    """No workers: no pointers are looked at."""
    assert call(lib, name, valid(name, batch=0)) == pg.PG_OK


def test_too_large_is_said_before_anything_else_of_the_sizes(lib):
    n = ctypes.c_size_t(7)
    for name, change in (("pg_causal_conv_grad", dict(channels=(1 << 19) + 1)), ("pg_selective_scan", dict(states=65)), ("pg_selective_scan_grad", dict(states=65)),
                         ("pg_selective_scan_grad", dict(channels=(1 << 19) + 1)), ("pg_add_layer_norm_grad", dict(cols=16385))):
        assert getattr(lib, name + "_workspace_bytes")(ctypes.byref(valid(name, **change)), ctypes.byref(n)) == pg.PG_ERR_TOO_LARGE, name
        assert n.value == 7
    a = valid("pg_distillation_loss", batch=0, top=1025)
    a.ids.ld = a.teacher.ld = 1025
    assert call(lib, "pg_distillation_loss", a) == pg.PG_ERR_TOO_LARGE


def test_workspaces_grow_with_what_they_hold(lib):
    n, m = ctypes.c_size_t(0), ctypes.c_size_t(0)
    query = lib.pg_selective_scan_workspace_bytes
    assert query(ctypes.byref(valid("pg_selective_scan", sequences=1, length=35)), ctypes.byref(n)) == pg.PG_OK and n.value == 0     # one chunk
    assert query(ctypes.byref(valid("pg_selective_scan", sequences=1, length=8192)), ctypes.byref(n)) == pg.PG_OK
    assert n.value >= 4 * 3 * 8 * 17                                      # three chunks at least, states and a sum of steps each
    query = lib.pg_selective_scan_grad_workspace_bytes
    assert query(ctypes.byref(valid("pg_selective_scan_grad", sequences=1, length=35)), ctypes.byref(n)) == pg.PG_OK
    assert query(ctypes.byref(valid("pg_selective_scan_grad", sequences=3, length=35)), ctypes.byref(m)) == pg.PG_OK
    assert 4 * 35 * 2 * 16 <= n.value < m.value


def test_the_binding_refuses_cpu_tensors_and_odd_shapes():
    import torch

    x = torch.zeros(2, 4, 8, dtype=torch.bfloat16)
    w = torch.zeros(2, 8, 4)
    for f in (lambda: tr.pg_add_layer_norm(x), lambda: tr.pg_causal_conv(x, w), lambda: tr.pg_selective_scan(x, x, w, x, x),
              lambda: tr.pg_distillation_loss(x), lambda: tr.pg_distillation_loss_grad(None, x, None)):
        with pytest.raises(ValueError):
            f()
