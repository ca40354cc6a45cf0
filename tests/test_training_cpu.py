"""The training calls refuse bad arguments without a GPU, and the binding's structs are the header's."""
import ctypes
import os
import re

import pytest

from paper_2008_01425_b200 import binding as pg
from paper_2008_01425_b200 import build as pg_build

tr = pytest.importorskip("paper_2008_01425_b200.training")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CALLS = {"pg_add_rms_norm": tr.pg_norm_args, "pg_add_rms_norm_grad": tr.pg_norm_grad_args, "pg_linear": tr.pg_linear_args,
         "pg_linear_input_grad": tr.pg_input_grad_args, "pg_linear_weight_grad": tr.pg_weight_grad_args,
         "pg_activation_grad": tr.pg_activation_grad_args, "pg_checkpoint_write": tr.pg_checkpoint_args,
         "pg_checkpoint_read": tr.pg_checkpoint_args}
WITH_WORKSPACE = ("pg_add_rms_norm_grad", "pg_linear", "pg_linear_input_grad", "pg_linear_weight_grad")


@pytest.fixture(scope="module")
def lib():
    pg_build.build()
    return pg.load_library()


def call(lib, name, args):
    p = None if args is None else ctypes.byref(args)
    return getattr(lib, name)(p, None, 0, None) if name in WITH_WORKSPACE else getattr(lib, name)(p, None)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_null_and_empty_arguments_are_refused(lib, name):
    assert call(lib, name, None) == pg.PG_ERR_INVALID
    assert call(lib, name, CALLS[name]()) == pg.PG_ERR_INVALID            # zero widths
    if name in WITH_WORKSPACE:
        n = ctypes.c_size_t(7)
        assert getattr(lib, name + "_workspace_bytes")(None, ctypes.byref(n)) == pg.PG_ERR_INVALID
        assert getattr(lib, name + "_workspace_bytes")(ctypes.byref(CALLS[name]()), ctypes.byref(n)) == pg.PG_ERR_INVALID
        assert n.value == 7


@pytest.mark.parametrize("name", sorted(CALLS))
def test_missing_pointers_and_odd_sizes_are_refused(lib, name):
    for dtype, batch, tokens, width in ((0, 1, 4, 8), (2, 1, 4, 8), (-1, 1, 4, 8), (0, -1, 4, 8), (0, 1, -4, 8), (0, 1, 4, 0), (0, 70000, 4, 8)):
        a = CALLS[name]()
        a.dtype, a.batch, a.tokens = dtype, batch, tokens
        for f in ("cols", "in_features", "out_features"):
            if hasattr(a, f):
                setattr(a, f, width)
        assert call(lib, name, a) == pg.PG_ERR_INVALID


def test_structs_match_the_header():
    """Field names and order of every struct, read from the header's text."""
    text = open(os.path.join(ROOT, "include", "pg_training.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    for body, name in re.findall(r"typedef struct \w+ \{(.*?)\} (\w+);", text, flags=re.S):
        fields = []
        for line in body.split(";"):
            line = line.strip()
            if line:
                kind = line.replace("const ", "").split()[0]
                fields += [(kind, f.strip().split()[-1].lstrip("*"), "*" in f) for f in line.split(",")]
        mine = getattr(tr, name)._fields_
        assert [f[1] for f in fields] == [f[0] for f in mine], name
        for (kind, _, pointer), (_, ctype) in zip(fields, mine):
            want = ctypes.c_void_p if pointer else {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float,
                                                    "pg_matrix": tr.pg_matrix, "pg_matrix8": tr.pg_matrix8}[kind]
            assert ctype is want, (name, kind)


def test_the_binding_refuses_cpu_tensors():
    import torch

    x = torch.zeros(2, 4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        tr.pg_linear(x, x)
    with pytest.raises(ValueError):
        tr.pg_checkpoint_write(x)


def test_a_norm_gradient_that_is_too_wide_has_no_workspace(lib):
    """The query refuses what the call refuses, and does not touch the size."""
    query = lib.pg_add_rms_norm_grad_workspace_bytes
    for cols, status in ((1, pg.PG_OK), (16384, pg.PG_OK), (16385, pg.PG_ERR_TOO_LARGE), (20000, pg.PG_ERR_TOO_LARGE), (1 << 30, pg.PG_ERR_TOO_LARGE)):
        a = tr.pg_norm_grad_args()
        a.batch, a.tokens, a.cols, a.dgain = 2, 64, cols, 256
        n = ctypes.c_size_t(7)
        assert query(ctypes.byref(a), ctypes.byref(n)) == status, cols
        # at least one row of partial sums per worker, at most one per token
        assert n.value == 7 if status else 2 * cols * 4 <= n.value <= 2 * 64 * cols * 4, cols
