"""Python binding of ``include/pg_training.h``: forward and backward pass of residual blocks for all
simulated workers at once (ctypes, same names as the C calls).

Tensors are CUDA tensors of shape (workers, tokens, features), or (tokens, features) for one worker;
16-bit ones are bf16 or fp16, the same in one call, with features contiguous and any row stride.
Weights are (workers, out, in), biases and gains fp32 (workers, n).  An axis of workers that was
expanded (stride 0) is shared by all workers.  Results are allocated with torch unless ``out`` is
given; their rows start on 16-byte boundaries, where every kernel takes its fastest path.

The calls are not part of torch's differentiation: results do not require gradients, whatever the inputs
do, and the gradients are calls of their own.

``stream`` is a torch stream or a raw handle; None means torch's current stream on the tensors'
device, and a call is then ordered like any torch operation.  On another stream the caller orders the
call after what writes its inputs and before what reads its results.  The memory of both looks after
itself: results and workspaces come from that stream's memory (torch's current stream may still have work
to do on its own that is free again), and neither they nor the inputs are reused before both streams have passed.

    from paper_2008_01425_b200 import training as tr
    n = tr.pg_add_rms_norm(x, gain, residual=r, eight_bit=True)      # n.h, n.y, n.y8, n.rstd
    y, z8 = tr.pg_linear(n.y, W, bias, activation="gelu", save_z=True)
    dz, db = tr.pg_activation_grad(dy, z8, "gelu")
    dW = tr.pg_linear_weight_grad(dz, n.y8)
    dn = tr.pg_linear_input_grad(dz, W)
    dx, dgain = tr.pg_add_rms_norm_grad(dn, n.h, n.rstd, gain)

``python -m paper_2008_01425_b200.sgd_experiment`` runs them under gossip rounds.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional, Union

import torch

from .binding import _check, load_library

PG_BF16, PG_F16 = 0, 1
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
BLOCK8 = 32                      # values that share a scale in the 8-bit form
_DTYPES = {torch.bfloat16: PG_BF16, torch.float16: PG_F16}
_vp, _i32, _i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64


class pg_matrix(ctypes.Structure):
    _fields_ = [("data", _vp), ("ld", _i64), ("stride", _i64)]


class pg_matrix8(ctypes.Structure):
    _fields_ = [("values", _vp), ("scales", _vp), ("ld", _i64), ("stride", _i64), ("scale_ld", _i64), ("scale_stride", _i64)]


class pg_norm_args(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("batch", _i32), ("tokens", _i32), ("cols", _i32), ("eps", ctypes.c_float),
                ("x", pg_matrix), ("residual", pg_matrix), ("gain", _vp), ("gain_stride", _i64), ("h", pg_matrix),
                ("y", pg_matrix), ("y8", pg_matrix8), ("h8", pg_matrix8), ("rstd", _vp)]


class pg_norm_grad_args(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("batch", _i32), ("tokens", _i32), ("cols", _i32), ("accumulate", _i32),
                ("dy", pg_matrix), ("h", pg_matrix), ("h8", pg_matrix8), ("rstd", _vp), ("gain", _vp), ("gain_stride", _i64),
                ("dh", pg_matrix), ("dx", pg_matrix), ("dgain", _vp), ("dgain_stride", _i64)]


class pg_linear_args(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("activation", _i32), ("batch", _i32), ("tokens", _i32), ("in_features", _i32),
                ("out_features", _i32), ("x", pg_matrix), ("weight", pg_matrix), ("bias", _vp), ("bias_stride", _i64),
                ("residual", pg_matrix), ("y", pg_matrix), ("z8", pg_matrix8)]


class pg_input_grad_args(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("batch", _i32), ("tokens", _i32), ("in_features", _i32), ("out_features", _i32),
                ("dz", pg_matrix), ("weight", pg_matrix), ("residual", pg_matrix), ("dx", pg_matrix)]


class pg_weight_grad_args(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("batch", _i32), ("tokens", _i32), ("in_features", _i32), ("out_features", _i32),
                ("accumulate", _i32), ("dz", pg_matrix), ("x", pg_matrix), ("x8", pg_matrix8), ("dweight", pg_matrix)]


class pg_activation_grad_args(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("activation", _i32), ("batch", _i32), ("tokens", _i32), ("cols", _i32), ("accumulate", _i32),
                ("dy", pg_matrix), ("z8", pg_matrix8), ("dz", pg_matrix), ("dbias", _vp), ("dbias_stride", _i64)]


class pg_checkpoint_args(ctypes.Structure):
    _fields_ = [("dtype", _i32), ("batch", _i32), ("tokens", _i32), ("cols", _i32), ("x", pg_matrix), ("x8", pg_matrix8)]


class Checkpoint8(NamedTuple):
    """A tensor in 8 bits: int8 `values` of the tensor's shape (rows padded to 16 bytes in memory), one
    uint8 power of two (bias 127) per 32 values of a row in `scales`, and the 16-bit type it stands for."""
    values: torch.Tensor
    scales: torch.Tensor
    dtype: torch.dtype


class NormOutput(NamedTuple):
    h: Optional[torch.Tensor]
    y: Optional[torch.Tensor]
    y8: Optional[Checkpoint8]
    h8: Optional[Checkpoint8]
    rstd: torch.Tensor


def _refuse(where: str, why: str):
    raise ValueError("%s: %s" % (where, why))


_raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
_empty = torch.empty_strided
_NONE = pg_matrix(None, 0, 0)
_NONE8 = pg_matrix8(None, None, 0, 0, 0, 0)


class _Call:
    """Shape, device and stream of one call, taken from its first tensor; checks the others against it.  (Small calls cost
    what this costs, so it asks torch for as little as it can.)"""

    __slots__ = ("where", "dtype", "kind", "index", "device", "single", "batch", "tokens", "cols", "handle", "other")

    def __init__(self, where: str, first, stream):
        dtype = getattr(first, "dtype", None)
        if type(first) is Checkpoint8:
            first = first.values
        kind = _DTYPES.get(dtype)
        if kind is None or not isinstance(first, torch.Tensor) or not first.is_cuda:
            _refuse(where, "expected a bf16 or fp16 CUDA tensor")
        shape = first.shape
        if len(shape) == 3:
            self.single = False
            self.batch, self.tokens, self.cols = shape
        elif len(shape) == 2:
            self.single = True
            self.batch = 1
            self.tokens, self.cols = shape
        else:
            _refuse(where, "expected two or three dimensions")
        if self.batch > 65535 or self.tokens > 1 << 30 or self.cols > 1 << 30:
            _refuse(where, "shape %s is too large" % (tuple(shape),))
        self.where, self.dtype, self.kind = where, dtype, kind
        self.device = first.device
        self.index = first.get_device()
        self.handle, self.other = _raw_stream(self.index), None
        if stream is not None:
            handle = stream if isinstance(stream, int) else stream.cuda_stream
            if handle != self.handle:
                self.handle, self.other = handle, torch.cuda.ExternalStream(handle, device=self.device)

    def matrix(self, t, rows: int, cols: int, dtype, name: str) -> pg_matrix:
        if t is None:
            return _NONE
        if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != self.index:
            _refuse(self.where, "%s must be a %s tensor on %s" % (name, dtype, self.device))
        shape, strides = t.shape, t.stride()
        if len(shape) == 3 and shape == (self.batch, rows, cols):
            stride, ld, one = strides
        elif self.single and shape == (rows, cols):
            ld, one = strides
            stride = 0
        else:
            _refuse(self.where, "%s has shape %s, expected %s" % (name, tuple(shape), (rows, cols) if self.single else (self.batch, rows, cols)))
        if one != 1 and cols > 1:
            _refuse(self.where, "%s must have its last dimension contiguous" % name)
        if self.other is not None:
            t.record_stream(self.other)
        return pg_matrix(t.data_ptr(), ld if rows > 1 else max(ld, cols), stride if self.batch > 1 else 0)

    def matrix8(self, c, rows: int, cols: int, name: str) -> pg_matrix8:
        if c is None:
            return _NONE8
        if type(c) is not Checkpoint8 or c.dtype is not self.dtype:
            _refuse(self.where, "%s must be a checkpoint of %s" % (name, self.dtype))
        v = self.matrix(c.values, rows, cols, torch.int8, name + ".values")
        s = self.matrix(c.scales, rows, (cols + BLOCK8 - 1) // BLOCK8, torch.uint8, name + ".scales")
        return pg_matrix8(v.data, s.data, v.ld if rows > 1 else (v.ld + 15) // 16 * 16, v.stride, s.ld, s.stride)

    def vector(self, t, n: int, name: str):
        """(pointer, stride) of an fp32 (workers, n) tensor; (n,) for one worker or shared by all."""
        if t is None:
            return None, 0
        if not isinstance(t, torch.Tensor) or t.dtype is not torch.float32 or t.get_device() != self.index:
            _refuse(self.where, "%s must be an fp32 tensor on %s" % (name, self.device))
        shape, strides = t.shape, t.stride()
        if shape != (self.batch, n) and shape != (n,):
            _refuse(self.where, "%s has shape %s, expected %s" % (name, tuple(shape), (self.batch, n)))
        if n > 1 and strides[-1] != 1:
            _refuse(self.where, "%s must have its last dimension contiguous" % name)
        if self.other is not None:
            t.record_stream(self.other)
        return t.data_ptr(), strides[0] if len(shape) == 2 and self.batch > 1 else 0

    def _new(self, shape, strides, dtype) -> torch.Tensor:
        if self.other is None:
            return _empty(shape, strides, dtype=dtype, device=self.device)
        current = torch.cuda.current_stream(self.device)
        with torch.cuda.stream(self.other):
            t = _empty(shape, strides, dtype=dtype, device=self.device)
        t.record_stream(current)
        return t

    def empty(self, rows: int, cols: int, dtype, unit: int) -> torch.Tensor:
        """Rows start on multiples of `unit` elements."""
        ld = (cols + unit - 1) // unit * unit
        if self.single:
            return self._new((rows, cols), (ld, 1), dtype)
        return self._new((self.batch, rows, cols), (rows * ld, ld, 1), dtype)

    def like(self, rows: int, cols: int) -> torch.Tensor:
        # 16-byte boundaries; 64-byte ones for long rows, whose pieces then fill whole 32-byte sectors of the cache
        return self.empty(rows, cols, self.dtype, 32 if cols >= 256 else 8)

    def empty8(self, rows: int, cols: int) -> Checkpoint8:
        return Checkpoint8(self.empty(rows, cols, torch.int8, 32 if cols >= 256 else 16), self.empty(rows, (cols + BLOCK8 - 1) // BLOCK8, torch.uint8, 1), self.dtype)

    def flat(self, n: int) -> torch.Tensor:
        """fp32 (workers, n), or (n,) for one worker."""
        if self.single:
            return self._new((n,), (1,), torch.float32)
        return self._new((self.batch, n), (n, 1), torch.float32)

    def run(self, fn, args, size_fn=None) -> None:
        if _current_device() != self.index:
            with torch.cuda.device(self.index):
                return self.run(fn, args, size_fn)
        args = ctypes.byref(args)
        if size_fn is None:
            status = fn(args, self.handle)
        else:
            need = ctypes.c_size_t(0)
            status = size_fn(args, ctypes.byref(need))
            if status == 0:
                if need.value:
                    scratch = self._new((need.value,), (1,), torch.uint8)
                    status = fn(args, scratch.data_ptr(), need.value, self.handle)
                else:
                    status = fn(args, None, 0, self.handle)
        if status != 0:
            _check(status, self.where)


def _activation(where: str, name: str) -> int:
    if name not in ACTIVATIONS:
        _refuse(where, "activation must be one of %s" % ", ".join(sorted(ACTIVATIONS)))
    return ACTIVATIONS[name]


def pg_add_rms_norm(x, gain=None, residual=None, eps: float = 1e-5, eight_bit: bool = False, save_h8: bool = False,
                    out=None, stream=None) -> NormOutput:
    """h = x + residual, y = h / rms(h) * gain.  eight_bit: also y8, and y holds the values of y8.
    save_h8: also the 8-bit checkpoint of h, for pg_add_rms_norm_grad.  out: tensor for y.  Without a
    residual, h is x itself."""
    c = _Call("pg_add_rms_norm", x, stream)
    t, n = c.tokens, c.cols
    h = x if residual is None else c.like(t, n)
    y = c.like(t, n) if out is None else out
    y8 = c.empty8(t, n) if eight_bit else None
    h8 = c.empty8(t, n) if save_h8 else None
    rstd = c.flat(t)
    gp, gs = c.vector(gain, n, "gain")
    args = pg_norm_args(c.kind, c.batch, t, n, eps, c.matrix(x, t, n, c.dtype, "x"),
                        c.matrix(residual, t, n, c.dtype, "residual"), gp, gs,
                        c.matrix(None if residual is None else h, t, n, c.dtype, "h"), c.matrix(y, t, n, c.dtype, "out"),
                        c.matrix8(y8, t, n, "y8"), c.matrix8(h8, t, n, "h8"), rstd.data_ptr())
    c.run(load_library().pg_add_rms_norm, args)
    return NormOutput(h, y, y8, h8, rstd)


def pg_add_rms_norm_grad(dy, h: Union[torch.Tensor, Checkpoint8], rstd, gain=None, dh=None, out=None, gain_grad=None,
                         accumulate: bool = False, stream=None):
    """(dx, dgain) of pg_add_rms_norm; dx is the residual's gradient too.  h: the stored sum or its 8-bit
    checkpoint.  dh: gradient that reaches h on the residual path.  gain_grad: where dgain goes
    (added to with accumulate)."""
    c = _Call("pg_add_rms_norm_grad", dy, stream)
    t, n = c.tokens, c.cols
    if accumulate and gain_grad is None:
        _refuse(c.where, "accumulate needs gain_grad")
    dx = c.like(t, n) if out is None else out
    dgain = c.flat(n) if gain_grad is None else gain_grad
    if not isinstance(rstd, torch.Tensor) or rstd.device != c.device or rstd.dtype != torch.float32 or rstd.numel() != c.batch * t \
            or not rstd.is_contiguous():
        _refuse(c.where, "rstd must be a contiguous fp32 tensor of %d x %d on %s" % (c.batch, t, c.device))
    if c.other is not None:
        rstd.record_stream(c.other)
    eight = isinstance(h, Checkpoint8)
    gp, gs = c.vector(gain, n, "gain")
    dp, ds = c.vector(dgain, n, "gain_grad")
    args = pg_norm_grad_args(c.kind, c.batch, t, n, int(accumulate), c.matrix(dy, t, n, c.dtype, "dy"),
                             c.matrix(None if eight else h, t, n, c.dtype, "h"), c.matrix8(h if eight else None, t, n, "h"),
                             rstd.data_ptr(), gp, gs, c.matrix(dh, t, n, c.dtype, "dh"), c.matrix(dx, t, n, c.dtype, "out"), dp, ds)
    c.run(load_library().pg_add_rms_norm_grad, args, load_library().pg_add_rms_norm_grad_workspace_bytes)
    return dx, dgain


def _weight(c: _Call, weight, cols_are_in: bool):
    if not isinstance(weight, torch.Tensor) or weight.dim() not in (2, 3) or max(weight.shape) > 1 << 30:
        _refuse(c.where, "weight must be a tensor of shape (workers, out, in)")
    n_out, n_in = weight.shape[-2:]
    if (n_in if cols_are_in else n_out) != c.cols:
        _refuse(c.where, "weight has shape %s, which does not fit rows of %d values" % (tuple(weight.shape), c.cols))
    return int(n_out), int(n_in)


def pg_linear(x, weight, bias=None, residual=None, activation: str = "none", save_z: bool = False, out=None, stream=None):
    """y = activation(x W^T + bias) + residual.  save_z: returns (y, z8), z8 the 8-bit checkpoint of the
    pre-activation for pg_activation_grad."""
    c = _Call("pg_linear", x, stream)
    n_out, n_in = _weight(c, weight, True)
    t = c.tokens
    y = c.like(t, n_out) if out is None else out
    z8 = c.empty8(t, n_out) if save_z else None
    bp, bs = c.vector(bias, n_out, "bias")
    args = pg_linear_args(c.kind, _activation(c.where, activation), c.batch, t, n_in, n_out,
                          c.matrix(x, t, n_in, c.dtype, "x"), c.matrix(weight, n_out, n_in, c.dtype, "weight"), bp, bs,
                          c.matrix(residual, t, n_out, c.dtype, "residual"), c.matrix(y, t, n_out, c.dtype, "out"), c.matrix8(z8, t, n_out, "z8"))
    c.run(load_library().pg_linear, args, load_library().pg_linear_workspace_bytes)
    return (y, z8) if save_z else y


def pg_linear_input_grad(dz, weight, residual=None, out=None, stream=None):
    """dx = dz W + residual."""
    c = _Call("pg_linear_input_grad", dz, stream)
    n_out, n_in = _weight(c, weight, False)
    t = c.tokens
    dx = c.like(t, n_in) if out is None else out
    args = pg_input_grad_args(c.kind, c.batch, t, n_in, n_out, c.matrix(dz, t, n_out, c.dtype, "dz"),
                              c.matrix(weight, n_out, n_in, c.dtype, "weight"), c.matrix(residual, t, n_in, c.dtype, "residual"),
                              c.matrix(dx, t, n_in, c.dtype, "out"))
    c.run(load_library().pg_linear_input_grad, args, load_library().pg_linear_input_grad_workspace_bytes)
    return dx


def pg_linear_weight_grad(dz, x: Union[torch.Tensor, Checkpoint8], out=None, accumulate: bool = False, stream=None):
    """dW = dz^T x in fp32; x a 16-bit tensor or an 8-bit checkpoint.  out: where it goes, for instance a
    view of a gradient buffer (added to with accumulate)."""
    c = _Call("pg_linear_weight_grad", dz, stream)
    eight = isinstance(x, Checkpoint8)
    t, n_out, n_in = c.tokens, c.cols, int((x.values if eight else x).shape[-1])
    if accumulate and out is None:
        _refuse(c.where, "accumulate needs out")
    dw = c.empty(n_out, n_in, torch.float32, 4) if out is None else out
    args = pg_weight_grad_args(c.kind, c.batch, t, n_in, n_out, int(accumulate), c.matrix(dz, t, n_out, c.dtype, "dz"),
                               c.matrix(None if eight else x, t, n_in, c.dtype, "x"), c.matrix8(x if eight else None, t, n_in, "x"),
                               c.matrix(dw, n_out, n_in, torch.float32, "out"))
    c.run(load_library().pg_linear_weight_grad, args, load_library().pg_linear_weight_grad_workspace_bytes)
    return dw


def pg_activation_grad(dy, z8: Optional[Checkpoint8], activation: str = "none", out=None, bias_grad=None,
                       accumulate: bool = False, stream=None):
    """(dz, dbias): dz = dy * activation'(z) and its sum over tokens.  z8 may be None for "none".
    bias_grad: where dbias goes (added to with accumulate)."""
    c = _Call("pg_activation_grad", dy, stream)
    t, n = c.tokens, c.cols
    if accumulate and bias_grad is None:
        _refuse(c.where, "accumulate needs bias_grad")
    dz = c.like(t, n) if out is None else out
    dbias = c.flat(n) if bias_grad is None else bias_grad
    dp, ds = c.vector(dbias, n, "bias_grad")
    args = pg_activation_grad_args(c.kind, _activation(c.where, activation), c.batch, t, n, int(accumulate),
                                   c.matrix(dy, t, n, c.dtype, "dy"), c.matrix8(z8, t, n, "z8"), c.matrix(dz, t, n, c.dtype, "out"), dp, ds)
    c.run(load_library().pg_activation_grad, args)
    return dz, dbias


def pg_checkpoint_write(x, out: Optional[Checkpoint8] = None, stream=None) -> Checkpoint8:
    """The 8-bit form of a 16-bit tensor."""
    c = _Call("pg_checkpoint_write", x, stream)
    x8 = c.empty8(c.tokens, c.cols) if out is None else out
    args = pg_checkpoint_args(c.kind, c.batch, c.tokens, c.cols, c.matrix(x, c.tokens, c.cols, c.dtype, "x"),
                              c.matrix8(x8, c.tokens, c.cols, "out"))
    c.run(load_library().pg_checkpoint_write, args)
    return x8


def pg_checkpoint_read(x8: Checkpoint8, out=None, stream=None):
    """The 16-bit tensor that an 8-bit form stands for."""
    c = _Call("pg_checkpoint_read", x8, stream)
    x = c.like(c.tokens, c.cols) if out is None else out
    args = pg_checkpoint_args(c.kind, c.batch, c.tokens, c.cols, c.matrix(x, c.tokens, c.cols, c.dtype, "out"),
                              c.matrix8(x8, c.tokens, c.cols, "x8"))
    c.run(load_library().pg_checkpoint_read, args)
    return x


def _ask(fn, stream, device) -> int:
    device = torch.device(device)
    with torch.cuda.device(device):
        handle = torch.cuda.current_stream(device).cuda_stream if stream is None else \
            stream if isinstance(stream, int) else stream.cuda_stream
        return int(fn(_vp(handle)))


def pg_training_status(stream=None, device="cuda") -> int:
    """Waits for `stream` (torch's current one if None) and returns PG_OK, or PG_ERR_TIMEOUT if a bounded
    device-side wait gave up on the device, on any stream, since the last call: outputs since then are not
    to be trusted.  No other call asks, so ask before results are used (once a step, say)."""
    return _ask(load_library().pg_training_status, stream, device)


def pg_selftest_training_timeout(stream=None, device="cuda") -> int:
    """Lets a bounded wait run out, within a millisecond; PG_ERR_TIMEOUT if that is reported."""
    return _ask(load_library().pg_selftest_training_timeout, stream, device)


def pg_selftest_training_bounds(stream=None, device="cuda") -> int:
    """PG_ERR_BOUNDS from the bounds-checked build, whose check it asks about an address outside; PG_OK elsewhere."""
    return _ask(load_library().pg_selftest_training_bounds, stream, device)
