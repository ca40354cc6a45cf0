"""Python binding of ``include/pg_training.h``: forward and backward pass of residual blocks for all
simulated workers at once (ctypes, same names as the C calls).

Tensors are CUDA tensors of shape (workers, tokens, features), or (tokens, features) for one worker;
16-bit ones are bf16 or fp16, the same in one call, with features contiguous and any row stride.
Weights are (workers, out, in), biases and gains fp32 (workers, n).  An axis of workers that was
expanded (stride 0) is shared by all workers.  Results are allocated with torch unless ``out`` is
given; their rows start on 16-byte boundaries, where every kernel takes its fastest path.

``stream`` is a torch stream or a raw handle; None means torch's current stream on the tensors'
device, and a call is then ordered like any torch operation.  On another stream the caller orders
inputs, and what this module allocates is kept from reuse until that stream has passed the call.

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


def _lib() -> ctypes.CDLL:
    return load_library()


def _refuse(where: str, why: str):
    raise ValueError("%s: %s" % (where, why))


class _Call:
    """Shape and device of one call, taken from its first tensor; checks the others against it."""

    def __init__(self, where: str, first, stream):
        dtype = getattr(first, "dtype", None)
        first = first.values if isinstance(first, Checkpoint8) else first
        if not isinstance(first, torch.Tensor) or not first.is_cuda or first.dim() not in (2, 3) or dtype not in _DTYPES:
            _refuse(where, "expected a bf16 or fp16 CUDA tensor of two or three dimensions")
        if max(first.shape) > 1 << 30:
            _refuse(where, "shape %s is too large" % (tuple(first.shape),))
        self.where, self.device, self.dtype = where, first.device, dtype
        self.single = first.dim() == 2
        self.batch = 1 if self.single else first.shape[0]
        self.tokens, self.cols = first.shape[-2:]
        current = torch.cuda.current_stream(self.device)
        self.other = None
        if stream is None:
            self.handle = current.cuda_stream
        else:
            self.handle = stream if isinstance(stream, int) else stream.cuda_stream
            if self.handle != current.cuda_stream:
                self.other = torch.cuda.ExternalStream(self.handle, device=self.device)

    def _own(self, t: torch.Tensor) -> torch.Tensor:
        if self.other is not None:
            t.record_stream(self.other)
        return t

    def matrix(self, t: Optional[torch.Tensor], rows: int, cols: int, dtype=None, name: str = "") -> pg_matrix:
        if t is None:
            return pg_matrix(None, cols, 0)
        dtype = dtype or self.dtype
        if not isinstance(t, torch.Tensor) or t.device != self.device or t.dtype != dtype:
            _refuse(self.where, "%s must be a %s tensor on %s" % (name, dtype, self.device))
        want = (rows, cols) if self.single else (self.batch, rows, cols)
        if t.dim() == 3 and self.single and t.shape[0] == 1:
            want = (1, rows, cols)
        if tuple(t.shape) != want:
            _refuse(self.where, "%s has shape %s, expected %s" % (name, tuple(t.shape), want))
        s = t.stride()
        if cols > 1 and s[-1] != 1:
            _refuse(self.where, "%s must have its last dimension contiguous" % name)
        ld = s[-2] if rows > 1 else max(cols, s[-2] if s[-2] >= cols else cols)
        return pg_matrix(t.data_ptr(), ld, s[0] if t.dim() == 3 and self.batch > 1 else 0)

    def matrix8(self, c: Optional[Checkpoint8], rows: int, cols: int, name: str = "") -> pg_matrix8:
        if c is None:
            return pg_matrix8(None, None, (cols + 15) // 16 * 16, 0, (cols + 31) // 32, 0)
        if c.dtype != self.dtype:
            _refuse(self.where, "%s is a checkpoint of %s, expected %s" % (name, c.dtype, self.dtype))
        v = self.matrix(c.values, rows, cols, torch.int8, name + ".values")
        s = self.matrix(c.scales, rows, (cols + BLOCK8 - 1) // BLOCK8, torch.uint8, name + ".scales")
        if rows <= 1:
            v.ld = (v.ld + 15) // 16 * 16
        return pg_matrix8(v.data, s.data, v.ld, v.stride, s.ld, s.stride)

    def vector(self, t: Optional[torch.Tensor], n: int, name: str):
        """(pointer, stride) of an fp32 (workers, n) tensor; (n,) for one worker or shared by all."""
        if t is None:
            return None, 0
        if not isinstance(t, torch.Tensor) or t.device != self.device or t.dtype != torch.float32 or t.shape[-1] != n \
                or t.dim() not in (1, 2) or (t.dim() == 2 and t.shape[0] != self.batch) or (n > 1 and t.stride(-1) != 1):
            _refuse(self.where, "%s must be an fp32 tensor of shape (%d, %d) on %s" % (name, self.batch, n, self.device))
        return t.data_ptr(), t.stride(0) if t.dim() == 2 and self.batch > 1 else 0

    def empty(self, rows: int, cols: int, dtype=None) -> torch.Tensor:
        """Rows start on 16-byte boundaries."""
        dtype = dtype or self.dtype
        unit = 4 if dtype == torch.float32 else 16 if dtype == torch.int8 else 8
        t = self._own(torch.empty((self.batch, rows, (cols + unit - 1) // unit * unit), dtype=dtype, device=self.device))
        if t.shape[-1] != cols:
            t = t[..., :cols]
        return t[0] if self.single else t

    def empty8(self, rows: int, cols: int) -> Checkpoint8:
        scales = self._own(torch.empty((self.batch, rows, (cols + BLOCK8 - 1) // BLOCK8), dtype=torch.uint8, device=self.device))
        return Checkpoint8(self.empty(rows, cols, torch.int8), scales[0] if self.single else scales, self.dtype)

    def flat(self, *shape: int, zero: bool = False) -> torch.Tensor:
        shape = shape[1:] if self.single else shape
        return self._own((torch.zeros if zero else torch.empty)(shape, dtype=torch.float32, device=self.device))

    def run(self, fn, args, size_fn=None) -> None:
        with torch.cuda.device(self.device):
            if size_fn is None:
                _check(fn(ctypes.byref(args), _vp(self.handle)), self.where)
                return
            need = ctypes.c_size_t(0)
            _check(size_fn(ctypes.byref(args), ctypes.byref(need)), self.where)
            scratch = None
            if need.value:
                scratch = self._own(torch.empty(need.value, dtype=torch.uint8, device=self.device))
            _check(fn(ctypes.byref(args), _vp(scratch.data_ptr() if need.value else None), ctypes.c_size_t(need.value),
                      _vp(self.handle)), self.where)


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
    h = x if residual is None else c.empty(t, n)
    y = c.empty(t, n) if out is None else out
    y8 = c.empty8(t, n) if eight_bit else None
    h8 = c.empty8(t, n) if save_h8 else None
    rstd = c.flat(c.batch, t)
    gp, gs = c.vector(gain, n, "gain")
    args = pg_norm_args(_DTYPES[c.dtype], c.batch, t, n, eps, c.matrix(x, t, n, name="x"),
                        c.matrix(residual, t, n, name="residual"), gp, gs,
                        c.matrix(None if residual is None else h, t, n, name="h"), c.matrix(y, t, n, name="out"),
                        c.matrix8(y8, t, n), c.matrix8(h8, t, n), rstd.data_ptr())
    c.run(_lib().pg_add_rms_norm, args)
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
    dx = c.empty(t, n) if out is None else out
    dgain = c.flat(c.batch, n) if gain_grad is None else gain_grad
    if not isinstance(rstd, torch.Tensor) or rstd.device != c.device or rstd.dtype != torch.float32 or rstd.numel() != c.batch * t \
            or not rstd.is_contiguous():
        _refuse(c.where, "rstd must be a contiguous fp32 tensor of %d x %d on %s" % (c.batch, t, c.device))
    eight = isinstance(h, Checkpoint8)
    gp, gs = c.vector(gain, n, "gain")
    dp, ds = c.vector(dgain, n, "gain_grad")
    args = pg_norm_grad_args(_DTYPES[c.dtype], c.batch, t, n, int(accumulate), c.matrix(dy, t, n, name="dy"),
                             c.matrix(None if eight else h, t, n, name="h"), c.matrix8(h if eight else None, t, n, "h"),
                             rstd.data_ptr(), gp, gs, c.matrix(dh, t, n, name="dh"), c.matrix(dx, t, n, name="out"), dp, ds)
    c.run(_lib().pg_add_rms_norm_grad, args, _lib().pg_add_rms_norm_grad_workspace_bytes)
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
    y = c.empty(t, n_out) if out is None else out
    z8 = c.empty8(t, n_out) if save_z else None
    bp, bs = c.vector(bias, n_out, "bias")
    args = pg_linear_args(_DTYPES[c.dtype], _activation(c.where, activation), c.batch, t, n_in, n_out,
                          c.matrix(x, t, n_in, name="x"), c.matrix(weight, n_out, n_in, name="weight"), bp, bs,
                          c.matrix(residual, t, n_out, name="residual"), c.matrix(y, t, n_out, name="out"), c.matrix8(z8, t, n_out))
    c.run(_lib().pg_linear, args, _lib().pg_linear_workspace_bytes)
    return (y, z8) if save_z else y


def pg_linear_input_grad(dz, weight, residual=None, out=None, stream=None):
    """dx = dz W + residual."""
    c = _Call("pg_linear_input_grad", dz, stream)
    n_out, n_in = _weight(c, weight, False)
    t = c.tokens
    dx = c.empty(t, n_in) if out is None else out
    args = pg_input_grad_args(_DTYPES[c.dtype], c.batch, t, n_in, n_out, c.matrix(dz, t, n_out, name="dz"),
                              c.matrix(weight, n_out, n_in, name="weight"), c.matrix(residual, t, n_in, name="residual"),
                              c.matrix(dx, t, n_in, name="out"))
    c.run(_lib().pg_linear_input_grad, args, _lib().pg_linear_input_grad_workspace_bytes)
    return dx


def pg_linear_weight_grad(dz, x: Union[torch.Tensor, Checkpoint8], out=None, accumulate: bool = False, stream=None):
    """dW = dz^T x in fp32; x a 16-bit tensor or an 8-bit checkpoint.  out: where it goes, for instance a
    view of a gradient buffer (added to with accumulate)."""
    c = _Call("pg_linear_weight_grad", dz, stream)
    eight = isinstance(x, Checkpoint8)
    t, n_out, n_in = c.tokens, c.cols, int((x.values if eight else x).shape[-1])
    if accumulate and out is None:
        _refuse(c.where, "accumulate needs out")
    dw = c.empty(n_out, n_in, torch.float32) if out is None else out
    args = pg_weight_grad_args(_DTYPES[c.dtype], c.batch, t, n_in, n_out, int(accumulate), c.matrix(dz, t, n_out, name="dz"),
                               c.matrix(None if eight else x, t, n_in, name="x"), c.matrix8(x if eight else None, t, n_in, "x"),
                               c.matrix(dw, n_out, n_in, torch.float32, "out"))
    c.run(_lib().pg_linear_weight_grad, args, _lib().pg_linear_weight_grad_workspace_bytes)
    return dw


def pg_activation_grad(dy, z8: Optional[Checkpoint8], activation: str = "none", out=None, bias_grad=None,
                       accumulate: bool = False, stream=None):
    """(dz, dbias): dz = dy * activation'(z) and its sum over tokens.  z8 may be None for "none".
    bias_grad: where dbias goes (added to with accumulate)."""
    c = _Call("pg_activation_grad", dy, stream)
    t, n = c.tokens, c.cols
    if accumulate and bias_grad is None:
        _refuse(c.where, "accumulate needs bias_grad")
    dz = c.empty(t, n) if out is None else out
    dbias = c.flat(c.batch, n) if bias_grad is None else bias_grad
    dp, ds = c.vector(dbias, n, "bias_grad")
    args = pg_activation_grad_args(_DTYPES[c.dtype], _activation(c.where, activation), c.batch, t, n, int(accumulate),
                                   c.matrix(dy, t, n, name="dy"), c.matrix8(z8, t, n, "z8"), c.matrix(dz, t, n, name="out"), dp, ds)
    c.run(_lib().pg_activation_grad, args)
    return dz, dbias


def pg_checkpoint_write(x, out: Optional[Checkpoint8] = None, stream=None) -> Checkpoint8:
    """The 8-bit form of a 16-bit tensor."""
    c = _Call("pg_checkpoint_write", x, stream)
    x8 = c.empty8(c.tokens, c.cols) if out is None else out
    args = pg_checkpoint_args(_DTYPES[c.dtype], c.batch, c.tokens, c.cols, c.matrix(x, c.tokens, c.cols, name="x"),
                              c.matrix8(x8, c.tokens, c.cols, "out"))
    c.run(_lib().pg_checkpoint_write, args)
    return x8


def pg_checkpoint_read(x8: Checkpoint8, out=None, stream=None):
    """The 16-bit tensor that an 8-bit form stands for."""
    c = _Call("pg_checkpoint_read", x8, stream)
    x = c.empty(c.tokens, c.cols) if out is None else out
    args = pg_checkpoint_args(_DTYPES[c.dtype], c.batch, c.tokens, c.cols, c.matrix(x, c.tokens, c.cols, name="out"),
                              c.matrix8(x8, c.tokens, c.cols, "x8"))
    c.run(_lib().pg_checkpoint_read, args)
    return x


def pg_training_status(stream=None, device="cuda") -> int:
    """Waits for `stream` (torch's current one if None) and returns PG_OK, or PG_ERR_TIMEOUT if a bounded
    device-side wait gave up since the last call."""
    device = torch.device(device)
    with torch.cuda.device(device):
        handle = torch.cuda.current_stream(device).cuda_stream if stream is None else \
            stream if isinstance(stream, int) else stream.cuda_stream
        return int(_lib().pg_training_status(_vp(handle)))
