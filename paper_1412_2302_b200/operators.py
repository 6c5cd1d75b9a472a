"""Operators on the caller's CUDA tensors, next to those that run inside a handle: group normalisation with an activation, 8-bit
activation checkpoints, and the weight gradient of a linear layer from such a checkpoint (include/alexnet.h, the last part).

    r = group_norm(x, groups, weight, bias, activation="silu", keep_input="int8")      # r.y, r.mean, r.rstd, r.input
    dx, dweight, dbias = group_norm_backward(dy, r.input, r.mean, r.rstd, weight, bias, activation="silu")
    kept = checkpoint_encode(h, "e4m3")
    dw = linear_weight_grad(dz, kept)

Tensors are channels-last: [n, h, w, c], [n, l, c] or [n, c] (`checkpoint_*` and `linear_weight_grad`: any number of leading dimensions that
form rows) with adjacent channels, dense or a view of a larger grid; bfloat16, float16 or float32.  Weights, biases, statistics and their
gradients are float32.  Every call queues its work on `stream` (a torch.cuda.Stream; default: the current stream of the tensors' device)
and returns without waiting; tensors that are let go before that stream has passed the call need their record_stream, as with any
other work on a stream of one's own.  Outputs and workspace come from torch's allocator on that stream unless `out` gives the output.  A wrong
argument raises AlexNetError with code ERR_ARG before anything is launched.  There is no CPU fallback.

Autograd does not see these calls: gradients come from group_norm_backward and linear_weight_grad, which the caller puts in their places (in the
backward of a torch.autograd.Function, for instance).  So that none is lost in silence, a y of inputs that require a gradient requires one too, and a
backward pass that comes to it raises AlexNetError.  (An `out` stays as it is.)
"""
from __future__ import annotations

import ctypes
import functools
import operator
import struct
import threading
from typing import NamedTuple, Optional

import torch

from . import alexnet as _alexnet
from .alexnet import ERR_ARG, OK, AlexNetError

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2}
FORMATS = {"int8": 1, "e4m3": 2}
CODE_DTYPES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
_FORMAT_OF = {dtype: name for name, dtype in CODE_DTYPES.items()}

# the argument blocks of include/alexnet.h (all fields naturally aligned)
_NORM = "q4i2ifi"
_VIEW = "P3q"
_KEPT = "2P2i"
_pack_shape = struct.Struct("=" + _NORM.replace("P", "Q")).pack
_pack_checkpoint = struct.Struct(("=q4i" + _VIEW + _KEPT).replace("P", "Q")).pack
_pack_forward = struct.Struct(("=" + _NORM + 2 * _VIEW + "4P" + 2 * _KEPT + "PQ").replace("P", "Q")).pack
_pack_backward = struct.Struct(("=" + _NORM + 3 * _VIEW + _KEPT + "6PPQ").replace("P", "Q")).pack
_pack_linear = struct.Struct(("=q2iPq" + _KEPT + "PPQ").replace("P", "Q")).pack

_local = threading.local()


class Checkpoint:
    """codes (int8 or float8_e4m3fn, the shape of the tensor) and scales (uint8, one exponent byte per 32 channels, rounded up): both dense."""
    __slots__ = ("codes", "scales")

    def __init__(self, codes, scales):
        if codes.dtype not in _FORMAT_OF or scales.dtype != torch.uint8:
            raise AlexNetError(ERR_ARG, "a checkpoint's codes are int8 or float8_e4m3fn and its scales uint8")
        if codes.dim() < 1 or scales.shape != (*codes.shape[:-1], (codes.shape[-1] + 31) // 32):
            raise AlexNetError(ERR_ARG, f"scales {tuple(scales.shape)} do not fit codes {tuple(codes.shape)}: one per 32 channels, rounded up")
        if codes.device != scales.device or not codes.is_contiguous() or not scales.is_contiguous():
            raise AlexNetError(ERR_ARG, "a checkpoint's codes and scales are dense and on one device")
        self.codes, self.scales = codes, scales

    @property
    def format(self):
        return _FORMAT_OF[self.codes.dtype]

    @property
    def shape(self):
        return self.codes.shape

    @property
    def nbytes(self):
        return self.codes.numel() + self.scales.numel()


class GroupNormResult(NamedTuple):
    y: torch.Tensor
    mean: torch.Tensor                      # [n, groups]
    rstd: torch.Tensor
    input: Optional[Checkpoint] = None      # of x, when keep_input was given
    output: Optional[Checkpoint] = None     # of y, when keep_output was given


def _refuse(message):
    raise AlexNetError(ERR_ARG, message)


def _name(table, key, what):
    try:
        return table[key]
    except (KeyError, TypeError):
        _refuse(f"unknown {what} {key!r}: one of {', '.join(map(str, table))}")


# The calls below cost the host 9 to 20 us, most of it in the tensors they create and the launches; so they are written without helper objects.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _raw_stream(index):
    return torch.cuda.current_stream(index).cuda_stream


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _raw_stream)


def _elsewhere(index, stream):
    """The context in which to repeat a call whose tensors are not on the current device, or that was given a stream."""
    if index < 0:
        _refuse("the tensors must be on a CUDA device (there is no CPU fallback)")
    if stream is None:
        return torch.cuda.device(index)
    if stream.device.index != index:
        _refuse(f"the stream belongs to {stream.device}, the tensors are on cuda:{index}")
    return torch.cuda.stream(stream)                # sets the device too


def _pack(pack, *fields):
    try:
        return pack(*fields)
    except (struct.error, OverflowError):
        _refuse("a size, a stride or eps is not a number that the library's arguments hold")


def _run(function, index, pack, *fields):
    err = getattr(_local, "err", None)
    if err is None:
        err = _local.err = ctypes.create_string_buffer(256)
    rc = function(_pack(pack, *fields), _raw_stream(index), err, 256)
    if rc != OK:
        raise AlexNetError(rc, err.value.decode())


def _other_device():
    _refuse("all tensors of a call must be on one device")


def _rows(t, what):
    """(n, h, w, c) and the strides of n, h, w of a channels-last tensor of two to four dimensions."""
    shape, st = t.shape, t.stride()
    d = len(shape)
    if d == 4:
        if st[3] != 1 and shape[3] > 1:
            _refuse(f"the channels of {what} are not adjacent")
        return shape, st[:3]
    if d < 2 or d > 4:
        _refuse(f"{what} has {d} dimensions: [n, h, w, c], [n, l, c] or [n, c] is wanted")
    if st[-1] != 1 and shape[-1] > 1:
        _refuse(f"the channels of {what} are not adjacent")
    if d == 3:
        return (shape[0], 1, shape[1], shape[2]), (st[0], 0, st[1])
    return (shape[0], 1, 1, shape[1]), (st[0], 0, 0)


def _rows_any(t, what):
    """The same for a checkpoint: more leading dimensions, or none, are folded where they are dense."""
    if t.dim() > 4:
        if not t.is_contiguous():
            _refuse(f"{what} has {t.dim()} dimensions and is not dense")
        if t.shape[-1] == 0:
            _refuse(f"{what} has no channels")
        t = t.view(-1, t.shape[-1])
    elif t.dim() == 1:
        t = t.view(1, -1)
    elif t.dim() == 0:
        _refuse(f"{what} has no channels")
    return _rows(t, what)


def _vector(t, n, what, index):
    if t is None:
        return 0
    if t.dtype is not torch.float32 or t.dim() != 1 or t.numel() != n or not t.is_contiguous():
        _refuse(f"{what} must be a dense float32 vector of {n}")
    if t.get_device() != index:
        _other_device()
    return t.data_ptr()


def _dense_like(t):
    """a dense tensor of t's shape and type (of a dense one empty_like is the cheapest)"""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _output(out, shape, dtype, index):
    if out.dtype is not dtype or out.shape != shape:
        _refuse(f"out must be {dtype} {tuple(shape)}, not {out.dtype} {tuple(out.shape)}")
    if out.get_device() != index:
        _other_device()
    return out


class _NoGradient(torch.autograd.Function):
    """y as it is, in the place where its gradient would be wanted; `leaf` is there to require it."""

    @staticmethod
    def forward(ctx, y, leaf):
        ctx.mark_dirty(y)
        return y

    @staticmethod
    def backward(ctx, dy):
        _refuse("group_norm has no gradient of its own: call group_norm_backward with this dy, for instance in the backward of a torch.autograd.Function")


def _without_gradient(y):
    return _NoGradient.apply(y, torch.empty(0, requires_grad=True))


def _new_checkpoint(x, fmt):
    shape = x.shape
    k = Checkpoint.__new__(Checkpoint)
    dtype = _name(CODE_DTYPES, fmt, "checkpoint format")
    k.codes = torch.empty_like(x, dtype=dtype) if x.is_contiguous() else x.new_empty(shape, dtype=dtype)
    k.scales = x.new_empty((*shape[:-1], (shape[-1] + 31) // 32), dtype=torch.uint8)
    return k


_NOT_KEPT = (0, 0, 0, 0)


def _kept(k):
    return k.codes.data_ptr(), k.scales.data_ptr(), FORMATS[_FORMAT_OF[k.codes.dtype]], 0


def _norm_bytes(n, shape):
    if n == 0:
        raise AlexNetError(ERR_ARG, f"invalid group norm: n, h, w, channels, groups = {tuple(shape[:5])}, eps = {shape[7]}")
    return n if n > 256 else 0


def _norm_workspace(shape, backward):
    """bytes of workspace for the sizes, whatever the tensors (0: no call needs any)"""
    return _norm_bytes(int(_alexnet.load_library().alexnet_group_norm_workspace_bytes(_pack(_pack_shape, *shape), backward)), shape)


# by sizes, strides and alignment: the pointers are given modulo 16
@functools.lru_cache(maxsize=1024)
def _forward_workspace(shape, x, xs, y, ys):
    return _norm_bytes(int(_alexnet.load_library().alexnet_group_norm_forward_workspace_bytes(
        _pack(_pack_forward, *shape, x, *xs, y, *ys, 0, 0, 0, 0, *_NOT_KEPT, *_NOT_KEPT, 0, 0))), shape)


@functools.lru_cache(maxsize=1024)
def _backward_workspace(shape, dy, ds, x, xs, dx, dxs, codes, fmt):
    return _norm_bytes(int(_alexnet.load_library().alexnet_group_norm_backward_workspace_bytes(
        _pack(_pack_backward, *shape, dy, *ds, x, *xs, dx, *dxs, codes, 16 if fmt else 0, fmt, 0, 0, 0, 0, 0, 0, 0, 0, 0))), shape)


@functools.lru_cache(maxsize=1024)
def _linear_workspace(rows, n_in, n_out, stride, dy_offset, codes_offset, fmt):
    """by sizes and alignment: the pointers are given modulo 16"""
    n = int(_alexnet.load_library().alexnet_linear_weight_grad_workspace_bytes(
        _pack(_pack_linear, rows, n_in, n_out, 16 + dy_offset, stride, 16 + codes_offset, 16, fmt, 0, 0, 0, 0)))
    if n == 0:
        raise AlexNetError(ERR_ARG, f"invalid linear weight gradient: rows, in, out = {rows, n_in, n_out}, stride {stride}")
    return n if n > 256 else 0


def check():
    """Wait for all work of the current device, on whatever stream, and raise if a bounded wait inside an operator's kernel has ever run out (its
    outputs are NaN)."""
    rc = _alexnet.load_library().alexnet_operators_check()
    if rc != OK:
        raise AlexNetError(rc, "a wait inside an operator's kernel ran out" if rc == _alexnet.ERR_DEVICE_TIMEOUT else "the device could not be read")


def checkpoint_encode(x, format="int8", out=None, stream=None):
    """The 8-bit checkpoint of x: 33 bytes for 32 values.  out: a Checkpoint to write instead of a new one."""
    index = x.get_device()
    if stream is not None or index < 0 or index != _current_device():
        with _elsewhere(index, stream):
            return checkpoint_encode(x, format, out)
    dtype = _name(DTYPES, x.dtype, "dtype")
    (n, h, w, c), st = _rows_any(x, "x")
    if out is None:
        out = _new_checkpoint(x, format)
    else:
        if out.shape != x.shape or out.codes.dtype != _name(CODE_DTYPES, format, "checkpoint format"):
            _refuse("out is a checkpoint of another shape or format")
        if out.codes.get_device() != index:
            _other_device()
    _run(_alexnet.load_library().alexnet_checkpoint_encode, index, _pack_checkpoint, n, h, w, c, dtype, x.data_ptr(), *st, *_kept(out))
    return out


def checkpoint_decode(checkpoint, dtype=torch.bfloat16, out=None, stream=None):
    """The values that a checkpoint stands for, rounded to dtype (exact in float32 and, but for e4m3 values below 2^-116, in bfloat16)."""
    codes = checkpoint.codes
    index = codes.get_device()
    if stream is not None or index < 0 or index != _current_device():
        with _elsewhere(index, stream):
            return checkpoint_decode(checkpoint, dtype, out)
    code = _name(DTYPES, dtype, "dtype")
    out = codes.new_empty(codes.shape, dtype=dtype) if out is None else _output(out, codes.shape, dtype, index)
    (n, h, w, c), st = _rows_any(out, "out")
    _run(_alexnet.load_library().alexnet_checkpoint_decode, index, _pack_checkpoint, n, h, w, c, code, out.data_ptr(), *st, *_kept(checkpoint))
    return out


def group_norm(x, groups, weight=None, bias=None, eps=1e-5, activation="none", keep_input=None, keep_output=None, out=None, stream=None):
    """y = act((x - mean) rstd weight + bias) with the statistics of a group of channels over all positions of a sample.  A group with an
    infinity or a NaN has statistics and results of NaN; values are below 2^76 in magnitude.

    x [n, h, w, c], [n, l, c] or [n, c]; activation "none", "relu" or "silu"; keep_input / keep_output: "int8" or "e4m3" writes a
    checkpoint of x (what group_norm_backward needs) or of y (what the weight gradient of a layer behind needs) on the way."""
    index = x.get_device()
    if stream is not None or index < 0 or index != _current_device():
        with _elsewhere(index, stream):
            return group_norm(x, groups, weight, bias, eps, activation, keep_input, keep_output, out)
    if type(groups) is not int or type(eps) is not float:
        try:
            groups, eps = operator.index(groups), float(eps)
        except (TypeError, ValueError):
            _refuse(f"groups must be an integer and eps a number, not {groups!r} and {eps!r}")
    (n, h, w, c), xs = _rows(x, "x")
    shape = (n, h, w, c, groups, _name(DTYPES, x.dtype, "dtype"), _name(ACTIVATIONS, activation, "activation"), eps, 0)
    px = x.data_ptr()
    if out is None:                                 # (asked before y is created: a shape may be refused)
        ys = (h * w * c, w * c, c)
        nbytes = _forward_workspace(shape, px % 16, xs, 0, ys)
        y = _dense_like(x)
        py = y.data_ptr()
    else:
        y = _output(out, x.shape, x.dtype, index)
        py, ys = y.data_ptr(), _rows(y, "out")[1]
        nbytes = _forward_workspace(shape, px % 16, xs, py % 16, ys)
    mean = x.new_empty((n, groups), dtype=torch.float32)
    rstd = torch.empty_like(mean)
    kx = ky = None
    pkx = pky = _NOT_KEPT
    if keep_input is not None:
        kx = _new_checkpoint(x, keep_input)
        pkx = _kept(kx)
    if keep_output is not None:
        ky = _new_checkpoint(x, keep_output)
        pky = _kept(ky)
    ws = x.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    _run(_alexnet.load_library().alexnet_group_norm_forward, index, _pack_forward,
         *shape, px, *xs, py, *ys, _vector(weight, c, "weight", index), _vector(bias, c, "bias", index), mean.data_ptr(), rstd.data_ptr(),
         *pkx, *pky, 0 if ws is None else ws.data_ptr(), nbytes)
    if out is None and torch.is_grad_enabled() and (x.requires_grad or (weight is not None and weight.requires_grad) or (bias is not None and bias.requires_grad)):
        y = _without_gradient(y)
    return GroupNormResult(y, mean, rstd, kx, ky)


def group_norm_backward(dy, x, mean, rstd, weight=None, bias=None, activation="none", out=None, stream=None):
    """(dx, dweight, dbias) of group_norm for the gradient dy of y.  x: the tensor that group_norm was given, or a Checkpoint of it; mean and
    rstd [n, groups] as group_norm returned them.  out: the tensor that takes dx."""
    index = dy.get_device()
    if stream is not None or index < 0 or index != _current_device():
        with _elsewhere(index, stream):
            return group_norm_backward(dy, x, mean, rstd, weight, bias, activation, out)
    (n, h, w, c), ds = _rows(dy, "dy")
    if x.shape != dy.shape:
        _refuse(f"x {tuple(x.shape)} and dy {tuple(dy.shape)} differ in shape")
    if isinstance(x, Checkpoint):
        kept, xv = _kept(x), _NOT_KEPT
        other = x.codes.get_device() != index
    else:
        if x.dtype is not dy.dtype:
            _refuse(f"x is {x.dtype}, dy {dy.dtype}")
        kept, xv = _NOT_KEPT, (x.data_ptr(), *_rows(x, "x")[1])
        other = x.get_device() != index
    if mean.dim() != 2 or mean.shape[0] != n or mean.dtype is not torch.float32 or rstd.shape != mean.shape or rstd.dtype is not torch.float32 \
            or not mean.is_contiguous() or not rstd.is_contiguous():
        _refuse("mean and rstd must be dense float32 [n, groups]")
    if other or mean.get_device() != index or rstd.get_device() != index:
        _other_device()
    shape = (n, h, w, c, mean.shape[1], _name(DTYPES, dy.dtype, "dtype"), _name(ACTIVATIONS, activation, "activation"), 1.0, 0)
    pdy = dy.data_ptr()
    if out is None:
        dxs = (h * w * c, w * c, c)
        nbytes = _backward_workspace(shape, pdy % 16, ds, xv[0] % 16, xv[1:], 0, dxs, kept[0] % 16, kept[2])
        dx = _dense_like(dy)
        pdx = dx.data_ptr()
    else:
        dx = _output(out, dy.shape, dy.dtype, index)
        pdx, dxs = dx.data_ptr(), _rows(dx, "out")[1]
        nbytes = _backward_workspace(shape, pdy % 16, ds, xv[0] % 16, xv[1:], pdx % 16, dxs, kept[0] % 16, kept[2])
    dweight = dy.new_empty(c, dtype=torch.float32)
    dbias = torch.empty_like(dweight)
    ws = dy.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    _run(_alexnet.load_library().alexnet_group_norm_backward, index, _pack_backward,
         *shape, pdy, *ds, *xv, pdx, *dxs, *kept, mean.data_ptr(), rstd.data_ptr(), _vector(weight, c, "weight", index),
         _vector(bias, c, "bias", index), dweight.data_ptr(), dbias.data_ptr(), 0 if ws is None else ws.data_ptr(), nbytes)
    return dx, dweight, dbias


def linear_weight_grad(dy, x, out=None, stream=None):
    """dw [out features, in features] = dy^T x, float32, for dy bfloat16 [..., out features] and a Checkpoint x of [..., in features]."""
    if not isinstance(x, Checkpoint):
        _refuse("x must be a Checkpoint")
    if dy.dtype is not torch.bfloat16:
        _refuse(f"dy must be bfloat16, not {dy.dtype}")
    codes = x.codes
    if dy.dim() < 1 or dy.shape[:-1] != codes.shape[:-1]:
        _refuse(f"dy {tuple(dy.shape)} and x {tuple(codes.shape)} differ in their rows")
    index = dy.get_device()
    if stream is not None or index < 0 or index != _current_device():
        with _elsewhere(index, stream):
            return linear_weight_grad(dy, x, out)
    n_in, n_out = codes.shape[-1], dy.shape[-1]
    if n_in == 0 or n_out == 0:
        _refuse(f"features must be 1 to 1048576, not {n_in} and {n_out}")
    if dy.dim() != 2:
        if not dy.is_contiguous():
            _refuse("dy of other than two dimensions must be dense")
        dy = dy.view(-1, n_out)
    rows, (stride, last) = dy.shape[0], dy.stride()
    if last != 1 and n_out > 1:
        _refuse("the features of dy are not adjacent")
    if codes.get_device() != index:
        _other_device()
    if out is None:
        dw = dy.new_empty((n_out, n_in), dtype=torch.float32)
    else:
        dw = _output(out, (n_out, n_in), torch.float32, index)
        if not dw.is_contiguous():
            _refuse("out must be dense")
    p, q = dy.data_ptr(), codes.data_ptr()
    nbytes = _linear_workspace(rows, n_in, n_out, stride, p % 16, q % 16, FORMATS[x.format])
    ws = dy.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    _run(_alexnet.load_library().alexnet_linear_weight_grad, index, _pack_linear,
         rows, n_in, n_out, p, stride, *_kept(x), dw.data_ptr(), 0 if ws is None else ws.data_ptr(), nbytes)
    return dw
