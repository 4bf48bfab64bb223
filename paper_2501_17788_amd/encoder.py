"""The operators of a token encoder's head, on torch device tensors: layer norm with its gradients,
products of 8-bit rows, and the AdamW step.

As in `warp`, everything runs in the HIP kernels behind the C ABI of include/warp.h; this module checks
tensors, allocates outputs with torch and passes pointers. A call works on the current stream of its
tensors' device, or on `stream`; inputs of another stream are the caller's to wait for. Tensors have
any row stride (a dimension's elements one after the other); leading dimensions are flattened to rows.
"""
from __future__ import annotations

import ctypes
import operator
from typing import NamedTuple

import numpy as np
import torch

from .warp import _check, lib

_NONE = type(None)
_dtype_of = operator.attrgetter("dtype")
_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}  # WARP_F32, WARP_F16, WARP_BF16
PAD = 128    # int8 rows are padded with zeros to a multiple of this width
BLOCK = 256  # elements of a tensor that share a scale of 8-bit moments


class QuantizedRows(NamedTuple):
    """Rows of 8-bit integers: values [rows, width] int8, of which the first `cols` columns count and the
    others, up to a multiple of 128, are zeros; scale [rows] float32. A row stands for values * scale."""
    values: torch.Tensor
    scale: torch.Tensor
    cols: int

    @classmethod
    def from_int8(cls, values, scale) -> "QuantizedRows":
        """Rows quantised elsewhere: int8 [rows, cols] and float32 [rows] device tensors, copied."""
        if values.dim() != 2 or values.dtype != torch.int8 or scale.shape != values.shape[:1]:
            raise ValueError("from_int8 needs int8 values [rows, cols] and a scale for each row")
        rows, cols = values.shape
        padded = torch.zeros((rows, -(-cols // PAD) * PAD), dtype=torch.int8, device=values.device)
        padded[:, :cols] = values
        return cls(padded, scale.to(torch.float32).contiguous(), cols)


_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _here(first, *others):
    """The current stream's handle, if that is where a call on these tensors works; None if their device is not
    the current one. What torch.cuda.current_stream() gives, without making a Python object of it."""
    index = first.get_device()
    for t in others:
        if t is not None and t.get_device() != index:
            raise ValueError(f"expected tensors on {first.device}, got {t.device}")
    if index < 0:
        raise ValueError(f"expected device tensors, got {first.device}")
    return _raw_stream(index) if index == _device() else None


def _there(stream, tensors, call, *args):
    """call(*args) with `stream` (or the current one of the tensors' device) current, so that outputs and copies
    are allocated and enqueued there; the tensors are kept for its work."""
    dev = tensors[0].device
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise ValueError(f"expected device tensors, got {t.device}")
    stream = torch.cuda.current_stream(dev) if stream is None else stream
    with torch.cuda.device(dev), torch.cuda.stream(stream):
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
        return call(*args)


def _rows(x, name):
    """(x or a copy whose rows have contiguous elements, number of rows, row stride) of x [..., cols]."""
    if x.dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32, float16 or bfloat16, got {x.dtype}")
    shape = x.shape
    if len(shape) == 2:
        rows, cols = shape
        stride, inner = x.stride()
        if (inner == 1 or cols == 1) and (stride >= cols or rows <= 1):
            return x, rows, stride
    elif not shape:
        raise ValueError(f"{name} must have at least one dimension")
    x = x.contiguous()
    cols = shape[-1]
    if cols < 1:
        raise ValueError(f"{name} has rows of no columns")
    return x, x.numel() // cols, cols


def _params(x, weight, bias):
    """weight and bias as the kernels take them, and their dtype."""
    shape, dtype = x.shape[-1:], None
    if weight is not None:
        if weight.shape != shape:
            raise ValueError(f"weight must have shape {tuple(shape)}, got {tuple(weight.shape)}")
        weight, dtype = weight.contiguous(), weight.dtype
    if bias is not None:
        if bias.shape != shape:
            raise ValueError(f"bias must have shape {tuple(shape)}, got {tuple(bias.shape)}")
        if dtype is not None and bias.dtype is not dtype:
            raise ValueError(f"weight and bias must be of one type, got {dtype} and {bias.dtype}")
        bias, dtype = bias.contiguous(), bias.dtype
    if dtype is None:
        dtype = torch.float32
    elif dtype is not torch.float32 and dtype is not x.dtype:
        raise ValueError(f"weight and bias must be float32 or {x.dtype}, got {dtype}")
    return weight, bias, dtype


def _ptr(t):
    return None if t is None else t.data_ptr()


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, stream=None):
    """Layer norm over the last dimension of x [..., cols]: (y like x, mean, rstd), the row statistics in
    float32 [...] for `layer_norm_backward`. weight and bias [cols] are float32 or of x's type."""
    s = _here(x, weight, bias) if stream is None else None
    if s is None:
        return _there(stream, (x, weight, bias), layer_norm, x, weight, bias, eps)
    weight, bias, pt = _params(x, weight, bias)
    x, rows, stride = _rows(x, "x")
    shape = x.shape
    cols = shape[-1]
    y = torch.empty_like(x) if x.is_contiguous() else torch.empty(shape, dtype=x.dtype, device=x.device)
    mean, rstd = torch.empty((2, *shape[:-1]), dtype=torch.float32, device=x.device).unbind(0)
    _check(lib.warp_layer_norm(x.data_ptr(), stride, rows, cols, _DTYPES[x.dtype], _ptr(weight), _ptr(bias),
                               _DTYPES[pt], eps, y.data_ptr(), cols, mean.data_ptr(), rstd.data_ptr(), s))
    return y, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd, stream=None):
    """Gradients (dx, dweight, dbias) of `layer_norm` for the gradient dy of its y. dweight and dbias have
    weight's type (float32 without a weight)."""
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError(f"dy must be like x ({tuple(x.shape)}, {x.dtype}), got {tuple(dy.shape)}, {dy.dtype}")
    for name, t in (("mean", mean), ("rstd", rstd)):
        if t.shape != x.shape[:-1] or t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError(f"{name} must be what layer_norm gave: contiguous float32 {tuple(x.shape[:-1])}")
    s = _here(x, dy, weight, mean, rstd) if stream is None else None
    if s is None:
        return _there(stream, (x, dy, weight, mean, rstd), layer_norm_backward, dy, x, weight, mean, rstd)
    weight, _, pt = _params(x, weight, None)
    x, rows, stride = _rows(x, "x")
    dy, _, dy_stride = _rows(dy, "dy")
    cols = x.shape[-1]
    need = ctypes.c_int64()
    _check(lib.warp_layer_norm_backward_scratch(rows, cols, _DTYPES[x.dtype], ctypes.byref(need)))
    dx = torch.empty_like(x) if x.is_contiguous() else torch.empty(x.shape, dtype=x.dtype, device=x.device)
    dw, db = torch.empty((2, cols), dtype=pt, device=x.device).unbind(0)
    scratch = torch.empty(need.value, dtype=torch.uint8, device=x.device)
    _check(lib.warp_layer_norm_backward(dy.data_ptr(), dy_stride, x.data_ptr(), stride, rows, cols, _DTYPES[x.dtype],
                                        _ptr(weight), _DTYPES[pt], mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(),
                                        cols, dw.data_ptr(), db.data_ptr(), scratch.data_ptr(), need.value, s))
    return dx, dw, db


def _int8_out(x, rows):
    q = torch.empty((rows, -(-x.shape[-1] // PAD) * PAD), dtype=torch.int8, device=x.device)
    return q, torch.empty(rows, dtype=torch.float32, device=x.device)


def quantize_rows(x, stream=None) -> QuantizedRows:
    """Rows of x [..., cols] in 8 bits with a scale each: token activations, or a weight [n, cols] with a
    scale for each output channel."""
    s = _here(x) if stream is None else None
    if s is None:
        return _there(stream, (x,), quantize_rows, x)
    x, rows, stride = _rows(x, "x")
    cols = x.shape[-1]
    q, scale = _int8_out(x, rows)
    _check(lib.warp_quantize_rows(x.data_ptr(), stride, rows, cols, _DTYPES[x.dtype], q.data_ptr(), q.shape[1],
                                  scale.data_ptr(), s))
    return QuantizedRows(q, scale, cols)


def layer_norm_int8(x, weight=None, bias=None, eps: float = 1e-5, stream=None) -> QuantizedRows:
    """`quantize_rows` of `layer_norm`'s rows in one pass, without rounding them to x's type in between."""
    s = _here(x, weight, bias) if stream is None else None
    if s is None:
        return _there(stream, (x, weight, bias), layer_norm_int8, x, weight, bias, eps)
    weight, bias, pt = _params(x, weight, bias)
    x, rows, stride = _rows(x, "x")
    cols = x.shape[-1]
    q, scale = _int8_out(x, rows)
    _check(lib.warp_layer_norm_int8(x.data_ptr(), stride, rows, cols, _DTYPES[x.dtype], _ptr(weight), _ptr(bias),
                                    _DTYPES[pt], eps, q.data_ptr(), q.shape[1], scale.data_ptr(), s))
    return QuantizedRows(q, scale, cols)


def linear_int8(a: QuantizedRows, w: QuantizedRows, bias=None, dtype=torch.bfloat16, stream=None):
    """Product [rows, n] of quantised tokens a [rows, cols] with a quantised weight w [n, cols], plus bias [n]
    float32, in `dtype`. The integer sums are exact."""
    if dtype not in _DTYPES:
        raise ValueError(f"dtype must be float32, float16 or bfloat16, got {dtype}")
    (av, sa, cols), (wv, sw, w_cols) = a, w
    if cols != w_cols:
        raise ValueError(f"tokens of {cols} columns against a weight of {w_cols}")
    padded = -(-cols // PAD) * PAD
    for name, v, s in (("a", av, sa), ("w", wv, sw)):
        if v.dtype != torch.int8 or v.dim() != 2 or v.stride(1) != 1:
            raise ValueError(f"{name}: int8 rows of contiguous elements are needed")
        if s.dtype != torch.float32 or s.shape != v.shape[:1] or not s.is_contiguous():
            raise ValueError(f"{name}: a contiguous float32 scale for each row is needed")
        if v.shape[1] < padded:  # what the kernels read of a row must lie inside the tensor
            raise ValueError(f"{name}: rows of {v.shape[1]} columns are not padded to a multiple of {PAD}; "
                             "see QuantizedRows.from_int8")
    rows, n = av.shape[0], wv.shape[0]
    if bias is not None and (bias.shape != (n,) or bias.dtype != torch.float32):
        raise ValueError(f"bias must be float32 ({n},), got {bias.dtype} {tuple(bias.shape)}")
    s = _here(av, sa, wv, sw, bias) if stream is None else None
    if s is None:
        return _there(stream, (av, sa, wv, sw, bias), linear_int8, a, w, bias, dtype)
    bias = None if bias is None else bias.contiguous()
    out = torch.empty((rows, n), dtype=dtype, device=av.device)
    _check(lib.warp_linear_int8(av.data_ptr(), av.stride(0), sa.data_ptr(), rows, wv.data_ptr(), wv.stride(0),
                                sw.data_ptr(), n, cols, _ptr(bias), out.data_ptr(), n, _DTYPES[dtype], s))
    return out


class AdamW:
    """AdamW over many tensors, all of one type, one step a call; moments in 32 or in 8 bits.

    The moments of all tensors are two flat tensors (with 8 bits also a scale for each block of 256
    elements), each tensor's part starting at a multiple of 256. `params` are contiguous device tensors and
    are updated in place."""

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 0.01, bits: int = 32):
        self.params = list(params)
        if not self.params:
            raise ValueError("no parameters")
        if bits not in (8, 32):
            raise ValueError(f"bits must be 8 or 32, got {bits}")
        first = self.params[0]
        for p in self.params:
            if not p.is_cuda or not p.is_contiguous() or p.device != first.device or p.dtype != first.dtype:
                raise ValueError("parameters must be contiguous tensors of one type on one device")
        if first.dtype not in _DTYPES:
            raise ValueError(f"parameters must be float32, float16 or bfloat16, got {first.dtype}")
        self.lr, self.betas, self.eps, self.weight_decay, self.bits = lr, tuple(betas), eps, weight_decay, bits
        self.steps = 0
        self._dtype = first.dtype
        self._sizes = [p.numel() for p in self.params]
        room = -(-np.asarray(self._sizes, np.int64) // BLOCK) * BLOCK
        ends = np.cumsum(room)
        self.size = int(ends[-1])  # elements of a flat moment tensor
        # the library's records: parameter, gradient, elements, start of the moments
        self._table = np.zeros((len(self.params), 4), np.int64)
        self._table[:, 2] = self._sizes
        self._table[:, 3] = ends - room
        dev = first.device
        self.m = torch.zeros(self.size, dtype=torch.float32 if bits == 32 else torch.int8, device=dev)
        self.v = torch.zeros(self.size, dtype=torch.float32 if bits == 32 else torch.uint8, device=dev)
        self.m_scale = self.v_scale = None
        if bits == 8:
            self.m_scale = torch.zeros(self.size // BLOCK, dtype=torch.float32, device=dev)
            self.v_scale = torch.zeros(self.size // BLOCK, dtype=torch.float32, device=dev)

    def step(self, grads, grad_scale=None, stream=None) -> None:
        """One step. grads: a contiguous tensor like each parameter, all of one floating type, or None for a
        parameter that this step leaves as it is. grad_scale: a float32 device tensor of one element that
        every gradient is multiplied by. The number of the step is a constant of the launched kernels: a graph
        that captured a step repeats that number. Parameters change without autograd's notice (it counts no
        version)."""
        params, index = self.params, self.m.get_device()
        if len(grads) != len(params):
            raise ValueError(f"{len(grads)} gradients for {len(params)} parameters")
        given, sizes = grads, self._sizes
        if _NONE in map(type, grads):
            given = [g for g in grads if g is not None]
            sizes = [n for g, n in zip(grads, sizes) if g is not None]
        dtype = given[0].dtype if given else torch.float32
        if dtype not in _DTYPES:
            raise ValueError(f"gradients must be float32, float16 or bfloat16, got {dtype}")
        if not self._fit(given, sizes, dtype):
            raise ValueError("gradients must be contiguous tensors of one type and of their parameters' sizes, on "
                             f"{self.m.device}")
        if not self._fit(params, self._sizes, self._dtype):
            raise ValueError("parameters must stay contiguous tensors of their type, size and device")
        if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1
                                       or grad_scale.get_device() != index):
            raise ValueError("grad_scale must be a float32 device tensor of one element")
        s = _here(self.m) if stream is None else None
        if s is None:
            return _there(stream, (self.m, self.v, self.m_scale, self.v_scale, grad_scale, *params, *grads),
                          self.step, grads, grad_scale)
        table = self._table
        table[:, 0] = [*map(torch.Tensor.data_ptr, params)]
        table[:, 1] = ([*map(torch.Tensor.data_ptr, grads)] if given is grads
                       else [0 if g is None else g.data_ptr() for g in grads])
        _check(lib.warp_adamw_step(table.ctypes.data, len(params), _DTYPES[self._dtype], _DTYPES[dtype], self.bits,
                                   self.m.data_ptr(), _ptr(self.m_scale), self.v.data_ptr(), _ptr(self.v_scale),
                                   self.lr, *self.betas, self.eps, self.weight_decay, self.steps + 1,
                                   _ptr(grad_scale), s))
        self.steps += 1

    def _fit(self, tensors, sizes, dtype) -> bool:
        """Whether these are contiguous tensors of these sizes, of one type, on the moments' device."""
        return not tensors or (
            [*map(torch.Tensor.numel, tensors)] == sizes and all(map(torch.Tensor.is_contiguous, tensors))
            and {*map(_dtype_of, tensors)} == {dtype}
            and {*map(torch.Tensor.get_device, tensors)} == {self.m.get_device()})

    def moments(self, stream=None):
        """The flat float32 moments (m, v): with 32 bits the optimizer's own, with 8 the values of its codes."""
        if self.bits == 32:
            return self.m, self.v
        s = _here(self.m) if stream is None else None
        if s is None:
            return _there(stream, (self.m, self.v, self.m_scale, self.v_scale), self.moments)
        m, v = torch.empty((2, self.size), dtype=torch.float32, device=self.m.device).unbind(0)
        _check(lib.warp_adamw_moments(self.m.data_ptr(), self.m_scale.data_ptr(), self.v.data_ptr(),
                                      self.v_scale.data_ptr(), self.size, m.data_ptr(), v.data_ptr(), s))
        return m, v

    def state_dict(self) -> dict:
        """What a checkpoint holds: the number of steps, the bits and the moments (the tensors themselves)."""
        d = {"step": self.steps, "bits": self.bits, "m": self.m, "v": self.v}
        return d if self.bits == 32 else {**d, "m_scale": self.m_scale, "v_scale": self.v_scale}

    def load_state_dict(self, state: dict) -> None:
        """Takes over (copies) a `state_dict` of the same parameters' sizes and bits."""
        mine = self.state_dict()
        if set(state) != set(mine) or state["bits"] != self.bits:
            raise ValueError(f"the state holds {sorted(state)}, {state.get('bits')} bits; needed: {sorted(mine)}, "
                             f"{self.bits}")
        for k, t in mine.items():
            if isinstance(t, torch.Tensor) and (state[k].shape != t.shape or state[k].dtype != t.dtype):
                raise ValueError(f"{k} must be {t.dtype} {tuple(t.shape)}")
        for k, t in mine.items():
            if isinstance(t, torch.Tensor):
                t.copy_(state[k])
        self.steps = int(state["step"])
