"""The operators of a token encoder's head, on torch device tensors: layer norm with its gradients,
products of 8-bit rows, and the AdamW step.

As in `warp`, everything runs in the HIP kernels behind the C ABI of include/warp.h; this module checks
tensors, allocates outputs with torch and passes pointers. A call works on the current stream of its
tensors' device, or on `stream`; inputs of another stream are the caller's to wait for. Tensors have
any row stride (a dimension's elements one after the other); leading dimensions are flattened to rows.
"""
from __future__ import annotations

import contextlib
import ctypes
from typing import NamedTuple

import numpy as np
import torch

from .warp import _check, lib

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


@contextlib.contextmanager
def _on(stream, tensors):
    """Makes `stream` current while a call allocates and enqueues, and keeps its inputs alive for it."""
    dev = tensors[0].device
    with torch.cuda.device(dev), torch.cuda.stream(stream):
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
        yield


def _run(stream, tensors, call):
    """call() with the current stream of the tensors' device, or with `stream`."""
    dev = tensors[0].device
    for t in tensors:
        if t is not None and (t.device != dev or not t.is_cuda):
            raise ValueError(f"expected device tensors on {dev}, got {t.device}")
    if stream is None and dev.index == torch.cuda.current_device():
        return call(torch.cuda.current_stream(dev).cuda_stream)
    stream = torch.cuda.current_stream(dev) if stream is None else stream
    with _on(stream, tensors):
        return call(stream.cuda_stream)


def _rows(x, name):
    """(tensor whose rows have contiguous elements, number of rows, row stride) of x [..., cols]."""
    if x.dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32, float16 or bfloat16, got {x.dtype}")
    if x.dim() == 2 and (x.stride(1) == 1 or x.shape[1] == 1):
        if x.shape[0] <= 1 or x.stride(0) >= x.shape[1]:
            return x, x.shape[0], x.stride(0)
    elif x.dim() == 0:
        raise ValueError(f"{name} must have at least one dimension")
    x = x.contiguous()
    cols = x.shape[-1]
    if cols < 1:
        raise ValueError(f"{name} has rows of no columns")
    return x, x.numel() // cols, cols


def _param(p, cols, name):
    if p is None:
        return None
    if p.shape != (cols,):
        raise ValueError(f"{name} must have shape ({cols},), got {tuple(p.shape)}")
    return p.contiguous()


def _params(x, weight, bias):
    """weight and bias as the kernels take them, and their dtype."""
    cols = x.shape[-1]
    weight, bias = _param(weight, cols, "weight"), _param(bias, cols, "bias")
    known = [p.dtype for p in (weight, bias) if p is not None]
    dtype = known[0] if known else torch.float32
    if any(d != dtype for d in known) or dtype not in (torch.float32, x.dtype):
        raise ValueError(f"weight and bias must both be float32 or both {x.dtype}, got {known}")
    return weight, bias, dtype


def _ptr(t):
    return None if t is None else t.data_ptr()


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, stream=None):
    """Layer norm over the last dimension of x [..., cols]: (y like x, mean, rstd), the row statistics in
    float32 [...] for `layer_norm_backward`. weight and bias [cols] are float32 or of x's type."""
    def call(s):
        w, b, pt = _params(x, weight, bias)
        r, rows, stride = _rows(x, "x")
        cols = r.shape[-1]
        y = torch.empty(r.shape, dtype=r.dtype, device=r.device)
        mean, rstd = torch.empty((2, *r.shape[:-1]), dtype=torch.float32, device=r.device).unbind(0)
        _check(lib.warp_layer_norm(r.data_ptr(), stride, rows, cols, _DTYPES[r.dtype], _ptr(w), _ptr(b), _DTYPES[pt],
                                   eps, y.data_ptr(), cols, mean.data_ptr(), rstd.data_ptr(), s))
        return y, mean, rstd

    return _run(stream, (x, weight, bias), call)


def layer_norm_backward(dy, x, weight, mean, rstd, stream=None):
    """Gradients (dx, dweight, dbias) of `layer_norm` for the gradient dy of its y. dweight and dbias have
    weight's type (float32 without a weight)."""
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError(f"dy must be like x ({tuple(x.shape)}, {x.dtype}), got {tuple(dy.shape)}, {dy.dtype}")
    for name, t in (("mean", mean), ("rstd", rstd)):
        if t.shape != x.shape[:-1] or t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError(f"{name} must be what layer_norm gave: contiguous float32 {tuple(x.shape[:-1])}")

    def call(s):
        w, _, pt = _params(x, weight, None)
        r, rows, stride = _rows(x, "x")
        d, _, d_stride = _rows(dy, "dy")
        cols = r.shape[-1]
        need = ctypes.c_int64()
        _check(lib.warp_layer_norm_backward_scratch(rows, cols, ctypes.byref(need)))
        dx = torch.empty(r.shape, dtype=r.dtype, device=r.device)
        dw, db = torch.empty((2, cols), dtype=pt, device=r.device).unbind(0)
        scratch = torch.empty(need.value, dtype=torch.uint8, device=r.device)
        _check(lib.warp_layer_norm_backward(d.data_ptr(), d_stride, r.data_ptr(), stride, rows, cols,
                                            _DTYPES[r.dtype], _ptr(w), _DTYPES[pt], mean.data_ptr(), rstd.data_ptr(),
                                            dx.data_ptr(), cols, dw.data_ptr(), db.data_ptr(), scratch.data_ptr(),
                                            need.value, s))
        return dx, dw, db

    return _run(stream, (x, dy, weight, mean, rstd), call)


def _int8_out(x, rows):
    q = torch.empty((rows, -(-x.shape[-1] // PAD) * PAD), dtype=torch.int8, device=x.device)
    return q, torch.empty(rows, dtype=torch.float32, device=x.device)


def quantize_rows(x, stream=None) -> QuantizedRows:
    """Rows of x [..., cols] in 8 bits with a scale each: token activations, or a weight [n, cols] with a
    scale for each output channel."""
    def call(s):
        r, rows, stride = _rows(x, "x")
        cols = r.shape[-1]
        q, scale = _int8_out(r, rows)
        _check(lib.warp_quantize_rows(r.data_ptr(), stride, rows, cols, _DTYPES[r.dtype], q.data_ptr(), q.shape[1],
                                      scale.data_ptr(), s))
        return QuantizedRows(q, scale, cols)

    return _run(stream, (x,), call)


def layer_norm_int8(x, weight=None, bias=None, eps: float = 1e-5, stream=None) -> QuantizedRows:
    """`quantize_rows` of `layer_norm`'s rows in one pass, without rounding them to x's type in between."""
    def call(s):
        w, b, pt = _params(x, weight, bias)
        r, rows, stride = _rows(x, "x")
        cols = r.shape[-1]
        q, scale = _int8_out(r, rows)
        _check(lib.warp_layer_norm_int8(r.data_ptr(), stride, rows, cols, _DTYPES[r.dtype], _ptr(w), _ptr(b),
                                        _DTYPES[pt], eps, q.data_ptr(), q.shape[1], scale.data_ptr(), s))
        return QuantizedRows(q, scale, cols)

    return _run(stream, (x, weight, bias), call)


def linear_int8(a: QuantizedRows, w: QuantizedRows, bias=None, dtype=torch.bfloat16, stream=None):
    """Product [rows, n] of quantised tokens a [rows, cols] with a quantised weight w [n, cols], plus bias [n]
    float32, in `dtype`. The integer sums are exact."""
    if dtype not in _DTYPES:
        raise ValueError(f"dtype must be float32, float16 or bfloat16, got {dtype}")
    if a.cols != w.cols:
        raise ValueError(f"tokens of {a.cols} columns against a weight of {w.cols}")
    for name, r in (("a", a), ("w", w)):
        v, s = r.values, r.scale
        if v.dtype != torch.int8 or v.dim() != 2 or (v.stride(1) != 1 and v.shape[1] > 1) or v.shape[1] < r.cols:
            raise ValueError(f"{name}: int8 rows of at least {r.cols} columns are needed")
        if s.dtype != torch.float32 or s.shape != v.shape[:1] or not s.is_contiguous():
            raise ValueError(f"{name}: a contiguous float32 scale for each row is needed")
        # what the kernels read of a row must lie inside the tensor
        if v.shape[1] < -(-r.cols // PAD) * PAD:
            raise ValueError(f"{name}: rows of {v.shape[1]} columns are not padded to a multiple of {PAD}; "
                             "see QuantizedRows.from_int8")
    rows, n = a.values.shape[0], w.values.shape[0]
    if bias is not None and (bias.shape != (n,) or bias.dtype != torch.float32):
        raise ValueError(f"bias must be float32 ({n},), got {bias.dtype} {tuple(bias.shape)}")
    def call(s):
        b = None if bias is None else bias.contiguous()
        out = torch.empty((rows, n), dtype=dtype, device=a.values.device)
        _check(lib.warp_linear_int8(a.values.data_ptr(), a.values.stride(0), a.scale.data_ptr(), rows,
                                    w.values.data_ptr(), w.values.stride(0), w.scale.data_ptr(), n, a.cols,
                                    _ptr(b), out.data_ptr(), n, _DTYPES[dtype], s))
        return out

    return _run(stream, (a.values, a.scale, w.values, w.scale, bias), call)


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
        every gradient is multiplied by."""
        params, sizes, table = self.params, self._sizes, self._table
        if len(grads) != len(params):
            raise ValueError(f"{len(grads)} gradients for {len(params)} parameters")
        dev, dtype, grad_dtype = self.m.device, params[0].dtype, None
        pointers = []
        for p, g, n in zip(params, grads, sizes):
            if g is None:
                pointers.append(0)
                continue
            if grad_dtype is None:
                grad_dtype = g.dtype
                if grad_dtype not in _DTYPES:
                    raise ValueError(f"gradients must be float32, float16 or bfloat16, got {grad_dtype}")
            if (g.dtype is not grad_dtype or g.numel() != n or g.device != dev or not g.is_contiguous()
                    or p.numel() != n or p.device != dev or p.dtype is not dtype or not p.is_contiguous()):
                raise ValueError("gradients must be contiguous tensors of one type and of their parameters' sizes, "
                                 "and parameters as they were given")
            pointers.append(g.data_ptr())
        if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1
                                       or grad_scale.device != dev):
            raise ValueError("grad_scale must be a float32 device tensor of one element")
        table[:, 0] = [p.data_ptr() for p in params]
        table[:, 1] = pointers
        if grad_dtype is None:
            grad_dtype = torch.float32

        def call(s):
            _check(lib.warp_adamw_step(table.ctypes.data, len(params), _DTYPES[dtype], _DTYPES[grad_dtype], self.bits,
                                       self.m.data_ptr(), _ptr(self.m_scale), self.v.data_ptr(), _ptr(self.v_scale),
                                       self.lr, self.betas[0], self.betas[1], self.eps, self.weight_decay,
                                       self.steps + 1, _ptr(grad_scale), s))

        if stream is None:
            _run(None, (self.m,), call)
        else:
            _run(stream, (self.m, self.v, self.m_scale, self.v_scale, grad_scale, *params, *grads), call)
        self.steps += 1

    def moments(self, stream=None):
        """The flat float32 moments (m, v): with 32 bits the optimizer's own, with 8 the values of its codes."""
        if self.bits == 32:
            return self.m, self.v

        def call(s):
            out = torch.empty((2, self.size), dtype=torch.float32, device=self.m.device).unbind(0)
            _check(lib.warp_adamw_moments(self.m.data_ptr(), self.m_scale.data_ptr(), self.v.data_ptr(),
                                          self.v_scale.data_ptr(), self.size, out[0].data_ptr(), out[1].data_ptr(),
                                          s))
            return out

        return _run(stream, (self.m, self.v, self.m_scale, self.v_scale), call)

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
