"""The operators that train a token encoder and serve its head, on torch device tensors: table lookup, layer norm,
linear layers and softmax cross entropy with their gradients, products of 8-bit rows, and the AdamW step.

As in `warp`, everything runs in the HIP kernels behind the C ABI of include/warp.h. `_encoder.so` (from
csrc_encoder/encoder_binding.cpp) checks tensors, allocates outputs with torch and passes pointers: a ValueError
for tensors that do not fit, a WarpError for what the library refuses. A call works on the current stream of its
tensors' device, or on `stream`; inputs of another stream are the caller's to wait for. Tensors have any row
stride (a dimension's elements one after the other); leading dimensions are flattened to rows. autograd follows
`embedding`, `layer_norm`, `linear` and `cross_entropy` backwards, and refuses forward-mode tangents there (a
NotImplementedError); 8-bit rows and what is made of them carry no gradient. torch.jit.trace records these four (a
`linear` without `rows`); every other call is refused under it (a RuntimeError).
Calls can be captured into graphs; a backward pass only while no graph of the leaves that it leads to from outside the
capture lives (a RuntimeError).
"""
from __future__ import annotations

import os
from typing import NamedTuple

import numpy as np
import torch

from . import warp  # loads libwarp.so, which the binding calls

if not os.path.exists(os.path.join(os.path.dirname(os.path.abspath(__file__)), "_encoder.so")):
    raise ImportError("_encoder.so is not built; run __graft_entry__.build()")
from . import _encoder as _native  # noqa: E402

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


def _on(stream, tensors, call, *args):
    """call(*args) with `stream` current, so that outputs and copies are allocated and enqueued there; the
    tensors are kept for its work."""
    for t in tensors:
        if t is not None and not t.is_cuda:
            raise ValueError(f"expected device tensors, got {t.device}")
        if t is not None and t.device != stream.device:
            raise ValueError(f"a stream of {stream.device} for tensors on {t.device}")
    with torch.cuda.stream(stream):
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
        return call(*args)


def _leaves(node):
    """The leaves to which gradients go from a node of autograd's graph, through whatever nodes lie between."""
    seen, todo = set(), [f for f, _ in node.next_functions]
    while todo:
        f = todo.pop()
        if f is None or f in seen:
            continue
        seen.add(f)
        if isinstance(f, torch._C._functions.AccumulateGrad):
            yield f.variable
        else:
            todo += [g for g, _ in f.next_functions]


def _refuse_capture(ctx):
    """Refuses a backward pass under capture whose leaves' gradients would be added on the default stream, since a graph
    made there lives: a stream under capture cannot be joined with it, and trying ends the process."""
    if torch.cuda.is_current_stream_capturing() and any(map(_native.adds_on_default_stream, _leaves(ctx))):
        raise RuntimeError("a backward pass cannot be captured while a graph of the same leaves from outside the capture lives")


def _refuse_tangent(dy):
    """Refuses a gradient with a forward-mode tangent, which the gradients made of it would silently lose."""
    if _native.has_tangent(dy):
        raise NotImplementedError("forward-mode differentiation of a backward pass is not implemented")


class _LayerNorm(torch.autograd.Function):
    """What `layer_norm` is to autograd. The statistics have no gradient, and y no second derivative."""

    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = _native.layer_norm_forward(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.mark_non_differentiable(mean, rstd)
        ctx.bias_type = None if bias is None else bias.dtype
        return y, mean, rstd

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, *_):
        _refuse_capture(ctx)
        _refuse_tangent(dy)
        x, weight, mean, rstd = ctx.saved_tensors
        dx, dw, db = _native.layer_norm_backward(dy, x, weight, mean, rstd)
        return dx, None if weight is None else dw, None if ctx.bias_type is None else db.to(ctx.bias_type), None


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, stream=None):
    """Layer norm over the last dimension of x [..., cols]: (y like x, mean, rstd), the row statistics in
    float32 [...] for `layer_norm_backward`. weight and bias [cols] are float32 or of x's type. autograd follows y,
    not the statistics."""
    if stream is None:
        return _native.layer_norm(x, weight, bias, eps)
    return _on(stream, (x, weight, bias), _native.layer_norm, x, weight, bias, eps)


def layer_norm_backward(dy, x, weight, mean, rstd, stream=None):
    """Gradients (dx, dweight, dbias) of `layer_norm` for the gradient dy of its y, unknown to autograd. dweight and
    dbias have weight's type (float32 without a weight)."""
    if stream is None:
        return _native.layer_norm_backward(dy, x, weight, mean, rstd)
    return _on(stream, (x, dy, weight, mean, rstd), _native.layer_norm_backward, dy, x, weight, mean, rstd)


def quantize_rows(x, stream=None) -> QuantizedRows:
    """Rows of x [..., cols] in 8 bits with a scale each: token activations, or a weight [n, cols] with a
    scale for each output channel. At most 16,384 columns; wider rows that were quantised elsewhere come in through
    `QuantizedRows.from_int8`."""
    if stream is None:
        return QuantizedRows._make(_native.quantize_rows(x))
    return QuantizedRows._make(_on(stream, (x,), _native.quantize_rows, x))


def layer_norm_int8(x, weight=None, bias=None, eps: float = 1e-5, stream=None) -> QuantizedRows:
    """`quantize_rows` of `layer_norm`'s rows in one pass, without rounding them to x's type in between."""
    if stream is None:
        return QuantizedRows._make(_native.layer_norm_int8(x, weight, bias, eps))
    return QuantizedRows._make(_on(stream, (x, weight, bias), _native.layer_norm_int8, x, weight, bias, eps))


def linear_int8(a: QuantizedRows, w: QuantizedRows, bias=None, dtype=torch.bfloat16, stream=None):
    """Product [rows, n] of quantised tokens a [rows, cols] with a quantised weight w [n, cols], plus bias [n]
    float32, in `dtype`. The integer sums are exact."""
    if stream is None:
        return _native.linear_int8(*a, *w, bias, dtype)
    return _on(stream, (a.values, a.scale, w.values, w.scale, bias), _native.linear_int8, *a, *w, bias, dtype)


class _Embedding(torch.autograd.Function):
    """What `embedding` is to autograd."""

    @staticmethod
    def forward(ctx, ids, table, scale):
        ctx.save_for_backward(ids)
        ctx.vocabulary, ctx.scale = table.shape[0], scale
        return _native.embedding_forward(ids, table, scale)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        _refuse_capture(ctx)
        _refuse_tangent(dy)
        return None, _native.embedding_backward(dy, *ctx.saved_tensors, ctx.vocabulary, ctx.scale), None


def embedding(ids, table, scale: float = 1.0, stream=None):
    """Rows of table [vocabulary, cols] for ids [...] (int64 or int32), times scale: [..., cols] of table's type. A negative
    id is padding and gives zeros; one outside the table gives NaN. autograd follows the table."""
    if stream is None:
        return _native.embedding(ids, table, scale)
    return _on(stream, (ids, table), _native.embedding, ids, table, scale)


def embedding_backward(dy, ids, vocabulary: int, scale: float = 1.0, stream=None):
    """Gradient [vocabulary, cols] of `embedding`'s table for the gradient dy [..., cols] of its rows. The sums' order is
    the tokens': the same call gives the same bits."""
    if stream is None:
        return _native.embedding_backward(dy, ids, vocabulary, scale)
    return _on(stream, (dy, ids), _native.embedding_backward, dy, ids, vocabulary, scale)


class _CrossEntropy(torch.autograd.Function):
    """What `cross_entropy` is to autograd. lse has no gradient, and the losses no second derivative."""

    @staticmethod
    def forward(ctx, hidden, table, targets, scale):
        loss, lse = _native.cross_entropy_forward(hidden, table, targets, scale)
        # a copy: the caller may change its losses in place
        ctx.save_for_backward(hidden, table, targets, loss.clone(), lse.clone())
        ctx.mark_non_differentiable(lse)
        ctx.scale = scale
        return loss, lse

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss, _):
        _refuse_capture(ctx)
        _refuse_tangent(dloss)
        want = ctx.needs_input_grad
        return *_native.cross_entropy_backward(dloss, *ctx.saved_tensors, ctx.scale, want[0], want[1]), None, None


def cross_entropy(hidden, table, targets, scale: float = 1.0, stream=None):
    """Softmax cross entropy of rows hidden [..., cols] over a vocabulary, with the logits scale * hidden . table[v] of a
    table [vocabulary, cols]: (loss, lse), both float32 [...], lse the logarithm of the sum of the logits' exponentials.
    The logits are never written. A row with a negative target is left out (both are 0) and costs next to nothing, so that a
    batch with few predicted tokens needs no selection; a target outside the vocabulary gives NaN. autograd follows
    loss."""
    if stream is None:
        return _native.cross_entropy(hidden, table, targets, scale)
    return _on(stream, (hidden, table, targets), _native.cross_entropy, hidden, table, targets, scale)


def cross_entropy_backward(dloss, hidden, table, targets, loss, lse, scale: float = 1.0, stream=None):
    """Gradients (dhidden, dtable) of `cross_entropy` for the gradient dloss of its losses (float32), from the loss and lse
    that it gave."""
    args = dloss, hidden, table, targets, loss, lse
    if stream is None:
        return _native.cross_entropy_backward(*args, scale, True, True)
    return _on(stream, args, _native.cross_entropy_backward, *args, scale, True, True)


class _Linear(torch.autograd.Function):
    """What `linear` is to autograd: of its input it keeps 8-bit rows, and those only if the weight has a gradient."""

    @staticmethod
    def forward(ctx, x, weight, bias, rows):
        y = _native.linear_forward(x, weight, bias)
        values = scale = None
        if ctx.needs_input_grad[1]:
            values, scale, cols = _native.quantize_rows_forward(x) if rows is None else rows
            if rows is not None:
                count = x.numel() // x.shape[-1]
                if cols != x.shape[-1] or values.shape[0] != count or values.dtype != torch.int8 or scale.shape != (count,):
                    raise ValueError(f"rows in 8 bits of {tuple(values.shape)}, {cols} columns, for x {tuple(x.shape)}")
        ctx.save_for_backward(values, scale, weight)
        ctx.bias_type = torch.float32 if bias is None else bias.dtype
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        _refuse_capture(ctx)
        _refuse_tangent(dy)
        return *_native.linear_backward(dy, *ctx.saved_tensors, *ctx.needs_input_grad[:3], ctx.bias_type), None


def linear(x, weight, bias=None, rows: QuantizedRows | None = None, stream=None):
    """x [..., cols] by a weight [n, cols] of its type, plus bias [n] (float32 or of x's type): [..., n]. For autograd it
    keeps x in 8 bits (`quantize_rows`) in every type, from which the weight's gradient is made: of steps of 1/127 of a row's largest
    element, which are coarse for the others where one is far larger. x's own gradient does not need x. `rows`: x's 8-bit rows, where
    the caller has them already, as for several layers of one input; above 16,384 columns they are needed for the weight's gradient."""
    if stream is None:
        return _native.linear(x, weight, bias, rows)
    kept = () if rows is None else (rows.values, rows.scale)
    return _on(stream, (x, weight, bias, *kept), _native.linear, x, weight, bias, rows)


def linear_backward(dy, rows: QuantizedRows, weight, stream=None):
    """Gradients (dx, dweight, dbias) of `linear` for the gradient dy of its result, from the 8-bit rows of its input. They
    have dy's type."""
    if rows.cols != weight.shape[-1]:
        raise ValueError(f"rows of {rows.cols} columns for a weight {tuple(weight.shape)}")
    args = dy, rows.values, rows.scale, weight, True, True, True, dy.dtype
    if stream is None:
        return _native.linear_backward(*args)
    return _on(stream, args[:4], _native.linear_backward, *args)


def _overlap(tensors):
    """The places of two of these contiguous tensors that share memory, or None."""
    spans = sorted((t.data_ptr(), t.numel() * t.element_size(), i) for i, t in enumerate(tensors) if t.numel())
    for (start, size, i), (after, _, j) in zip(spans, spans[1:]):
        if after < start + size:
            return min(i, j), max(i, j)
    return None


class AdamW:
    """AdamW over many tensors, all of one type, one step a call; moments in 32 or in 8 bits.

    The moments of all tensors are two flat tensors (with 8 bits also a scale for each block of 256
    elements), each tensor's part starting at a multiple of 256. `params` are contiguous device tensors that share
    no memory (one that a model uses twice is given once) and are updated in place.

    8 bits are for tensors whose gradients stay alive, within an order of magnitude among 256 neighbours. An element
    whose gradient vanishes, or turns and is below 0.5% of its block's largest, keeps the first moment that it had (as
    long as the largest stays) and goes on moving, by tens of lr in thousands of steps: token tables and layers with
    dead columns belong in an optimizer of 32 bits."""

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
        if first.dtype not in (torch.float32, torch.float16, torch.bfloat16):
            raise ValueError(f"parameters must be float32, float16 or bfloat16, got {first.dtype}")
        if shared := _overlap(self.params):  # two workgroups would move the same elements at once
            raise ValueError("parameters %d and %d share memory" % shared)
        self.lr, self.betas, self.eps, self.weight_decay, self.bits = lr, tuple(betas), eps, weight_decay, bits
        self.steps = 0
        self._dtype = first.dtype
        sizes = np.asarray([p.numel() for p in self.params], np.int64)
        room = -(-sizes // BLOCK) * BLOCK
        ends = np.cumsum(room)
        self.size = int(ends[-1])  # elements of a flat moment tensor
        # the library's records: parameter, gradient, elements, start of the moments
        self._table = np.zeros((len(self.params), 4), np.int64)
        self._table[:, 2] = sizes
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
        that captured a step repeats that number. autograd counts the change of a parameter as any in place."""
        args = (self.params, grads, self._table, self._dtype, self.bits, self.m, self.m_scale, self.v, self.v_scale,
                self.lr, *self.betas, self.eps, self.weight_decay, self.steps + 1, grad_scale)
        if stream is None:
            _native.adamw_step(*args)
        else:
            _on(stream, (self.m, self.v, self.m_scale, self.v_scale, grad_scale, *self.params, *grads),
                _native.adamw_step, *args)
        self.steps += 1

    def moments(self, stream=None):
        """The flat float32 moments (m, v): with 32 bits the optimizer's own, with 8 the values of its codes."""
        if self.bits == 32:
            return self.m, self.v
        args = self.m, self.m_scale, self.v, self.v_scale
        return _native.adamw_moments(*args) if stream is None else _on(stream, args, _native.adamw_moments, *args)

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
