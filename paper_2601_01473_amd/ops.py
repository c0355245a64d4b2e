"""Operators of a training or serving step on torch CUDA tensors.

Thin wrappers of the C entry points agnes_embedding_*, agnes_distill_* and
agnes_mx4_*: they check what only the tensors know (device, layout), allocate
outputs and workspace from torch's caching allocator, and enqueue on `stream`
(default: the current stream).  Nothing waits for the GPU.

With another stream than the current one, outputs and workspace are allocated
for that stream and the inputs are recorded on it, so their memory is not
handed out again while the call reads it; ordering the stream after the work
that makes the inputs is the caller's, as for any stream.

Autograd does not see these calls: a result has no history, also where an input
requires a gradient.  A backward pass calls embedding_grad or
embedding_grad_rows and distill_grad or distill_loss_grad itself (or wraps them
in a torch.autograd.Function); 4-bit products have no backward pass.
"""
from __future__ import annotations

import collections
import contextlib
import functools

import torch

from . import _binding as B

_FLOATS = {torch.float32: B.AGNES_FLOAT32, torch.float16: B.AGNES_FLOAT16, torch.bfloat16: B.AGNES_BFLOAT16}
_INDEXES = {torch.int32: B.AGNES_INT32, torch.int64: B.AGNES_INT64}

Mx4 = collections.namedtuple("Mx4", "codes scales cols")
Mx4.__doc__ = """Rows in microscaled 4-bit floating point: codes uint8 [rows, 16 ceil(cols / 32)] (two elements per byte, the
even one in the low four bits), scales uint8 [rows, ceil(cols / 32)] (2^(code - 127), 255 = NaN), and the row length."""


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)   # once a CUDA tensor exists


def _handle(stream) -> int:
    """The HIP stream that a call enqueues on (None: the current one)."""
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(_current_device())
        return torch.cuda.current_stream().cuda_stream
    return int(getattr(stream, "cuda_stream", stream))


_HERE = contextlib.nullcontext()


def _on(stream, *inputs):
    """A context in which torch allocates for `stream`; records the inputs on it if it is not the current one."""
    if stream is None or _handle(stream) == _handle(None):
        return _HERE
    s = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream))
    for t in inputs:
        if t is not None:
            t.record_stream(s)
    return torch.cuda.stream(s)


def _device(t: torch.Tensor, name: str) -> None:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % name)
    if t.get_device() != _current_device():
        raise ValueError("%s is on device %d, the current device is %d"
                         % (name, t.get_device(), _current_device()))


def _matrix(t: torch.Tensor, name: str) -> B.agnes_matrix:
    _device(t, name)
    code = _FLOATS.get(t.dtype)
    if code is None:
        raise TypeError("%s must be float32, float16 or bfloat16" % name)
    if t.dim() != 2:
        raise ValueError("%s must be 2-D" % name)
    rows, cols = t.shape
    row_stride, col_stride = t.stride()
    if col_stride != 1 and cols > 1:
        raise ValueError("%s must have adjacent columns" % name)
    return B.agnes_matrix(t.data_ptr(), rows, cols, row_stride, code)


def _new(like: torch.Tensor, rows: int, cols: int, dtype: torch.dtype):
    """A new matrix beside `like` and its structure."""
    t = like.new_empty((rows, cols), dtype=dtype)
    code = _FLOATS.get(dtype)
    if code is None:
        raise TypeError("the result must be float32, float16 or bfloat16")
    return t, B.agnes_matrix(t.data_ptr(), rows, cols, cols, code)


def _rows_of(t: torch.Tensor) -> torch.Tensor:
    """t with adjacent columns (a copy if it has none, as an expanded scalar's gradient)."""
    return t if t.dim() != 2 or t.shape[1] <= 1 or t.stride(1) == 1 else t.contiguous()


def _index(t: torch.Tensor, name: str) -> int:
    _device(t, name)
    code = _INDEXES.get(t.dtype)
    if code is None:
        raise TypeError("%s must be int32 or int64" % name)
    return code


# Workspace sizes follow from the sizes alone.
_grad_bytes = functools.lru_cache(1024)(B.agnes_embedding_grad_bytes)
_distill_bytes = functools.lru_cache(1024)(B.agnes_distill_bytes)
_product_bytes = functools.lru_cache(1024)(B.agnes_mx4_product_bytes)
_linear_bytes = functools.lru_cache(1024)(B.agnes_mx4_linear_bytes)


def _workspace(like: torch.Tensor, nbytes: int):
    return like.new_empty(nbytes, dtype=torch.uint8) if nbytes else None


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


# ----------------------------------------------------------------- embedding

def embedding_lookup(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, dtype: torch.dtype | None = None,
                     out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """scale * table[ids] (agnes_embedding_lookup): ids int32 or int64 of any
    shape, one outside [0, len(table)) gives a zero row; returns [*ids.shape,
    dim] of `dtype` (default: the table's)."""
    m = _matrix(table, "table")
    code = _index(ids, "ids")
    with _on(stream, table, ids, out):
        flat = ids if ids.is_contiguous() else ids.contiguous()
        n = ids.numel()
        if out is None:
            rows, o = _new(table, n, m.cols, dtype or table.dtype)
            out = rows if ids.dim() == 1 else rows.view(*ids.shape, m.cols)
        elif tuple(out.shape) != (*ids.shape, m.cols) or (dtype is not None and out.dtype != dtype):
            raise ValueError("out must be [*ids.shape, dim] of the type asked for")
        else:
            o = _matrix(out if out.dim() == 2 else out.view(n, m.cols), "out")
        B.agnes_embedding_lookup(m, flat.data_ptr(), code, scale, o, _handle(stream))
    return out


def _grad_args(grad_out, ids, dim_name="grad_out"):
    code = _index(ids, "ids")
    if not isinstance(grad_out, torch.Tensor) or grad_out.dim() < 1 or grad_out.shape[:-1] != ids.shape:
        raise ValueError("%s must be [*ids.shape, dim]" % dim_name)
    if grad_out.dim() != 2:
        grad_out = grad_out.reshape(ids.numel(), grad_out.shape[-1])
    g = _rows_of(grad_out)
    return g, _matrix(g, dim_name), code, ids if ids.is_contiguous() else ids.contiguous()


def embedding_grad(grad_out: torch.Tensor, ids: torch.Tensor, num_rows: int, scale: float = 1.0,
                   dtype: torch.dtype | None = None, out: torch.Tensor | None = None, accumulate: bool = False,
                   stream=None) -> torch.Tensor:
    """The lookup's gradient as a whole table [num_rows, dim] (agnes_embedding_grad),
    of `dtype` (default: grad_out's).  accumulate: add to `out` instead of writing it."""
    with _on(stream, grad_out, ids, out):
        keep, g, code, flat = _grad_args(grad_out, ids)
        if out is None:
            if accumulate:
                raise ValueError("accumulate needs out")
            out, o = _new(keep, num_rows, g.cols, dtype or grad_out.dtype)
        elif tuple(out.shape) != (num_rows, g.cols) or (dtype is not None and out.dtype != dtype):
            raise ValueError("out must be [num_rows, dim] of the type asked for")
        else:
            o = _matrix(out, "out")
        need = _grad_bytes(g.rows, num_rows, g.cols)
        ws = _workspace(keep, need)
        B.agnes_embedding_grad(g, flat.data_ptr(), code, scale, 1 if accumulate else 0, o, _ptr(ws), need,
                               _handle(stream))
    return out


def embedding_grad_rows(grad_out: torch.Tensor, ids: torch.Tensor, num_rows: int, max_rows: int | None = None,
                        scale: float = 1.0, dtype: torch.dtype | None = None, stream=None):
    """The lookup's gradient as distinct rows (agnes_embedding_grad_rows):
    (row_ids int32 [max_rows], rows [max_rows, dim], count int64 [1]).  The
    first min(count, max_rows) entries hold the distinct ids in ascending order
    and their gradients; the other ids are -1, the other rows undefined.
    max_rows defaults to min(ids.numel(), num_rows); for a batch's node list
    stats()["distinct_rows"] is the count."""
    if max_rows is None:
        max_rows = min(ids.numel(), num_rows)
    with _on(stream, grad_out, ids):
        keep, g, code, flat = _grad_args(grad_out, ids)
        row_ids = keep.new_empty(max_rows, dtype=torch.int32)
        rows, o = _new(keep, max_rows, g.cols, dtype or grad_out.dtype)
        count = keep.new_empty(1, dtype=torch.int64)
        need = _grad_bytes(g.rows, num_rows, g.cols)
        ws = _workspace(keep, need)
        B.agnes_embedding_grad_rows(g, flat.data_ptr(), code, scale, num_rows, row_ids.data_ptr(), o,
                                    count.data_ptr(), _ptr(ws), need, _handle(stream))
    return row_ids, rows, count


# ----------------------------------------------------------------- distillation

def _distill(logits, teacher, classes, labels, weight, temperature, soft, hard):
    z, t = _matrix(logits, "logits"), _matrix(teacher, "teacher")
    code = _index(classes, "classes")
    if classes.shape != teacher.shape or (classes.shape[1] > 1 and classes.stride(1) != 1):
        raise ValueError("classes must have the teacher's shape and adjacent columns")
    if labels is not None and (_index(labels, "labels") != code or labels.shape != logits.shape[:1] or
                               (labels.numel() > 1 and labels.stride(0) != 1)):
        raise ValueError("labels must be contiguous [rows] of the classes' type")
    if weight is not None:
        _device(weight, "weight")
        if weight.dtype != torch.float32 or weight.shape != logits.shape[:1] or \
                (weight.numel() > 1 and weight.stride(0) != 1):
            raise ValueError("weight must be contiguous float32 [rows]")
    return B.agnes_distill(z, t, classes.data_ptr(), classes.stride(0), code, _ptr(labels), _ptr(weight),
                           temperature, soft, hard)


def distill_loss(logits, teacher, classes, labels=None, weight=None, temperature: float = 1.0, soft: float = 1.0,
                 hard: float = 0.0, stream=None):
    """Per-row distillation loss (agnes_distill_loss): student logits [rows, C],
    the teacher's top logits [rows, k] and their classes [rows, k], labels
    [rows] (with hard > 0), weight float32 [rows].  Returns (loss float32
    [rows], stats float32 [rows, 3]); distill_grad takes the statistics."""
    d = _distill(logits, teacher, classes, labels, weight, temperature, soft, hard)
    with _on(stream, logits, teacher, classes, labels, weight):
        rows = d.logits.rows
        loss = logits.new_empty(rows, dtype=torch.float32)
        stats = logits.new_empty((rows, 3), dtype=torch.float32)
        need = _distill_bytes(rows, d.logits.cols)
        ws = _workspace(logits, need)
        B.agnes_distill_loss(d, loss.data_ptr(), stats.data_ptr(), _ptr(ws), need, _handle(stream))
    return loss, stats


def _grad_like(logits, out):
    if out is None:
        return _new(logits, logits.shape[0], logits.shape[1], logits.dtype)
    if out.shape != logits.shape:
        raise ValueError("out must have the logits' shape")
    return out, _matrix(out, "out")


def distill_grad(logits, teacher, classes, stats, labels=None, weight=None, temperature: float = 1.0,
                 soft: float = 1.0, hard: float = 0.0, out=None, stream=None) -> torch.Tensor:
    """The gradient of sum(weight * L) from distill_loss's statistics
    (agnes_distill_grad): as the backward pass of per-row losses, `weight` is
    the gradient that arrives.  out may be the logits themselves."""
    d = _distill(logits, teacher, classes, labels, weight, temperature, soft, hard)
    _device(stats, "stats")
    if stats.dtype != torch.float32 or tuple(stats.shape) != (d.logits.rows, 3) or not stats.is_contiguous():
        raise ValueError("stats must be distill_loss's statistics, contiguous float32 [rows, 3]")
    with _on(stream, logits, teacher, classes, stats, labels, weight, out):
        out, o = _grad_like(logits, out)
        B.agnes_distill_grad(d, stats.data_ptr(), o, _handle(stream))
    return out


def distill_loss_grad(logits, teacher, classes, labels=None, weight=None, temperature: float = 1.0,
                      soft: float = 1.0, hard: float = 0.0, out=None, stream=None):
    """(loss float32 [rows], gradient of sum(loss) [rows, C]) in one pass over
    the logits (agnes_distill_loss_grad).  out may be the logits themselves."""
    d = _distill(logits, teacher, classes, labels, weight, temperature, soft, hard)
    with _on(stream, logits, teacher, classes, labels, weight, out):
        out, o = _grad_like(logits, out)
        loss = logits.new_empty(d.logits.rows, dtype=torch.float32)
        need = _distill_bytes(d.logits.rows, d.logits.cols)
        ws = _workspace(logits, need)
        B.agnes_distill_loss_grad(d, loss.data_ptr(), o, _ptr(ws), need, _handle(stream))
    return loss, out


# ----------------------------------------------------------------- 4-bit rows

def _mx4(q: Mx4, name: str) -> B.agnes_mx4:
    codes, scales, cols = q
    blocks = -(-cols // 32)
    _device(codes, name + ".codes")
    _device(scales, name + ".scales")
    rows = codes.shape[0]
    if codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or \
            tuple(codes.shape) != (rows, 16 * blocks) or tuple(scales.shape) != (rows, blocks) or \
            not (codes.is_contiguous() and scales.is_contiguous()):
        raise ValueError("%s must be contiguous uint8 codes [rows, 16 ceil(cols / 32)] and scales "
                         "[rows, ceil(cols / 32)]" % name)
    return B.agnes_mx4(codes.data_ptr(), scales.data_ptr(), rows, cols)


def mx4_quantize(x: torch.Tensor, stream=None) -> Mx4:
    """Rows [R, K] to microscaled 4-bit floating point (agnes_mx4_quantize)."""
    m = _matrix(x, "x")
    blocks = -(-m.cols // 32)
    with _on(stream, x):
        q = Mx4(x.new_empty((m.rows, 16 * blocks), dtype=torch.uint8),
                x.new_empty((m.rows, blocks), dtype=torch.uint8), m.cols)
        d = B.agnes_mx4(q.codes.data_ptr(), q.scales.data_ptr(), m.rows, m.cols)
        B.agnes_mx4_quantize(m, d, _handle(stream))
    return q


def mx4_dequantize(q: Mx4, dtype: torch.dtype = torch.float32, stream=None) -> torch.Tensor:
    """The values [R, K] that 4-bit rows stand for (agnes_mx4_dequantize)."""
    d = _mx4(q, "q")
    with _on(stream, q.codes, q.scales):
        x, m = _new(q.codes, d.rows, d.cols, dtype)
        B.agnes_mx4_dequantize(d, m, _handle(stream))
    return x


def mx4_linear(x, weight: Mx4, bias: torch.Tensor | None = None, relu: bool = False,
               dtype: torch.dtype | None = None, out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """x weight^T + bias with 4-bit operands: x float rows [M, K], quantised on
    the way in (agnes_mx4_linear), or an Mx4 (agnes_mx4_product); bias float32
    [N].  Returns [M, N] of `dtype` (default: x's, float32 for an Mx4)."""
    w = _mx4(weight, "weight")
    given = isinstance(x, Mx4)
    a = _mx4(x, "x") if given else _matrix(x, "x")
    if bias is not None:
        _device(bias, "bias")
        if bias.dtype != torch.float32 or tuple(bias.shape) != (w.rows,) or not bias.is_contiguous():
            raise ValueError("bias must be contiguous float32 [N]")
    with _on(stream, *((x.codes, x.scales) if given else (x,)), weight.codes, weight.scales, bias, out):
        if out is None:
            out, o = _new(weight.codes, a.rows, w.rows, dtype or (torch.float32 if given else x.dtype))
        elif tuple(out.shape) != (a.rows, w.rows) or (dtype is not None and out.dtype != dtype):
            raise ValueError("out must be [M, N] of the type asked for")
        else:
            o = _matrix(out, "out")
        size, call = (_product_bytes, B.agnes_mx4_product) if given else (_linear_bytes, B.agnes_mx4_linear)
        need = size(a.rows, w.rows, a.cols)
        ws = _workspace(weight.codes, need)
        call(a, w, _ptr(bias), 1 if relu else 0, o, _ptr(ws), need, _handle(stream))
    return out
