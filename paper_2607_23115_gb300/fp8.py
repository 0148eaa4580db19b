"""Weights in 8-bit floating point: layout, products and gradients.

    w = fp8.quantize_weight(weight, grad=True)   # [n, k], or [experts, n, k]
    y = fp8.linear(x, w)                         # x [..., k] -> [..., n]
    dx, dw = fp8.linear_grad(dy, x, w)

A weight is held as e4m3 values with a scale for each block of 128 x 128, an
activation or gradient with one for each row and 128 values along the
contraction (include/gleam.h, "weights in 8 bits", has the definition and the
layout).  A 128 x 128 tile is 16 KiB of contiguous bytes: in a cache with 16 KiB
chunks, an upload of ``w.q`` finds every tile that another variant of the weight
shares.

Work is enqueued on ``stream`` (a torch.cuda.Stream, its raw handle, or None for
torch's current stream) of the tensors' GPU; buffers a call needs besides its
results come from torch's allocator on that stream.  A stream that is given is recorded for
the inputs, and the caller's current one for the results, which wait for nothing by that.  Everything happens in
libgleam.so; errors raise binding.GleamError.  What only the GPU can find (a plan of other rows
than the matrix has, a wait that ran out) leaves results unwritten and is kept: check() waits for
a stream and raises it.
"""
from __future__ import annotations

import contextlib
import functools
import struct
from typing import Optional, Tuple

import torch

from . import binding as B

TILE = 128
DTYPES = {torch.bfloat16: B.GLEAM_BF16, torch.float16: B.GLEAM_FP16, torch.float32: B.GLEAM_FP32}

# The header's structs as bytes, field by field: half the time of a ctypes.Structure, where a
# call of one token is short.
_matrix_bytes = struct.Struct("@PiIQQQQ").pack
_product_bytes = struct.Struct("@QQQPPPPiiPQIIPPiiP").pack
_linear_bytes = struct.Struct("@PiIQQQQQPPPQQPIIIIPPPQP").pack

# torch's current stream as a raw handle, without the Stream object around it
_current_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice


def _check(rc: int, what: str) -> None:
    if rc < 0:
        raise B.GleamError(rc, what)


def check(device=None, stream=None) -> None:
    """Waits for the work on the stream (default: the GPU's current one) and raises what products on
    the GPU (default: the current one) have found wrong since it was last called."""
    with torch.cuda.device(device):
        if stream is None:
            stream = torch.cuda.current_stream()
        _check(B.gleam_operators_status(stream), "fp8.check")


def tiles(n: int) -> int:
    return -(-n // TILE)


class Weight:
    """An [n, k] weight, or one per expert, in 8 bits.

    q, s     uint8 [count, tiles(n), tiles(k), 128, 128] and float32 [count, tiles(n), tiles(k)]
    qt, st   the same of the transpose, for gradients (None if not kept)
    """
    __slots__ = ("n", "k", "q", "s", "qt", "st", "count")

    def __init__(self, n: int, k: int, q: torch.Tensor, s: torch.Tensor,
                 qt: Optional[torch.Tensor] = None, st: Optional[torch.Tensor] = None):
        self.n, self.k, self.q, self.s, self.qt, self.st = n, k, q, s, qt, st
        self.count = count = q.shape[0]
        a, b = -(-n // TILE), -(-k // TILE)
        _expect(q, (count, a, b, TILE, TILE), torch.uint8, "q")
        _expect(s, (count, a, b), torch.float32, "s")
        if (qt is None) != (st is None):
            raise ValueError("qt and st come together")
        if qt is not None:
            _expect(qt, (count, b, a, TILE, TILE), torch.uint8, "qt")
            _expect(st, (count, b, a), torch.float32, "st")

    def _tensors(self):
        return self.q, self.s, self.qt, self.st


def _expect(t, shape, dtype, name):
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous():
        raise ValueError("%s: expected a contiguous %s tensor of shape %s, got %s %s"
                         % (name, dtype, shape, t.dtype, tuple(t.shape)))


def _raw(t: torch.Tensor) -> Optional[int]:
    """torch's current stream on t's GPU; None if another GPU is the current one."""
    i = t.get_device()
    if i < 0:
        raise ValueError("expected a CUDA tensor")
    return _current_stream(i) if i == _current_device() else None


class _On(contextlib.ExitStack):
    """Makes t's GPU and the stream torch's current ones; entered, the raw stream."""

    def __init__(self, t: torch.Tensor, stream):
        super().__init__()
        if not t.is_cuda:
            raise ValueError("expected a CUDA tensor")
        self.index = t.get_device()
        self.enter_context(torch.cuda.device(self.index))
        if stream is not None:
            self.enter_context(torch.cuda.stream(
                torch.cuda.ExternalStream(stream, device=t.device) if isinstance(stream, int)
                else stream))

    def __enter__(self):
        super().__enter__()
        return _current_stream(self.index)


def _record(o, stream) -> None:
    """The memory of tensors, weights and plans is free again only after the stream's work so far."""
    if isinstance(o, torch.Tensor):
        o.record_stream(stream)
    elif isinstance(o, tuple):
        for part in o:
            _record(part, stream)
    elif hasattr(o, "_tensors"):
        _record(o._tensors(), stream)


def _elsewhere(t: torch.Tensor, stream, call, *args):
    """call(*args) with t's GPU and the stream as torch's current ones.  What goes in was allocated on
    another stream, and what comes out is the caller's: torch's allocator is told of both."""
    caller = torch.cuda.current_stream(t.device) if stream is not None and t.is_cuda else None
    with _On(t, stream):
        out = call(*args)
        if caller is not None:
            mine = torch.cuda.current_stream()
            if mine != caller:
                _record(args, mine)
                _record(out, caller)
    return out


def _dtype(t: torch.Tensor) -> int:
    dtype = DTYPES.get(t.dtype)
    if dtype is None:
        raise ValueError("expected bfloat16, float16 or float32, got %s" % t.dtype)
    return dtype


def _grad_types(dy, x, dw_dtype) -> torch.dtype:
    """dw's type; refuses any that the kernels have not, before there is work."""
    _dtype(dy)
    _dtype(x)
    dw_dtype = dw_dtype or x.dtype
    if dw_dtype not in DTYPES:
        raise ValueError("dw_dtype: expected bfloat16, float16 or float32, got %s" % dw_dtype)
    return dw_dtype


class _Explicit(torch.autograd.Function):
    """The result of a call whose gradients are another's: a backward pass that reaches it is told so."""

    @staticmethod
    def forward(ctx, name, grad, y, *inputs):
        ctx.message = "%s records no gradient: %s gives it" % (name, grad)
        return y

    @staticmethod
    def backward(ctx, *dy):
        raise RuntimeError(ctx.message)


def _matrix(t: torch.Tensor) -> bytes:
    """gleam_matrix_t of a [rows, cols] tensor as _rows_of returns it."""
    rows, cols = t.shape
    return _matrix_bytes(t.data_ptr(), _dtype(t), 1, rows, cols, t.stride(0) if rows > 1 else max(cols, 1), 0)


def _rows_of(t: torch.Tensor) -> torch.Tensor:
    """[..., K] as a matrix whose rows may be any distance apart; copied only where it is no such."""
    if t.dim() != 2:
        t = t.reshape(t.shape[:-1].numel(), t.shape[-1])
    if t.is_contiguous():
        return t
    if ((t.shape[1] > 1 and t.stride(1) != 1) or
            (t.shape[0] > 1 and t.stride(0) < t.shape[1])):
        t = t.contiguous()
    return t


def _groups(rows: int, cols: int, x):
    q = torch.empty((tiles(rows), tiles(cols), TILE, TILE), dtype=torch.uint8, device=x.device)
    return q, torch.empty((tiles(cols), TILE * tiles(rows)), dtype=torch.float32, device=x.device)


def _quantize(raw, x, rows, cols, direct, transposed, src=0, per_token=0):
    """(q, s, qt, st) of x in groups of 128; src (a tensor or its address) as for
    gleam_fp8_quantize."""
    q = s = qt = st = None
    if direct:
        q, s = _groups(rows, cols, x)
    if transposed:
        qt, st = _groups(cols, rows, x)
    if rows and cols:
        rc = B.lib().gleam_fp8_quantize(
            _matrix(x), B.GLEAM_FP8_GROUPS, src if type(src) is int else src.data_ptr(), per_token, rows,
            q.data_ptr() if direct else None, s.data_ptr() if direct else None,
            qt.data_ptr() if transposed else None, st.data_ptr() if transposed else None, raw)
        if rc < 0:
            raise B.GleamError(rc, "gleam_fp8_quantize")
    return q, s, qt, st


def _product(raw, m, n, k, xq, xs, wq, ws, form, y, plan=None, over=B.GLEAM_OVER_ROWS):
    e = (0, 0, 0, 0) if plan is None else (plan.experts, 0, plan.at_offsets, plan.at_counts)
    rc = B.lib().gleam_fp8_product(
        _product_bytes(m, n, k, xq.data_ptr(), xs.data_ptr(), wq.data_ptr(), ws.data_ptr(), form,
                       DTYPES[y.dtype], y.data_ptr(), max(n, 1), *e, over, 0, 0), raw)
    if rc < 0:
        raise B.GleamError(rc, "gleam_fp8_product")


def quantize_weight(w: torch.Tensor, grad: bool = False, stream=None) -> Weight:
    """An [n, k] or [experts, n, k] weight in blocks of 128 x 128; with grad its
    transpose too, which linear_grad needs."""
    raw = _raw(w) if stream is None else None
    if raw is None:
        return _elsewhere(w, stream, quantize_weight, w, grad)
    dim = w.dim()
    if dim not in (2, 3):
        raise ValueError("expected [n, k] or [experts, n, k], got shape %s" % (tuple(w.shape),))
    if w.numel() and not w.is_contiguous() and not (
            w.stride(-1) == 1 and w.stride(-2) >= w.shape[-1] and
            (dim == 2 or w.stride(0) >= w.shape[1] * w.stride(1))):
        w = w.contiguous()
    n, k = w.shape[-2:]
    count = w.shape[0] if dim == 3 else 1
    a, b = tiles(n), tiles(k)
    q = torch.empty((count, a, b, TILE, TILE), dtype=torch.uint8, device=w.device)
    s = torch.empty((count, a, b), dtype=torch.float32, device=w.device)
    qt = st = None
    if grad:
        qt = torch.empty((count, b, a, TILE, TILE), dtype=torch.uint8, device=w.device)
        st = torch.empty((count, b, a), dtype=torch.float32, device=w.device)
    dtype = _dtype(w)
    if w.numel():
        m = _matrix_bytes(w.data_ptr(), dtype, count, n, k, w.stride(-2) if n > 1 else k,
                          w.stride(0) if dim == 3 else 0)
        _check(B.lib().gleam_fp8_quantize(m, B.GLEAM_FP8_BLOCKS, None, 0, n, q.data_ptr(), s.data_ptr(),
                                          None if qt is None else qt.data_ptr(),
                                          None if st is None else st.data_ptr(), raw),
               "gleam_fp8_quantize")
    return Weight(n, k, q, s, qt, st)


def _one(w: Weight):
    if w.count != 1:
        raise ValueError("a weight of %d experts: see experts.linear" % w.count)


# what include/gleam.h's function answers for these sizes, asked once for each
@functools.lru_cache(maxsize=4096)
def _work_bytes(rows: int, k: int, experts: int) -> int:
    return B.lib().gleam_fp8_linear_work(rows, k, experts)


def _linear(raw, x, w: Weight, rows, plan=None, per_token=0):
    """y [rows, n] of x [m, k], in the order of a plan's rows if there is one (per_token 0: x is)."""
    m, k = x.shape
    n, dtype, device = w.n, x.dtype, x.device
    y = torch.empty((rows, n), dtype=dtype, device=device)
    if plan is None:
        src, e = 0, (0, 0, 0, 0)
    else:
        src = plan.at_src_of
        e = (plan.experts, 0, plan.at_offsets, plan.at_counts)
    size = _work_bytes(rows, k, e[0])
    work = torch.empty(size, dtype=torch.uint8, device=device) if size else None
    rc = (B._lib or B.lib()).gleam_fp8_linear(
        _linear_bytes(x.data_ptr(), DTYPES[dtype] if dtype in DTYPES else _dtype(x), 1, m, k, x.stride(0) if m > 1 else k or 1, 0, n,
                      w.q.data_ptr(), w.s.data_ptr(), y.data_ptr(), n or 1, rows, src, per_token, 0, *e,
                      work.data_ptr() if size else 0, size, 0), raw)
    if rc < 0:
        raise B.GleamError(rc, "gleam_fp8_linear")
    return y


def linear(x: torch.Tensor, w: Weight, stream=None) -> torch.Tensor:
    """y = x W^T for x [..., k], of x's type.  Gradients are linear_grad's: a backward pass through y
    to an x that requires one raises."""
    if w.count != 1:
        _one(w)
    shape = x.shape
    if shape[-1] != w.k:
        raise ValueError("x has %d columns, the weight %d" % (shape[-1], w.k))
    raw = _raw(x) if stream is None else None
    if raw is None:
        return _elsewhere(x, stream, linear, x, w)
    if len(shape) == 2:
        y = _linear(raw, _rows_of(x), w, shape[0])
    else:
        rows = _rows_of(x)
        y = _linear(raw, rows, w, rows.shape[0]).view(*shape[:-1], w.n)
    if x.requires_grad and torch.is_grad_enabled():
        y = _Explicit.apply("fp8.linear", "fp8.linear_grad", y, x)
    return y


def linear_grad(dy: torch.Tensor, x: torch.Tensor, w: Weight, dw_dtype: Optional[torch.dtype] = None,
                stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(dx, dw) of linear(x, w) from dy [..., n]: dx = dy W of dy's type, with dy in groups
    along n, and dw = dy^T x [n, k] of dw_dtype (default: x's), with both in groups
    of 128 rows."""
    _one(w)
    if w.qt is None:
        raise ValueError("the weight has no transpose: quantize_weight(w, grad=True)")
    if dy.shape[-1] != w.n or x.shape[-1] != w.k or dy.shape[:-1] != x.shape[:-1]:
        raise ValueError("dy %s and x %s do not fit a weight [%d, %d]"
                         % (tuple(dy.shape), tuple(x.shape), w.n, w.k))
    dw_dtype = _grad_types(dy, x, dw_dtype)
    raw = _raw(dy) if stream is None else None
    if raw is None:
        return _elsewhere(dy, stream, linear_grad, dy, x, w, dw_dtype)
    d, rows = _rows_of(dy), _rows_of(x)
    m = d.shape[0]
    dx = torch.empty((m, w.k), dtype=dy.dtype, device=dy.device)
    dw = torch.empty((w.n, w.k), dtype=dw_dtype, device=dy.device)
    q, s, qt, st = _quantize(raw, d, m, w.n, True, True)
    _, _, xq, xs = _quantize(raw, rows, m, w.k, False, True)
    _product(raw, m, w.k, w.n, q, s, w.qt, w.st, B.GLEAM_FP8_BLOCKS, dx)
    _product(raw, w.n, w.k, m, qt, st, xq, xs, B.GLEAM_FP8_GROUPS, dw)
    return (dx if dy.dim() == 2 else dx.view(*dy.shape[:-1], w.k)), dw
