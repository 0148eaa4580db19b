"""Tokens sorted by expert, the experts' products, and back.

    plan = experts.sort(ids, n_experts)          # ids [tokens, per_token] of a router
    h = experts.linear(x, plan, w)               # rows sorted by expert, each by its expert's weight
    y = experts.combine(h, plan, weights)        # sum of each token's rows, weighted
    dh, dweights = experts.combine_grad(dy, h, plan, weights)
    drows, dw = experts.linear_grad(dh, x, plan, w)
    dx = experts.combine(drows, plan)            # the gradient of tokens taken per slot

A second layer takes the sorted rows of the first: linear(act(h), plan, w2, sorted_rows=True).

Slot i = t * per_token + j of a token's j-th expert takes row plan.row_of[t, j];
plan.src_of holds a row's slot, -1 for a row that only fills an expert's last block
(include/gleam.h, "tokens by expert").  Rows of no slot are zeros in what gather and
combine_grad return and are not written by linear and linear_grad; no function here
reads them.  Gradients are the calls above: a backward pass through a result to an input that
requires one raises.  Weights are fp8.Weight with one matrix per expert.  Streams and errors
as in module fp8, whose check() also reports a plan whose offsets or counts do not fit its rows.
"""
from __future__ import annotations

import functools
from typing import Optional, Tuple

import torch

from . import binding as B
from .fp8 import (TILE, Weight, _check, _elsewhere, _expect, _Explicit, _grad_types, _linear, _matrix, _product,
                  _quantize, _raw, _rows_of)


class Plan:
    """Where each slot's row is.  int32 tensors: offsets [experts + 1], counts [experts],
    row_of [tokens, per_token], src_of [rows]."""
    __slots__ = ("experts", "align", "tokens", "per_token", "rows", "at_offsets", "at_counts",
                 "at_row_of", "at_src_of", "_buf", "_parts")

    def __init__(self, experts: int, align: int, offsets: torch.Tensor, counts: torch.Tensor,
                 row_of: torch.Tensor, src_of: torch.Tensor):
        """A plan of given parts (contiguous); sort() makes them."""
        self.experts, self.align = experts, align
        if row_of.dim() != 2 or src_of.dim() != 1:
            raise ValueError("expected row_of [tokens, per_token] and src_of [rows]")
        self.tokens, self.per_token = row_of.shape
        self.rows = src_of.shape[0]
        _expect(offsets, (experts + 1,), torch.int32, "offsets")
        _expect(counts, (experts,), torch.int32, "counts")
        _expect(row_of, row_of.shape, torch.int32, "row_of")
        _expect(src_of, src_of.shape, torch.int32, "src_of")
        self._parts, self._buf = (offsets, counts, row_of, src_of), None
        self.at_offsets, self.at_counts = offsets.data_ptr(), counts.data_ptr()
        self.at_row_of, self.at_src_of = row_of.data_ptr(), src_of.data_ptr()

    def _tensors(self):
        return self._parts if self._buf is None else self._buf

    @classmethod
    def _laid_out(cls, experts, align, tokens, per_token, rows, like):
        """A plan whose parts share one new buffer; tensors of them are made when asked for."""
        p = cls.__new__(cls)
        p.experts, p.align, p.tokens, p.per_token, p.rows = experts, align, tokens, per_token, rows
        p._parts = a = _parts(experts, tokens * per_token, rows)
        p._buf = torch.empty(a[4], dtype=torch.int32, device=like.device)
        base = p._buf.data_ptr()
        p.at_offsets, p.at_counts = base, base + 4 * a[1]
        p.at_row_of, p.at_src_of = base + 4 * a[2], base + 4 * a[3]
        return p

    # a view each time it is asked for: a buffer and all four take 9 us, 14 by one split
    def _part(self, i: int, shape: Tuple[int, ...], strides: Tuple[int, ...] = (1,)) -> torch.Tensor:
        if self._buf is None:
            return self._parts[i]
        return self._buf.as_strided(shape, strides, self._parts[i])

    @property
    def offsets(self) -> torch.Tensor:
        return self._part(0, (self.experts + 1,))

    @property
    def counts(self) -> torch.Tensor:
        return self._part(1, (self.experts,))

    @property
    def row_of(self) -> torch.Tensor:
        return self._part(2, (self.tokens, self.per_token), (self.per_token, 1))

    @property
    def src_of(self) -> torch.Tensor:
        return self._part(3, (self.rows,))


def _parts(experts: int, slots: int, rows: int):
    """Where a plan's parts start in its buffer, and its size."""
    b = experts + 4 & ~3
    c = b + (experts + 3 & ~3)
    d = c + (slots + 3 & ~3)
    return 0, b, c, d, d + (rows + 3 & ~3)


# what include/gleam.h's function answers for these sizes, asked once for each
@functools.lru_cache(maxsize=4096)
def _rows(tokens: int, per_token: int, experts: int, align: int) -> int:
    return B.lib().gleam_expert_rows(tokens, per_token, experts, align)


def sort(ids: torch.Tensor, experts: int, align: int = TILE, stream=None) -> Plan:
    """Sorts the slots of ids [tokens, per_token] (int32 or int64; an id outside 0 .. experts
    - 1 goes to no expert).  The products need align = 128 (the default)."""
    if ids.dim() != 2 or ids.dtype not in (torch.int32, torch.int64):
        raise ValueError("expected int32 or int64 ids [tokens, per_token], got %s %s"
                         % (ids.dtype, tuple(ids.shape)))
    if not 1 <= experts <= 1024 or not 1 <= align <= 1 << 20:
        raise ValueError("1 .. 1024 experts and a positive alignment")
    raw = _raw(ids) if stream is None else None
    if raw is None:
        return _elsewhere(ids, stream, sort, ids, experts, align)
    t, k = ids.shape
    ids = ids.contiguous()
    lib = B.lib()
    rows = _rows(t, k, experts, align)
    plan = Plan._laid_out(experts, align, t, k, rows, ids)
    _check(lib.gleam_expert_sort(ids.data_ptr() or None, ids.element_size(), t, k, experts, align,
                                 plan.at_offsets, plan.at_counts, plan.at_row_of, plan.at_src_of, raw),
           "gleam_expert_sort")
    return plan


def _tokens(x, plan, name):
    if x.dim() != 2 or x.shape[0] != plan.tokens:
        raise ValueError("%s: expected a row for each of %d tokens, got %s"
                         % (name, plan.tokens, tuple(x.shape)))


def _sorted_rows(rows, plan, name):
    if rows.dim() != 2 or rows.shape[0] != plan.rows:
        raise ValueError("%s: expected %d sorted rows, got %s" % (name, plan.rows, tuple(rows.shape)))


def _weights(weights, plan):
    if weights.shape != (plan.tokens, plan.per_token) or weights.dtype != torch.float32:
        raise ValueError("weights: expected float32 %s, got %s %s"
                         % ((plan.tokens, plan.per_token), weights.dtype, tuple(weights.shape)))
    return weights.contiguous()


def gather(x: torch.Tensor, plan: Plan, stream=None) -> torch.Tensor:
    """Rows [plan.rows, cols]: each slot's token, zeros for a row of no slot."""
    _tokens(x, plan, "x")
    raw = _raw(x) if stream is None else None
    if raw is None:
        return _elsewhere(x, stream, gather, x, plan)
    given, x = x, _rows_of(x)
    out = torch.empty((plan.rows, x.shape[1]), dtype=x.dtype, device=x.device)
    if out.numel():
        _check(B.lib().gleam_expert_gather(_matrix(x), plan.at_src_of, plan.per_token, plan.rows,
                                           out.data_ptr(), raw), "gleam_expert_gather")
    if given.requires_grad and torch.is_grad_enabled():
        out = _Explicit.apply("experts.gather", "experts.combine without weights", out, given)
    return out


def combine(rows: torch.Tensor, plan: Plan, weights: Optional[torch.Tensor] = None,
            stream=None) -> torch.Tensor:
    """[tokens, cols]: sum over j of weights[t, j] * the row of slot (t, j); weights None: ones."""
    _sorted_rows(rows, plan, "rows")
    raw = _raw(rows) if stream is None else None
    if raw is None:
        return _elsewhere(rows, stream, combine, rows, plan, weights)
    given, rows = (rows, weights), _rows_of(rows)
    out = torch.empty((plan.tokens, rows.shape[1]), dtype=rows.dtype, device=rows.device)
    if weights is not None:
        weights = _weights(weights, plan)
    if out.numel():
        _check(B.lib().gleam_expert_combine(_matrix(rows), plan.at_row_of,
                                            None if weights is None else weights.data_ptr() or None,
                                            plan.tokens, plan.per_token, out.data_ptr(), raw),
               "gleam_expert_combine")
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in given):
        out = _Explicit.apply("experts.combine", "experts.combine_grad", out, *given)
    return out


def combine_grad(dy: torch.Tensor, rows: torch.Tensor, plan: Plan, weights: torch.Tensor,
                 stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(drows, dweights) of combine(rows, plan, weights) from dy [tokens, cols]."""
    _tokens(dy, plan, "dy")
    _sorted_rows(rows, plan, "rows")
    if dy.dtype != rows.dtype or dy.shape[1] != rows.shape[1]:
        raise ValueError("dy and rows differ in type or columns")
    raw = _raw(dy) if stream is None else None
    if raw is None:
        return _elsewhere(dy, stream, combine_grad, dy, rows, plan, weights)
    dy, rows, weights = _rows_of(dy), _rows_of(rows), _weights(weights, plan)
    drows = torch.empty((plan.rows, dy.shape[1]), dtype=dy.dtype, device=dy.device)
    dweights = torch.empty_like(weights)
    _check(B.lib().gleam_expert_combine_grad(_matrix(dy), _matrix(rows), plan.at_row_of, plan.at_src_of,
                                             weights.data_ptr() or None, plan.per_token,
                                             drows.data_ptr() or None, dweights.data_ptr() or None, raw),
           "gleam_expert_combine_grad")
    return drows, dweights


def _fits(w: Weight, plan: Plan):
    if w.count != plan.experts:
        raise ValueError("weights of %d experts, a plan of %d" % (w.count, plan.experts))
    if plan.align % TILE:
        raise ValueError("the products need a plan with align = %d" % TILE)


def _input(x: torch.Tensor, plan: Plan, sorted_rows: bool) -> int:
    """Slots that share a row of x: a token's, or 0 where x has the sorted rows themselves."""
    if sorted_rows:
        _sorted_rows(x, plan, "x")
        return 0
    _tokens(x, plan, "x")
    return plan.per_token


def linear(x: torch.Tensor, plan: Plan, w: Weight, sorted_rows: bool = False,
           stream=None) -> torch.Tensor:
    """[plan.rows, n]: each slot's row of x times its expert's W^T.  x is [tokens, k], taken in
    sorted order as it is quantised, or with sorted_rows [plan.rows, k] (what an earlier
    linear of the layer returned)."""
    _fits(w, plan)
    per_token = _input(x, plan, sorted_rows)
    if x.shape[1] != w.k:
        raise ValueError("x has %d columns, the weights %d" % (x.shape[1], w.k))
    raw = _raw(x) if stream is None else None
    if raw is None:
        return _elsewhere(x, stream, linear, x, plan, w, sorted_rows)
    h = _linear(raw, _rows_of(x), w, plan.rows, plan, per_token)
    if x.requires_grad and torch.is_grad_enabled():
        h = _Explicit.apply("experts.linear", "experts.linear_grad", h, x)
    return h


def linear_grad(dh: torch.Tensor, x: torch.Tensor, plan: Plan, w: Weight,
                dw_dtype: Optional[torch.dtype] = None, sorted_rows: bool = False,
                stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(drows, dw) of linear(x, plan, w, sorted_rows) from dh [plan.rows, n]: drows [plan.rows, k], the
    gradient of each slot's row, and dw [experts, n, k], zeros for an expert without tokens."""
    _fits(w, plan)
    per_token = _input(x, plan, sorted_rows)
    _sorted_rows(dh, plan, "dh")
    if w.qt is None:
        raise ValueError("the weight has no transpose: quantize_weight(w, grad=True)")
    if dh.shape[1] != w.n or x.shape[1] != w.k:
        raise ValueError("dh %s and x %s do not fit weights [%d, %d]"
                         % (tuple(dh.shape), tuple(x.shape), w.n, w.k))
    dw_dtype = _grad_types(dh, x, dw_dtype)
    raw = _raw(dh) if stream is None else None
    if raw is None:
        return _elsewhere(dh, stream, linear_grad, dh, x, plan, w, dw_dtype, sorted_rows)
    dh, x = _rows_of(dh), _rows_of(x)
    drows = torch.empty((plan.rows, w.k), dtype=dh.dtype, device=dh.device)
    dw = torch.empty((w.count, w.n, w.k), dtype=dw_dtype, device=dh.device)
    q, s, qt, st = _quantize(raw, dh, plan.rows, w.n, True, True, plan.at_src_of)
    _, _, xq, xs = _quantize(raw, x, plan.rows, w.k, False, True, plan.at_src_of, per_token)
    _product(raw, plan.rows, w.k, w.n, q, s, w.qt, w.st, B.GLEAM_FP8_BLOCKS, drows, plan)
    _product(raw, w.n, w.k, plan.rows, qt, st, xq, xs, B.GLEAM_FP8_GROUPS, dw, plan, B.GLEAM_OVER_SUMS)
    return drows, dw
