"""The sorted rows of a MoE layer with gradients: gather_rows and combine_rows as torch operations whose
forward and backward are the library's kernels (dmoe_gather_rows, dmoe_combine_rows and their
_backward calls). Between the two a program puts its own expert products:

    dmoe_sort_tokens(topk_idx, E, offsets, rows, pos, workspace=ws)
    xs = gather_rows(x, pos)                     # [T * k, d], expert by expert
    ys = ...                                     # row offsets[e] .. offsets[e + 1]: expert e
    y = combine_rows(ys, pos, gates, add)        # [T, d]

Rows of slots without an expert are zeros in xs, are not read from ys, and get no gradient. The
gradients can be taken once (there is no second derivative). `pos` is int32 and must not change
between forward and backward. It has to name every row once, as dmoe_sort_tokens writes it (and
dmoe_dispatch, unless it records a fault): the kernels write the rows that it names, so that others of
xs, and of the gradient by ys, would hold what the memory held.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import (dmoe_combine_rows, dmoe_combine_rows_backward, dmoe_gather_rows,
               dmoe_gather_rows_backward)

__all__ = ["gather_rows", "combine_rows"]


def _rows(t: torch.Tensor) -> torch.Tensor:
    """The matrix with contiguous rows at least their width apart (an expanded gradient has none)."""
    ok = t.shape[1] <= 1 or t.stride(1) == 1
    return t if ok and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1]) else t.contiguous()


class _Gather(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, pos):
        ctx.save_for_backward(pos)
        ctx.tokens = x.shape[0]
        xs = x.new_empty((pos.numel(), x.shape[1]))
        dmoe_gather_rows(_rows(x), pos, xs)
        return xs

    @staticmethod
    @once_differentiable
    def backward(ctx, dxs):
        pos, = ctx.saved_tensors
        dx = dxs.new_empty((ctx.tokens, dxs.shape[1]))
        dmoe_gather_rows_backward(_rows(dxs), pos, dx)
        return dx, None


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ys, pos, gates, add, tokens):
        # (the rows are needed for the gates' gradient only)
        ctx.save_for_backward(ys if ctx.needs_input_grad[2] else None, pos, gates)
        ctx.shape = ys.shape
        y = ys.new_empty((tokens, ys.shape[1]))
        dmoe_combine_rows(_rows(ys), pos, gates, None if add is None else _rows(add), y)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        ys, pos, gates = ctx.saved_tensors
        rows, gate = ctx.needs_input_grad[0], ctx.needs_input_grad[2]
        dys = dy.new_empty(ctx.shape) if rows else None
        dgates = torch.empty_like(gates) if gate else None
        if rows or gate:
            dmoe_combine_rows_backward(_rows(dy), _rows(ys) if gate else None, pos, gates, dys, dgates)
        return dys, None, dgates, dy if ctx.needs_input_grad[3] else None, None


def gather_rows(x: torch.Tensor, pos: torch.Tensor) -> torch.Tensor:
    """xs [T * k, d]: xs[pos[t, j]] = x[t] (x [T, d] in bf16, fp16 or fp32; pos as from dmoe_sort_tokens or
    dmoe_dispatch). Its gradient sums a token's rows in fp32."""
    return _Gather.apply(x, pos)


def combine_rows(ys: torch.Tensor, pos: torch.Tensor, gates: torch.Tensor,
                 add: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [T, d]: y[t] = add[t] + sum over the slots j of gates[t, j] * ys[pos[t, j]] (gates fp32 [T, k],
    contiguous). Gradients by ys, gates and add."""
    if gates.dim() != 2 or gates.numel() != pos.numel():
        raise ValueError("gates: expected [T, k], one for every entry of pos")
    return _Combine.apply(ys, pos, gates, add, gates.shape[0])
