"""The parts of a MoE block with gradients, as torch operations whose forward and backward are the
library's kernels: gather_rows and combine_rows (dmoe_gather_rows, dmoe_combine_rows), expert_ffn
between the two (dmoe_expert_ffn), norm_residual around them (dmoe_norm_residual), and their
_backward calls. A program may put its own expert products in expert_ffn's place:

    dmoe_sort_tokens(topk_idx, E, offsets, rows, pos, workspace=ws)
    xs = gather_rows(x, pos)                     # [T * k, d], expert by expert
    ys = expert_ffn(xs, offsets, w_gate, w_up, w_down)   # row offsets[e] .. offsets[e + 1]: expert e
    y = combine_rows(ys, pos, gates, add)        # [T, d]
    r, n = norm_residual(r, y, w_post, gate, w_pre)      # the residual, and the next block's input

moe_ffn does the first four.

Rows of slots without an expert are zeros in xs, are not read from ys, and get no gradient. The
gradients can be taken once (there is no second derivative). `pos` is int32 and must not change
between forward and backward. It has to name every row once, as dmoe_sort_tokens writes it (and
dmoe_dispatch, unless it records a fault): the kernels write the rows that it names, so that others of
xs, and of the gradient by ys, would hold what the memory held.

A forward and backward pass captured into a CUDA graph asks for its gradients with torch.autograd.grad:
leaves that accumulate them (backward()) keep the stream on which an eager pass first used them, and
torch does not let a capture wait for that one.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch
from torch.autograd.function import once_differentiable

from . import (alloc_norm_workspace, alloc_sort_workspace, dmoe_combine_rows, dmoe_combine_rows_backward,
               dmoe_expert_ffn, dmoe_expert_ffn_backward, dmoe_gather_rows, dmoe_gather_rows_backward,
               dmoe_norm_residual, dmoe_norm_residual_backward, dmoe_sort_tokens)

__all__ = ["gather_rows", "combine_rows", "expert_ffn", "moe_ffn", "norm_residual"]


def _rows(t: torch.Tensor) -> torch.Tensor:
    """The matrix with contiguous rows at least their width apart (an expanded gradient has none)."""
    if t.numel() == 0:                     # (any strides count as contiguous)
        return t.new_empty(t.shape)
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


def _rows16(t: torch.Tensor) -> torch.Tensor:
    """The same with rows that begin on 16-byte boundaries."""
    t = _rows(t)
    per = 16 // t.element_size()
    if t.data_ptr() % 16 == 0 and (t.shape[0] <= 1 or t.stride(0) % per == 0):
        return t
    return t.clone(memory_format=torch.contiguous_format)


def _dense16(t: torch.Tensor) -> torch.Tensor:
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


class _ExpertFFN(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, offsets, w_gate, w_up, w_down):
        x, w = _rows16(x), [_dense16(t) for t in (w_gate, w_up, w_down)]
        (R, d), I = x.shape, w[0].shape[1]
        want_x, _, want_g, want_u, want_d = ctx.needs_input_grad
        inner = want_x or want_g or want_u
        pre = x.new_empty((R, 2, I)) if inner else None
        h, y = x.new_empty((R, I)), x.new_empty((R, d))
        dmoe_expert_ffn(x, offsets, *w, h, y, pre=pre, zero_rest=True)
        ctx.save_for_backward(x if want_g or want_u else None, offsets, *w, pre, h if want_d else None)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, offsets, w_gate, w_up, w_down, pre, h = ctx.saved_tensors
        want_x, _, want_g, want_u, want_d = ctx.needs_input_grad
        dy = _rows16(dy)
        dpre = torch.empty_like(pre) if pre is not None else None
        dx = dy.new_empty(dy.shape) if want_x else None
        dwg, dwu = (torch.empty_like(w_gate), torch.empty_like(w_up)) if want_g or want_u else (None, None)
        dwd = torch.empty_like(w_down) if want_d else None
        if dx is not None or dwg is not None or dwd is not None:
            dmoe_expert_ffn_backward(dy, x, offsets, w_gate, w_up, w_down, pre, h, dpre, dx, dwg, dwu, dwd,
                                     zero_rest=True)
        return dx, None, dwg if want_g else None, dwu if want_u else None, dwd


def expert_ffn(x: torch.Tensor, offsets: Optional[torch.Tensor], w_gate: torch.Tensor,
               w_up: torch.Tensor, w_down: torch.Tensor) -> torch.Tensor:
    """y [R, d]: y[r] = w_down[e] (silu(w_gate[e] x[r]) * (w_up[e] x[r])) for the rows offsets[e] ..
    offsets[e + 1] of expert e (offsets int32 [E + 1], as from dmoe_sort_tokens; None: one expert, all
    rows). x, w_gate and w_up [E, I, d], w_down [E, d, I] in bf16 or fp16; d and I multiples of 8. Rows
    of no expert get zeros, and zeros as their gradient. Gradients by x and the three weights."""
    return _ExpertFFN.apply(x, offsets, w_gate, w_up, w_down)


def moe_ffn(x: torch.Tensor, topk_idx: torch.Tensor, gates: torch.Tensor, w_gate: torch.Tensor,
            w_up: torch.Tensor, w_down: torch.Tensor, add: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [T, d]: the experts of a routing that the program has (topk_idx int32 [T, k], negative: none;
    gates fp32 [T, k]), weighted and added up, with an optional addend: sort, gather_rows, expert_ffn
    and combine_rows. Gradients by x, the gates, the weights and the addend."""
    (T, k), E = topk_idx.shape, w_gate.shape[0]

    def ints(n):
        return torch.empty(n, dtype=torch.int32, device=x.device)
    offsets, rows, pos = ints(E + 1), ints(T * k), ints(T * k)
    dmoe_sort_tokens(topk_idx, E, offsets, rows, pos, workspace=alloc_sort_workspace(T, k, E, x.device))
    ys = expert_ffn(gather_rows(x, pos.view(T, k)), offsets, w_gate, w_up, w_down)
    return combine_rows(ys, pos.view(T, k), gates, add)


class _NormResidual(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, w_post, gate, w_pre, scale, eps, gate_tokens):
        ctx.set_materialize_grads(False)
        x, y, gate = (None if t is None else _rows(t) for t in (x, y, gate))
        w_post, w_pre = (None if t is None else _dense16(t) for t in (w_post, w_pre))
        r = x.new_empty(x.shape)
        n = x.new_empty(x.shape) if w_pre is not None else None
        stats = x.new_empty((2, x.shape[0]), dtype=torch.float32) if any(ctx.needs_input_grad) else None
        dmoe_norm_residual(x, y, w_post, gate, w_pre, r, n, stats=stats, scale=scale, eps=eps,
                           gate_tokens=gate_tokens)
        ctx.save_for_backward(x, y, w_post, gate, w_pre, stats)
        ctx.scale, ctx.gate_tokens = scale, gate_tokens
        return r, n

    @staticmethod
    @once_differentiable
    def backward(ctx, dr, dn):
        saved = ctx.saved_tensors
        inputs, stats = saved[:5], saved[5]
        if dr is None and dn is None:
            return (None,) * 8
        x = inputs[0]
        dr, dn = (None if t is None else _rows(t) for t in (dr, dn))
        grads = [None if t is None or not want else t.new_empty(t.shape)
                 for t, want in zip(inputs, ctx.needs_input_grad)]
        dx, dy, dw_post, dgate, dw_pre = grads
        if any(g is not None for g in grads):
            ws = alloc_norm_workspace(*x.shape, ctx.gate_tokens, x.device)
            dmoe_norm_residual_backward(*inputs, stats, dr, dn, dx, dy, dgate, dw_post, dw_pre,
                                        scale=ctx.scale, gate_tokens=ctx.gate_tokens, workspace=ws)
        return (*grads, None, None, None)


def norm_residual(x: torch.Tensor, y: Optional[torch.Tensor] = None,
                  w_post: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                  w_pre: Optional[torch.Tensor] = None, scale: float = 1.0, eps: float = 1e-6,
                  gate_tokens: Optional[int] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(r, n): r = scale * x + gate * norm(y) * w_post, the residual after a block with output y, and
    n = norm(r) * w_pre, the next block's input (None without w_pre); norm(v) = v / sqrt(mean(v^2) + eps)
    over a row. x, y [T, d] and gate in bf16, fp16 or fp32, all of one type; w_post and w_pre fp32 [d].
    Without w_post y is not normed; without y r is scale * x. gate [d] (all tokens), [T, d], or [G, d]
    with gate_tokens tokens to a row. Gradients by x, y, the gate and both weights."""
    tokens = x.shape[0]
    if gate is not None and gate.dim() == 1:
        gate = gate.unsqueeze(0)
    if gate is not None and tokens == 0:
        gate = gate[:0]                    # (its gradient is zeros)
    if gate is None:
        gate_tokens = 0
    elif gate_tokens is None:
        gate_tokens = max(tokens, 1) if gate.shape[0] == 1 else 1
    return _NormResidual.apply(x, y, w_post, gate, w_pre, float(scale), float(eps), int(gate_tokens))
