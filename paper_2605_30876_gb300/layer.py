"""Resident MoE layers: device weights, workspace and output buffers around the library's calls
(argument marshalling only; the forwards run in libdmoe's kernels). MoELayer holds bf16 weights,
MoELayerQ4 the same layer's experts in 4 bits."""
from __future__ import annotations

import contextlib
from typing import Dict, Optional

import torch

from . import (DMOE_ROUTE_BLOCK, LayerDesc, alloc_q4, alloc_workspace, dmoe_combine_rows,
               dmoe_dispatch, dmoe_layer_forward, dmoe_q4_linear, dmoe_q4_quantize, dmoe_q4_size,
               dmoe_q4_swiglu, dmoe_router, dmoe_router_prepare, make_desc, make_q4_desc)

_AS_IT_IS = contextlib.nullcontext()


def _indexed(device) -> torch.device:
    """The device with its number: "cuda" is the one that is current now, whichever is later."""
    device = torch.device(device)
    if device.type == "cuda" and device.index is None:
        return torch.device("cuda", torch.cuda.current_device())
    return device


def _on(device: torch.device):
    """Makes a layer's device the current one, on which the router's and the dispatch's calls run."""
    if device.type != "cuda" or device.index == torch.cuda.current_device():
        return _AS_IT_IS
    return torch.cuda.device(device)


WEIGHT_KEYS = ("w_r", "bias", "w_gate", "w_up", "w_down", "ws_gate", "ws_up", "ws_down")


class MoELayer:
    """One MoE layer with its weights resident in HBM.

    weights: dict with w_r fp32 [d,E], bias fp32 [E] (or None), w_gate/w_up bf16 [E,I,d],
    w_down bf16 [E,d,I] and, with a shared expert, ws_gate/ws_up bf16 [I_s,d],
    ws_down bf16 [d,I_s] (None otherwise).
    """

    def __init__(self, desc: LayerDesc, weights: Dict[str, Optional[torch.Tensor]],
                 device="cuda", workspace: Optional[torch.Tensor] = None):
        self.desc = desc
        self.w = {k: weights.get(k) for k in WEIGHT_KEYS}
        self.device = _indexed(device)
        T, k, E, d = desc.T, desc.top_k, desc.n_experts, desc.d_model
        self.ws = workspace if workspace is not None else alloc_workspace(desc, self.device)
        self.y = torch.empty((T, d), dtype=torch.bfloat16, device=self.device)
        self.topk_idx = torch.empty((T, k), dtype=torch.int32, device=self.device)
        self.topk_gate = torch.empty((T, k), dtype=torch.float32, device=self.device)
        self.n_unique = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.unique_ids = torch.empty(E, dtype=torch.int32, device=self.device)
        # the router weight's tensor-core split, once (the forwards on this workspace then
        # skip it); prepare() again after changing w_r in place
        self.prepare()

    def prepare(self, stream=None) -> None:
        with _on(self.device):
            dmoe_router_prepare(self.desc, self.w["w_r"], self.ws, stream=stream)

    @classmethod
    def from_shape(cls, shape, weights, device="cuda", workspace=None) -> "MoELayer":
        desc = make_desc(shape.d_model, shape.n_experts, shape.top_k, shape.d_ff,
                         shape.d_ff_shared, shape.block_size, shape.n_blocks,
                         getattr(shape, "mode", DMOE_ROUTE_BLOCK), getattr(shape, "top_p", 0.0),
                         getattr(shape, "block_top_k", 0))
        return cls(desc, weights, device, workspace)

    def forward(self, x: torch.Tensor, y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        out = self.y if y is None else y
        w = self.w
        with _on(self.device):
            dmoe_layer_forward(self.desc, x, w["w_r"], w["bias"], w["w_gate"], w["w_up"], w["w_down"],
                               w["ws_gate"], w["ws_up"], w["ws_down"], out, self.topk_idx,
                               self.topk_gate, self.n_unique, self.unique_ids, workspace=self.ws,
                               stream=stream)
        return out


def _in_stream(stream, device):
    """What torch allocates and copies in it is on the given stream, too (None: the current one)."""
    if stream is None:
        return _AS_IT_IS
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    return torch.cuda.stream(stream)


class Q4Weight:
    """Matrices in 4 bits with group scales: codes and scales of `desc`, quantised from bf16 [n_experts,
    n_out, n_in]. `more` ([n_out, n_in], a shared expert's) is one more expert behind them. With a
    stream the weights are read on it, and codes and scales are its allocations."""

    def __init__(self, w: torch.Tensor, group: int = 64, more: Optional[torch.Tensor] = None,
                 stream=None):
        E, n_out, n_in = w.shape
        self.desc = make_q4_desc(E + (more is not None), n_out, n_in, group)
        first = make_q4_desc(E, n_out, n_in, group)
        nc, ns = dmoe_q4_size(first)
        with _in_stream(stream, w.device):
            self.codes, self.scales = alloc_q4(self.desc, w.device)
            dmoe_q4_quantize(first, w.contiguous(), self.codes[:nc], self.scales[:ns])
            if more is not None:
                dmoe_q4_quantize(make_q4_desc(1, n_out, n_in, group), more.contiguous(),
                                 self.codes[nc:], self.scales[ns:])


class MoELayerQ4:
    """MoELayer with its experts (and its shared expert) in 4 bits, a bf16 scale per `group` inputs: the
    weights that a forward reads are a quarter. The router stays fp32; the routing, the unique
    experts and the rows are those of MoELayer, the experts' outputs those of the quantised
    weights, with the SwiGLU intermediate and the rows per (token, slot) rounded to bf16.

    weights: as for MoELayer, on `device` (the bf16 expert weights are not kept). The layer runs on that
    device, on its current stream or the one given, whichever device is current.
    Its buffers and its workspace serve one forward at a time, a replayed graph's too. A token's last bits
    may differ with other tokens beside it (dmoe_q4_linear).
    """

    def __init__(self, desc: LayerDesc, weights: Dict[str, Optional[torch.Tensor]],
                 device="cuda", workspace: Optional[torch.Tensor] = None, group: int = 64):
        self.desc = desc
        self.device = _indexed(device)
        for n, t in [*((n, weights.get(n)) for n in WEIGHT_KEYS), ("workspace", workspace)]:
            if t is not None and t.device != self.device:
                raise ValueError(f"{n}: on {t.device}, the layer on {self.device}")
        T, k, E, d, I = desc.T, desc.top_k, desc.n_experts, desc.d_model, desc.d_ff
        Is = desc.d_ff_shared
        self.w_r, self.bias = weights["w_r"], weights.get("bias")
        # A shared expert of the routed ones' size is one of them, with a group of all tokens behind the
        # routed groups; one of another size has products of its own.
        self.joined = Is == I
        self.gate, self.up, self.down = (
            Q4Weight(weights["w_" + n], group, weights["ws_" + n] if self.joined else None)
            for n in ("gate", "up", "down"))
        self.shared = tuple(Q4Weight(weights[n].unsqueeze(0), group)
                            for n in ("ws_gate", "ws_up", "ws_down")) if Is > 0 and not self.joined else None
        self.ws = workspace if workspace is not None else alloc_workspace(desc, self.device)

        def new(*shape, dtype=torch.bfloat16):
            return torch.empty(shape, dtype=dtype, device=self.device)
        i32, R = torch.int32, T * k
        self.topk_idx, self.topk_gate = new(T, k, dtype=i32), new(T, k, dtype=torch.float32)
        self.n_unique = new(1, dtype=i32)
        # the dispatch's outputs, and behind them the shared expert's group
        more = 1 if self.joined else 0
        self.groups, self.ids = new(E + 1 + more, dtype=i32), new(E + more, dtype=i32)
        self.all_rows = new(R + more * T, dtype=i32)
        self.offsets, self.unique_ids = self.groups[:E + 1], self.ids[:E]
        self.rows, self.pos = self.all_rows[:R], new(R, dtype=i32)
        if self.joined:
            self.groups[E + 1:].fill_(R + T)
            self.ids[E:].fill_(E)
            self.all_rows[R:] = torch.arange(0, R, k, dtype=i32, device=self.device)
        self.h, self.ys, self.y = new(R + more * T, I), new(R + more * T, d), new(T, d)
        self.hs = new(T, Is) if self.shared is not None else None
        self.y_shared = self.ys[R:] if self.joined else new(T, d) if Is > 0 else None
        self.prepare()

    def prepare(self, stream=None) -> None:
        with _on(self.device):
            dmoe_router_prepare(self.desc, self.w_r, self.ws, stream=stream)

    @classmethod
    def from_shape(cls, shape, weights, device="cuda", workspace=None, group=64) -> "MoELayerQ4":
        desc = make_desc(shape.d_model, shape.n_experts, shape.top_k, shape.d_ff,
                         shape.d_ff_shared, shape.block_size, shape.n_blocks,
                         getattr(shape, "mode", DMOE_ROUTE_BLOCK), getattr(shape, "top_p", 0.0),
                         getattr(shape, "block_top_k", 0))
        return cls(desc, weights, device, workspace, group)

    def forward(self, x: torch.Tensor, y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        # (the router goes by the desc's sizes, the other calls by the tensors')
        self._check(x, "x")
        if y is not None:
            self._check(y, "y")
        out = self.y if y is None else y
        with _on(self.device):
            self._forward(x, out, stream)
        return out

    def _check(self, t, name) -> None:
        if t.shape != self.y.shape or t.device != self.y.device:
            raise ValueError(f"{name}: expected {tuple(self.y.shape)} on {self.y.device}, "
                             f"got {tuple(t.shape)} on {t.device}")

    def _forward(self, x, out, stream) -> None:
        k = self.desc.top_k
        dmoe_router(self.desc, x, self.w_r, self.bias, self.topk_idx, self.topk_gate,
                    workspace=self.ws, stream=stream)
        dmoe_dispatch(self.desc, self.topk_idx, self.n_unique, self.unique_ids, self.offsets,
                      self.rows, self.pos, workspace=self.ws, stream=stream)
        g, u, d = self.gate, self.up, self.down
        dmoe_q4_swiglu(g.desc, x, self.groups, g.codes, g.scales, u.codes, u.scales, self.h,
                       rows=self.all_rows, k=k, expert_ids=self.ids, stream=stream)
        dmoe_q4_linear(d.desc, self.h, self.groups, d.codes, d.scales, self.ys,
                       expert_ids=self.ids, stream=stream)
        if self.shared is not None:
            g, u, d = self.shared
            dmoe_q4_swiglu(g.desc, x, None, g.codes, g.scales, u.codes, u.scales, self.hs,
                           stream=stream)
            dmoe_q4_linear(d.desc, self.hs, None, d.codes, d.scales, self.y_shared, stream=stream)
        dmoe_combine_rows(self.ys[:self.desc.T * k], self.pos, self.topk_gate, self.y_shared, out,
                          stream=stream)
