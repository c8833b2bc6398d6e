"""MoEBlock around a layer whose experts are in 4 bits, and a MoE block's training pass against one in 64 bits that
rounds where the kernels do."""
import pytest
import torch

import paper_2605_30876_gb300 as dm
from paper_2605_30876_gb300.autograd import moe_ffn, norm_residual
from paper_2605_30876_gb300.layer import MoEBlock, MoELayerQ4
from tests import norm_oracle as N
from tests.test_gpu_moe_block import generator, leaves, new, routing

pytestmark = pytest.mark.gpu


def test_moe_block_over_4_bit_experts():
    from dmoe_synth import TINY
    gen = generator(21)
    s = TINY
    desc = dm.make_desc(s.d_model, s.n_experts, s.top_k, s.d_ff, s.d_ff_shared, s.block_size, s.n_blocks,
                        dm.DMOE_ROUTE_BLOCK, 0.6, 0)
    T, d, E, I, Is = desc.T, desc.d_model, desc.n_experts, desc.d_ff, desc.d_ff_shared
    w = dict(w_r=new(gen, d, E, size=d ** -0.5, dtype=torch.float32), bias=None,
             w_gate=new(gen, E, I, d, size=0.05), w_up=new(gen, E, I, d, size=0.05), w_down=new(gen, E, d, I, size=0.05))
    if Is:
        w.update(ws_gate=new(gen, Is, d, size=0.05), ws_up=new(gen, Is, d, size=0.05), ws_down=new(gen, d, Is, size=0.05))
    layer = MoELayerQ4(desc, w)
    vec = lambda: 1 + new(gen, d, size=0.2, dtype=torch.float32)
    w_in, w_post, w_pre = vec(), vec(), vec()
    block = MoEBlock(layer, w_post, w_pre, scale=0.9)
    r, gate = new(gen, T, d), new(gen, -(-T // s.block_size), d)
    n = block.enter(r, w_in)
    r2, n2 = block.forward(r, n, gate, gate_tokens=s.block_size)
    y = layer.y.clone()
    assert torch.equal(layer.forward(n, y=torch.empty_like(y)), y) and y.abs().max() > 0
    want = N.norm_residual(r, y, w_post, gate, w_pre, 0.9, 1e-6, s.block_size)
    N.check("r", r2, want["r"])
    N.check("n", n2, want["n"])
    keep = r2.clone(), n2.clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    block.forward(r, n, gate, s.block_size, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(block.r, keep[0]) and torch.equal(block.n, keep[1])
    with torch.cuda.graph(graph):
        block.forward(r, n, gate, s.block_size)
    block.r.zero_(), block.n.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(block.r, keep[0]) and torch.equal(block.n, keep[1])
    again = block.forward(r, n, gate, s.block_size, r_out=r, n_out=n)       # in place
    assert again[0] is r and torch.equal(r, keep[0]) and torch.equal(n, keep[1])


class Rounded(torch.autograd.Function):
    """A tensor of the rows' type between two kernels: its values and its gradient are rounded to it."""

    @staticmethod
    def forward(ctx, v, dtype):
        ctx.dtype = dtype
        return v.to(dtype).double()

    @staticmethod
    def backward(ctx, g):
        return g.to(ctx.dtype).double(), None


class Inner(torch.autograd.Function):
    """h = silu(g) u, rounded; its gradients from g and u as the forward pass keeps them, rounded."""

    @staticmethod
    def forward(ctx, g, u, dtype):
        ctx.save_for_backward(g.to(dtype).double(), u.to(dtype).double())
        ctx.dtype = dtype
        return (g * torch.sigmoid(g) * u).to(dtype).double()

    @staticmethod
    def backward(ctx, dh):
        g, u = ctx.saved_tensors
        s = torch.sigmoid(g)
        dg, du = dh * u * s * (1 + g * (1 - s)), dh * g * s
        return dg.to(ctx.dtype).double(), du.to(ctx.dtype).double(), None


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_block_in_training_rounds_where_it_says(dtype):
    """Both passes against 64 bits with a rounding wherever a tensor of the type stands between two kernels. What is left
    are values that an error in fp32 takes over the middle between two of the type: one whole step each. A sum of K <=
    136 products of one size has an error of at most K * 2^-23 of the sum of their sizes, about sqrt(K) of the sum itself: 2e-4. In
    fp16 (steps of 2^-11 .. 2^-10 of a value) that is a third of a step, in bf16 less, so that of a dozen roundings on
    the way at most a third of the elements are a step (two half steps) off each: in quadrature sqrt(12 / 3) * 2 = 4
    half steps of the 2-norm."""
    gen = generator(22)
    T, k, E, d, I = 333, 4, 8, 136, 72
    idx, gates = routing(gen, T, k, E)
    vec = lambda: 1 + new(gen, d, size=0.2, dtype=torch.float32)
    args = leaves(new(gen, T, d, dtype=dtype), gates, vec(), vec(), vec(), new(gen, -(-T // 32), d, size=0.5, dtype=dtype),
                  new(gen, E, I, d, size=d ** -0.5, dtype=dtype), new(gen, E, I, d, size=d ** -0.5, dtype=dtype),
                  new(gen, E, d, I, size=I ** -0.5, dtype=dtype))
    x, gates, w_in, w_post, w_out, gate, *w = args
    _, n = norm_residual(x, w_pre=w_in)
    y = moe_ffn(n, idx, gates, *w, add=n)
    r, n2 = norm_residual(x, y, w_post, gate, w_out, gate_tokens=32)
    dr, dn = new(gen, T, d, dtype=dtype), new(gen, T, d, dtype=dtype)
    got = [r, n2, *torch.autograd.grad([r, n2], args, [dr, dn])]

    rd = lambda v: Rounded.apply(v, dtype)
    a64 = [t.detach().double().requires_grad_() for t in args]
    X, g64, wi, wp, wo, ga, wg, wu, wd = a64
    norm = lambda v: v * ((v * v).mean(1, keepdim=True) + 1e-6) ** -0.5
    n64 = rd(norm(rd(X)) * wi)           # (each use of x and of n gives a rounded gradient)
    rows, y64 = rd(n64), rd(n64)
    for e in range(E):
        t, j = torch.nonzero(idx == e, as_tuple=True)
        if len(t):
            xs = rd(rows[t])
            ys = rd(Inner.apply(xs @ wg[e].t(), xs @ wu[e].t(), dtype) @ wd[e].t())
            y64 = y64.index_add(0, t, g64[t, j, None] * ys)
    y64 = rd(y64)
    r64 = rd(X) + ga.repeat_interleave(32, 0)[:T] * norm(y64) * wp
    o64 = norm(r64) * wo
    want = [r64, o64, *torch.autograd.grad([r64, o64], a64, [dr.double(), dn.double()])]
    room = 4 * torch.finfo(dtype).eps / 2
    for i, (a, b) in enumerate(zip(got, want)):
        b = b.to(a.dtype).double()
        off = (a.double() - b).norm() / b.norm()
        assert off <= room, (i, off.item())
