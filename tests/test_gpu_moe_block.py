"""A MoE block for training and serving by its parts: norms, sort, gather, experts, combine, residual
together, the torch operations' gradients, and MoEBlock."""
import pytest
import torch

import paper_2605_30876_gb300 as dm
from paper_2605_30876_gb300.autograd import combine_rows, expert_ffn, gather_rows, moe_ffn, norm_residual
from paper_2605_30876_gb300.layer import MoEBlock, MoELayer
from tests import ffn_oracle as F
from tests import norm_oracle as N

pytestmark = pytest.mark.gpu


def new(gen, *shape, size=1.0, dtype=torch.bfloat16):
    return torch.empty(shape, device="cuda").normal_(0, size, generator=gen).to(dtype)


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def routing(gen, T, k, E, masked=0.1):
    idx = torch.rand((T, E), device="cuda", generator=gen).topk(k, 1).indices.to(torch.int32)
    off = torch.rand((T, k), device="cuda", generator=gen) < masked
    gates = torch.rand((T, k), device="cuda", generator=gen) + 0.1
    return torch.where(off, -1, idx), gates


def block64(x, idx, gates, w_gate, w_up, w_down, add=None):
    """The experts' weighted sum in 64 bits, expert by expert, with torch's gradients."""
    y = torch.zeros_like(x) if add is None else add
    for e in range(w_gate.shape[0]):
        t, j = torch.nonzero(idx == e, as_tuple=True)
        if len(t):
            g = x[t] @ w_gate[e].t()
            h = g * torch.sigmoid(g) * (x[t] @ w_up[e].t())
            y = y.index_add(0, t, gates[t, j, None] * (h @ w_down[e].t()))
    return y


def leaves(*tensors):
    return [t.detach().clone().requires_grad_() for t in tensors]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_expert_ffn_gradients_against_the_formula_and_differences(dtype):
    gen = generator(0)
    E, d, I, counts = 3, 72, 40, [17, 0, 50]
    R, offsets = 70, torch.tensor([0, 17, 17, 67], dtype=torch.int32, device="cuda")
    args = leaves(new(gen, R, d, dtype=dtype), new(gen, E, I, d, size=d ** -0.5, dtype=dtype),
                  new(gen, E, I, d, size=d ** -0.5, dtype=dtype), new(gen, E, d, I, size=I ** -0.5, dtype=dtype))
    x, *w = args
    y = expert_ffn(x, offsets, *w)
    dy = new(gen, R, d, dtype=dtype)
    grads = torch.autograd.grad(y, args, dy)
    with torch.no_grad():
        fwd = F.forward(x, offsets.tolist(), *w)
        F.check("y", y, fwd["y"])
        assert (y[67:] == 0).all() and (grads[0][67:] == 0).all()
        pre = torch.stack([fwd["g"][0], fwd["u"][0]], 1)
        want = F.backward(dy, x, offsets.tolist(), *w, pre, fwd["h"][0], [fwd[n][1] for n in "guh"])
        bounds = {}
        for name, g in zip(("dx", "dw_gate", "dw_up", "dw_down"), grads):
            F.check(name, g, want[name])
            bounds[name] = want[name][1].nan_to_num(0.0)

        def loss(*a):
            v = F.forward(*[a[0].double(), offsets.tolist()], *[t.double() for t in a[1:]])["y"][0]
            return (v[:67] * dy[:67].double()).sum()
        step = 1e-5
        for i, (name, g) in enumerate(zip(bounds, grads)):
            v = torch.empty(g.shape, dtype=torch.float64, device="cuda").normal_(generator=gen)
            at = [t.double() for t in args]
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + step * v, at[i] - step * v
            slope = (loss(*up) - loss(*down)) / (2 * step)
            mine = (g.double() * v).sum()
            # the gradient's bounds, and the difference's own: a third derivative of the loss's size
            # times step^2, and the loss's last bits over the step
            room = (bounds[name] * v.abs()).sum() + 1e-6 * slope.abs() + 1e-8
            assert (slope - mine).abs() <= room, (name, slope.item(), mine.item(), room.item())


def test_expert_ffn_of_any_rows_and_weights():
    """Rows and weights whose strides or bases the kernels do not take are copied."""
    gen = generator(1)
    x = new(gen, 30, 73)[:, 1:]
    w = [new(gen, 1 + 2 * 40 * 72)[1:].view(2, 40, 72), new(gen, 2, 72, 40).transpose(1, 2), new(gen, 2, 72, 40)]
    offsets = torch.tensor([0, 10, 30], dtype=torch.int32, device="cuda")
    got = expert_ffn(x, offsets, *w)
    assert torch.equal(got, expert_ffn(x.contiguous(), offsets, *[t.clone(memory_format=torch.contiguous_format) for t in w]))
    expanded = new(gen, 1, 72).requires_grad_()
    y = expert_ffn(expanded.expand(30, 72), offsets, *w)
    y.sum().backward()                     # (a gradient expanded from one number, too)
    assert expanded.grad.shape == (1, 72) and torch.isfinite(expanded.grad).all()


@pytest.mark.parametrize("wanted", [(0,), (1,), (2, 3), (3,), (0, 2)])
def test_expert_ffn_gradients_that_are_wanted(wanted):
    gen = generator(2)
    args = [new(gen, 40, 72), new(gen, 2, 40, 72, size=0.1), new(gen, 2, 40, 72, size=0.1), new(gen, 2, 72, 40, size=0.1)]
    offsets = torch.tensor([0, 15, 40], dtype=torch.int32, device="cuda")
    dy = new(gen, 40, 72)
    every = leaves(*args)
    whole = torch.autograd.grad(expert_ffn(every[0], offsets, *every[1:]), every, dy)
    some = [t.clone().requires_grad_(i in wanted) for i, t in enumerate(args)]
    expert_ffn(some[0], offsets, *some[1:]).backward(dy)
    for i, t in enumerate(some):
        assert (t.grad is None) if i not in wanted else torch.equal(t.grad, whole[i])
    with torch.no_grad():
        assert torch.equal(expert_ffn(args[0], offsets, *args[1:]), expert_ffn(every[0], offsets, *every[1:]))


@pytest.mark.parametrize("gate_shape", ["channel", "token", "groups", None])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm_residual_gradients_against_the_formula_and_differences(dtype, gate_shape):
    gen = generator(3)
    T, d = 50, 72
    G = {"channel": T, "token": 1, "groups": 7, None: 0}[gate_shape]
    gate = None if G == 0 else new(gen, d, dtype=dtype) if G == T else new(gen, -(-T // G), d, dtype=dtype)
    vec = lambda: 1 + new(gen, d, size=0.2, dtype=torch.float32)
    args = [new(gen, T, d, dtype=dtype), new(gen, T, d, dtype=dtype), vec(), gate, vec()]
    args = [None if t is None else t.requires_grad_() for t in args]
    x, y, w_post, gate, w_pre = args
    r, n = norm_residual(x, y, w_post, gate, w_pre, scale=0.8, eps=1e-5, gate_tokens=7 if G == 7 else None)
    dr, dn = new(gen, T, d, dtype=dtype), new(gen, T, d, dtype=dtype)
    some = [t for t in args if t is not None]
    grads = iter(torch.autograd.grad([r, n], some, [dr, dn]))
    grads = dict(zip(("dx", "dy", "dw_post", "dgate", "dw_pre"), (None if t is None else next(grads) for t in args)))
    with torch.no_grad():
        rows = None if gate is None else gate.view(-1, d)
        want = N.norm_residual(x, y, w_post, rows, w_pre, 0.8, 1e-5, max(G, 1), dr, dn)
        N.check("r", r, want["r"])
        N.check("n", n, want["n"])
        for k, g in grads.items():
            if g is not None:
                N.check(k, g.view(want[k][0].shape), want[k])

        def loss(*a):
            v = N.norm_residual(*a[:3], None if a[3] is None else a[3].view(-1, d), a[4], 0.8, 1e-5, max(G, 1))
            return (v["r"][0] * dr.double()).sum() + (v["n"][0] * dn.double()).sum()
        step = 1e-5
        for i, (k, g) in enumerate(grads.items()):
            if g is None:
                continue
            v = torch.empty(g.shape, dtype=torch.float64, device="cuda").normal_(generator=gen)
            at = [None if t is None else t.double() for t in args]
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + step * v, at[i] - step * v
            slope = (loss(*up) - loss(*down)) / (2 * step)
            room = (want[k][1].view(g.shape) * v.abs()).sum() + 1e-6 * slope.abs() + 1e-8
            assert (slope - (g.double() * v).sum()).abs() <= room, k


def test_norm_residual_parts():
    gen = generator(4)
    x = new(gen, 20, 72).requires_grad_()
    w = torch.ones(72, device="cuda", requires_grad=True)
    r, n = norm_residual(x, w_pre=w)             # the norm before a block alone
    assert torch.equal(r, x)
    n.sum().backward()
    assert x.grad is not None and w.grad is not None
    r, n = norm_residual(x, x.detach())          # a residual alone
    assert n is None and torch.equal(r, x + x.detach())
    x.grad = None
    r, n = norm_residual(x, w_pre=w)
    r.sum().backward()                            # n not used
    assert torch.equal(x.grad, torch.ones_like(x))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_block_in_training(dtype):
    """norm, sort, gather, experts, combine, norm with gate and residual, forward and backward, against
    64 bits. Between input and results a value is rounded at most 12 times (n, g, u, h, the row, y, r
    and back), by half a step each; products and norms add the roundings of their terms up in
    quadrature at worst twice as large as the terms, so that the 2-norm of an output is off by at
    most 12 * 2 half steps of its own (a weight's gradient, a sum over tokens, as well)."""
    gen = generator(5)
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

    a64 = [t.detach().double().requires_grad_() for t in args]
    X, g64, wi, wp, wo, ga, *w64 = a64
    norm = lambda v: v * ((v * v).mean(1, keepdim=True) + 1e-6) ** -0.5
    n64 = norm(X) * wi
    y64 = block64(n64, idx, g64, *w64, add=n64)
    r64 = X + ga.repeat_interleave(32, 0)[:T] * norm(y64) * wp
    o64 = norm(r64) * wo
    want = [r64, o64, *torch.autograd.grad([r64, o64], a64, [dr.double(), dn.double()])]
    room = 24 * torch.finfo(dtype).eps / 2
    for i, (a, b) in enumerate(zip(got, want)):
        off = (a.double() - b).norm() / b.norm()
        assert off <= room, (i, off.item())
    assert dm.dmoe_expert_device_error()[0] == 0


def test_no_tokens():
    """The gradients of what all tokens share are zeros then."""
    gen = generator(9)
    w = [new(gen, 2, 40, 72), new(gen, 2, 40, 72), new(gen, 2, 72, 40)]
    for gate in (new(gen, 72), new(gen, 0, 72), None):
        x, y = leaves(new(gen, 0, 72), new(gen, 0, 72))
        w_post, w_pre = (torch.ones(72, device="cuda", requires_grad=True) for _ in range(2))
        ws = leaves(*w)
        gate = None if gate is None else gate.requires_grad_()
        idx, gates = torch.zeros((0, 2), dtype=torch.int32, device="cuda"), torch.zeros((0, 2), device="cuda")
        r, n = norm_residual(x, moe_ffn(y, idx, gates, *ws), w_post, gate, w_pre)
        (r.sum() + n.sum()).backward()
        for t in (w_post, w_pre, gate, *ws):
            assert t is None or (t.grad.shape == t.shape and (t.grad == 0).all())


def test_a_captured_training_step():
    """Forward and backward of a block in a graph, replayed on other values. (Gradients are asked for by
    name: leaves that accumulate them keep the stream of their first use.)"""
    gen = generator(10)
    T, k, E, d, I = 150, 2, 4, 72, 40
    idx, gates = routing(gen, T, k, E)
    vec = lambda: 1 + new(gen, d, size=0.2, dtype=torch.float32)
    args = leaves(new(gen, T, d), gates, vec(), vec(), new(gen, -(-T // 32), d),
                  new(gen, E, I, d, size=0.1), new(gen, E, I, d, size=0.1), new(gen, E, d, I, size=0.1))
    dr, dn = new(gen, T, d), new(gen, T, d)

    def step():
        x, gates, w_in, w_out, gate, *w = args
        _, n = norm_residual(x, w_pre=w_in)
        r, n = norm_residual(x, moe_ffn(n, idx, gates, *w), None, gate, w_out, gate_tokens=32)
        return [r, n, *torch.autograd.grad([r, n], args, [dr, dn])]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    with torch.no_grad():
        args[0].mul_(-0.5)
        idx.copy_(idx.flip(0))
    want = step()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_moe_ffn_is_its_parts():
    gen = generator(6)
    T, k, E, d, I = 60, 3, 5, 72, 40
    idx, gates = routing(gen, T, k, E)
    x, w = new(gen, T, d), (new(gen, E, I, d, size=0.1), new(gen, E, I, d, size=0.1), new(gen, E, d, I, size=0.1))
    ints = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")
    offsets, rows, pos = ints(E + 1), ints(T * k), ints(T * k)
    dm.dmoe_sort_tokens(idx, E, offsets, rows, pos, workspace=dm.alloc_sort_workspace(T, k, E))
    y = combine_rows(expert_ffn(gather_rows(x, pos.view(T, k)), offsets, *w), pos.view(T, k), gates)
    assert torch.equal(y, moe_ffn(x, idx, gates, *w))
    none = torch.full_like(idx, -1)
    assert torch.equal(moe_ffn(x, none, gates, *w, add=x), x)       # no slot has an expert
    empty = moe_ffn(x[:0], idx[:0], gates[:0], *w)
    assert empty.shape == (0, d)


def test_experts_on_a_dispatch():
    """The serving form on dmoe_dispatch's groups (unique experts), one token and a block of them."""
    for T in (1, 32):
        gen = generator(7)
        E, d, I, k = 16, 256, 128, 4
        desc = dm.make_desc(d, E, k, I, 0, T, 1, dm.DMOE_ROUTE_TOKEN)
        idx, gates = routing(gen, T, k, E, masked=0.0)
        ints = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")
        n_unique, ids, offsets, rows, pos = ints(1), ints(E), ints(E + 1), ints(T * k), ints(T * k)
        dm.dmoe_dispatch(desc, idx, n_unique, ids, offsets, rows, pos, workspace=dm.alloc_workspace(desc))
        x, w = new(gen, T, d), (new(gen, E, I, d, size=0.06), new(gen, E, I, d, size=0.06), new(gen, E, d, I, size=0.1))
        xs = gather_rows(x, pos.view(T, k))
        h, ys = torch.empty((T * k, I), dtype=torch.bfloat16, device="cuda"), torch.empty_like(xs)
        dm.dmoe_expert_ffn(xs, offsets, *w, h, ys, expert_ids=ids)
        want = F.forward(xs, offsets.tolist(), *w, ids.tolist())
        assert not torch.isnan(want["y"][0]).any()
        F.check("y", ys, want["y"])


def test_moe_block():
    from dmoe_synth import TINY, layer_inputs
    gen = generator(8)
    s = TINY
    desc = dm.make_desc(s.d_model, s.n_experts, s.top_k, s.d_ff, s.d_ff_shared, s.block_size, s.n_blocks,
                        dm.DMOE_ROUTE_BLOCK, 0.6, 0)
    T, d, E, I, Is = desc.T, desc.d_model, desc.n_experts, desc.d_ff, desc.d_ff_shared
    w = dict(w_r=new(gen, d, E, size=d ** -0.5, dtype=torch.float32), bias=None,
             w_gate=new(gen, E, I, d, size=0.05), w_up=new(gen, E, I, d, size=0.05), w_down=new(gen, E, d, I, size=0.05))
    if Is:
        w.update(ws_gate=new(gen, Is, d, size=0.05), ws_up=new(gen, Is, d, size=0.05), ws_down=new(gen, d, Is, size=0.05))
    layer = MoELayer(desc, w)
    vec = lambda: 1 + new(gen, d, size=0.2, dtype=torch.float32)
    w_in, w_post, w_pre = vec(), vec(), vec()
    block = MoEBlock(layer, w_post, w_pre, scale=0.9)
    r, gate = new(gen, T, d), new(gen, -(-T // s.block_size), d)
    n = block.enter(r, w_in)
    N.check("n", n, N.norm_residual(r, None, None, None, w_in, 1.0, 1e-6, 0)["n"])
    r2, n2 = block.forward(r, n, gate, gate_tokens=s.block_size)
    want = N.norm_residual(r, layer.y, w_post, gate, w_pre, 0.9, 1e-6, s.block_size)
    N.check("r", r2, want["r"])
    N.check("n", n2, want["n"])
    keep = r2.clone(), n2.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    again = block.forward(r, n, gate, s.block_size, r_out=r, n_out=n, stream=side)   # in place
    torch.cuda.synchronize()
    assert again[0] is r and torch.equal(r, keep[0]) and torch.equal(n, keep[1])
