"""The parts of a layer together, as programs use them: experts of one's own between the gather and the
combine, trained; the layer with its experts in 4 bits; both captured."""
import numpy as np
import pytest
import torch

from dmoe_synth import LAYER, ROUTE_TOKEN, TINY, layer_inputs
from tests import parity as P
from tests import rows_oracle as O
from tests.test_gpu_q4 import bounds, f64, swiglu_bounds

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def parts():
    from paper_2605_30876_gb300 import autograd
    return autograd


def sorted_rows(idx, E):
    m = P.dm()
    T, k = idx.shape
    out = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (E + 1, T * k, T * k)]
    m.dmoe_sort_tokens(idx, E, *out, workspace=m.alloc_sort_workspace(T, k, E))
    return out


def problem(T, k, E, d, seed, masked):
    gen = torch.Generator().manual_seed(seed)
    idx = torch.stack([torch.randperm(E, generator=gen)[:k] for _ in range(T)]).to(torch.int32)
    if masked:
        idx[torch.rand(T, k, generator=gen) < 0.2] = -1
        idx[T // 2] = -1
    x = torch.randn(T, d, generator=gen)
    w = torch.randn(E, d, d, generator=gen) / d ** 0.5
    logits = torch.randn(T, k, generator=gen)
    add = torch.randn(T, d, generator=gen)
    return idx, x, w, logits, add


def plain(idx, x, w, logits, add):
    """The same layer token by token, in the inputs' precision."""
    gates = torch.softmax(logits, 1)
    y = []
    for t in range(x.shape[0]):
        acc = add[t]
        for j in range(idx.shape[1]):
            if idx[t, j] >= 0:
                acc = acc + gates[t, j] * torch.tanh(x[t] @ w[int(idx[t, j])])
        y.append(acc)
    return torch.stack(y)


def by_parts(idx, x, w, logits, add):
    A = parts()
    E = w.shape[0]
    offsets, rows, pos = sorted_rows(idx.cuda(), E)
    first = offsets.tolist()
    xs = A.gather_rows(x, pos)
    ys = torch.cat([torch.tanh(xs[first[e]:first[e + 1]] @ w[e]) for e in range(E)]
                   + [xs[first[E]:]])
    return A.combine_rows(ys, pos, torch.softmax(logits, 1), add)


@pytest.mark.parametrize("T,k,E,d,masked", [(1, 1, 3, 4, False), (23, 3, 7, 24, True), (40, 4, 4, 17, True)])
def test_training_step_by_parts(T, k, E, d, masked):
    idx, *leaves = problem(T, k, E, d, T, masked)
    dy = torch.randn(T, d, generator=torch.Generator().manual_seed(99))
    a = [t.double().requires_grad_() for t in leaves]
    ya = plain(idx, *a)
    ga = torch.autograd.grad(ya, a, dy.double())
    b = [t.cuda().requires_grad_() for t in leaves]
    yb = by_parts(idx, *b)
    gb = torch.autograd.grad(yb, b, dy.cuda())
    # fp32 throughout: products of d terms, sums of k slots and of the rows of an expert (at most T),
    # tanh and softmax within a few units. Every intermediate is below 8 in magnitude here, every
    # sum has at most T + d + k terms of at most 8 * 8: the error is below (T + d + k + 16) 2^-24 times that.
    tol = (T + d + k + 16) * 2.0 ** -24 * 64 * d ** 0.5
    assert not torch.backends.cuda.matmul.allow_tf32
    for p, q in zip([ya, *ga], [yb, *gb]):
        assert (p.detach() - q.detach().double().cpu()).abs().max().item() <= tol


def test_gradients_by_differences():
    """Differences in fp32: f is a sum of about 100 terms of order one, off by 2^-20 or so; over h = 2^-6
    that is 2^-13, and the third derivative's share h^2 / 6 is 2^-14."""
    A = parts()
    T, k, E, d = 5, 2, 4, 6
    idx, x, w, logits, add = problem(T, k, E, d, 1, True)
    _, _, pos = sorted_rows(idx.cuda(), E)
    gen = torch.Generator().manual_seed(3)
    ys = torch.randn(T * k, d, generator=gen).cuda()
    gates = torch.rand(T, k, generator=gen).cuda()
    dy = torch.randn(T, d, generator=gen).cuda()
    c = torch.randn(T * k, d, generator=gen).cuda()

    def f(x, ys, gates, add):
        return (A.combine_rows(ys, pos, gates, add) * dy).sum() + (A.gather_rows(x, pos) * c).sum()
    args = [x.cuda(), ys, gates, add.cuda()]
    leaves = [t.clone().requires_grad_() for t in args]
    grads = torch.autograd.grad(f(*leaves), leaves)
    h = 2.0 ** -6
    for i, g in enumerate(grads):
        flat = g.reshape(-1)
        for j in range(0, flat.numel(), 3):
            up, down = [t.clone() for t in args], [t.clone() for t in args]
            up[i].view(-1)[j] += h
            down[i].view(-1)[j] -= h
            num = (f(*up) - f(*down)).item() / (2 * h)
            assert abs(num - flat[j].item()) < 2.0 ** -11


def test_only_the_gradients_that_are_asked_for():
    A = parts()
    idx, x, w, logits, add = problem(9, 2, 4, 8, 0, True)
    _, _, pos = sorted_rows(idx.cuda(), 4)
    ys = torch.randn(18, 8, device="cuda", requires_grad=True)
    gates = torch.rand(9, 2, device="cuda")
    y = A.combine_rows(ys, pos, gates)
    y.sum().backward()                               # (an expanded gradient)
    want = O.combine_backward(np.ones((9, 8)), None, pos.cpu().numpy(), f64(gates))[0]
    assert np.array_equal(f64(ys.grad), want.astype(np.float32).astype(np.float64))
    gates.requires_grad_()
    y = A.combine_rows(ys.detach(), pos, gates)
    g, = torch.autograd.grad(y.sum(), gates)
    assert g.shape == gates.shape and ys.grad is not None
    xt = torch.randn(8, 9, device="cuda").t().requires_grad_()     # rows that are not contiguous
    xs = A.gather_rows(xt, pos)
    assert np.array_equal(f64(xs.detach()), O.gather(f64(xt.detach()), pos.cpu().numpy(), 2))
    g, = torch.autograd.grad((xs * 2).sum(), xt)
    assert g.shape == xt.shape


# ------------------------------------------------------------------------------ 4-bit layer

def layer_bounds(shape, host, vals, svals, idx, gates):
    """(y, how far it may be off) of the quantised layer on this routing, in 64 bits: the products'
    sums and roundings as in the products' own tests, carried through the steps."""
    T, k, d = shape.T, shape.top_k, shape.d_model
    x = host["x"]
    y, err, mag = np.zeros((T, d)), np.zeros((T, d)), np.zeros((T, d))

    def expert(rows, g, u, dn):
        a, am = rows @ g.T, np.abs(rows) @ np.abs(g).T
        b, bm = rows @ u.T, np.abs(rows) @ np.abs(u).T
        h, he = swiglu_bounds(a, am, b, bm, d, BF16)
        o, om = h @ dn.T, (np.abs(h) + he) @ np.abs(dn).T
        oe = he @ np.abs(dn).T
        return o, oe + bounds(np.abs(o) + oe, om, h.shape[1], BF16)[1]
    for e in np.unique(idx):
        t, j = np.nonzero(idx == e)
        o, oe = expert(x[t], vals[0][e], vals[1][e], vals[2][e])
        w = gates[t, j].astype(np.float64)[:, None]
        np.add.at(y, t, w * o)
        np.add.at(err, t, w * oe)
        np.add.at(mag, t, np.abs(w * o) + w * oe)
    if svals is not None:
        o, oe = expert(x, *svals)
        y, err, mag = y + o, err + oe, mag + np.abs(o) + oe
    err = err + 1.01 * (k + 2) * 2.0 ** -24 * mag
    return y, err + 2.0 ** -8 * (np.abs(y) + err) + 1e-37


SHAPES = {"tiny": (TINY.with_(top_p=0.6), 32),
          "tiny token": (TINY.with_(mode=ROUTE_TOKEN), 64),
          "shared": (TINY.with_(d_ff_shared=128, block_size=24, n_blocks=3), 64),
          "shared, larger": (TINY.with_(d_ff_shared=256, block_size=24, n_blocks=3), 64),
          "one token": (TINY.with_(d_ff_shared=128, block_size=1, n_blocks=1, mode=ROUTE_TOKEN), 32),
          "block of 32": (LAYER.with_(n_experts=32), 128),
          "token routing": (LAYER.with_(n_experts=32, mode=ROUTE_TOKEN), 64)}


@pytest.mark.parametrize("name", list(SHAPES))
def test_layer_in_4_bits(name):
    from paper_2605_30876_gb300.layer import MoELayerQ4
    shape, group = SHAPES[name]
    dev = layer_inputs(shape, seed=3, device="cuda:0")
    host = {n: None if v is None else f64(v) for n, v in dev.items()}
    layer = MoELayerQ4.from_shape(shape, dev, group=group)
    y = layer.forward(dev["x"])
    m = P.dm()
    assert m.dmoe_get_device_error(layer.ws)[0] == 0 and m.dmoe_q4_device_error()[0] == 0
    idx, gates = layer.topk_idx.cpu().numpy(), layer.topk_gate.cpu().numpy()
    from paper_2605_30876_gb300.layer import MoELayer
    full = MoELayer.from_shape(shape, dev)
    full.forward(dev["x"])
    assert torch.equal(full.topk_idx, layer.topk_idx) and torch.equal(full.topk_gate, layer.topk_gate)
    vals = [O.q4_values(host[n], group)[2] for n in ("w_gate", "w_up", "w_down")]
    svals = None
    if shape.d_ff_shared:
        svals = [O.q4_values(host[n], group)[2] for n in ("ws_gate", "ws_up", "ws_down")]
    want, tol = layer_bounds(shape, host, vals, svals, idx, gates)
    assert (np.abs(f64(y) - want) <= tol).all()
    # captured, replayed on other tokens
    graph = torch.cuda.CUDAGraph()
    x = dev["x"].clone()
    out = torch.empty_like(y)
    with torch.cuda.graph(graph):
        layer.forward(x, out)
    x.copy_(dev["x"].flip(0))
    graph.replay()
    torch.cuda.synchronize()
    again = layer.forward(dev["x"].flip(0).contiguous())
    assert torch.equal(out, again)


def test_two_layers_on_two_streams():
    """Two layers at once, each with its own buffers: what each gives alone."""
    from paper_2605_30876_gb300.layer import MoELayerQ4
    shape = TINY.with_(top_p=0.6, block_size=16, n_blocks=4)
    layers = []
    for seed in (0, 1):
        dev = layer_inputs(shape, seed=seed, device="cuda:0")
        layers.append((MoELayerQ4.from_shape(shape, dev), dev["x"]))
    alone = [l.forward(x).clone() for l, x in layers]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(20):
        for (l, x), s in zip(layers, streams):
            l.y.zero_()
        torch.cuda.synchronize()
        for (l, x), s in zip(layers, streams):
            l.forward(x, stream=s)
        torch.cuda.synchronize()
        for (l, _), want in zip(layers, alone):
            assert torch.equal(l.y, want)
