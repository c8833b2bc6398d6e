"""A workspace that calls with different shapes share. What has to be zero when a call begins (the
routing launch's ticket, at decode sizes the expert launch's counters and the published coresets)
lies at one place for every shape, where no call writes anything else: every call gives what it gives
on a workspace of its own."""
import itertools

import numpy as np
import pytest
import torch

from dmoe_synth import LAYER, ROUTE_TOKEN, TINY, layer_inputs
from tests import parity as P

pytestmark = pytest.mark.gpu
ZEROS = slice(256, 4352)

# decode sizes (counters and coresets of their own) and larger ones, whose scores and rows would lie there
SHAPES = {
    "tiny": TINY.with_(d_ff_shared=128), "tiny p": TINY.with_(top_p=0.6, block_size=32),
    "blocks of one": TINY.with_(block_size=1, n_blocks=64, top_k=3), "tiny token": TINY.with_(mode=ROUTE_TOKEN),
    "layer": LAYER.with_(n_experts=32), "layer p": LAYER.with_(n_experts=32, top_p=0.6),
    "many tokens": TINY.with_(block_size=32, n_blocks=5, top_k=4, d_ff_shared=128),
    "many, token": TINY.with_(block_size=32, n_blocks=9, mode=ROUTE_TOKEN, n_experts=32),
}


def layers(names, workspace=None):
    from paper_2605_30876_gb300.layer import MoELayer
    out = []
    for n in names:
        dev = layer_inputs(SHAPES[n], seed=3, device="cuda")
        out.append((MoELayer.from_shape(SHAPES[n], dev, workspace=workspace), dev["x"]))
    return out


@pytest.mark.parametrize("names", [*itertools.combinations(SHAPES, 2), tuple(SHAPES)])
def test_layers_on_one_workspace(names):
    m = P.dm()
    want = [(l.forward(x).clone(), l.topk_idx.clone()) for l, x in layers(names)]
    size = max(m.dmoe_workspace_size(P.desc_of(SHAPES[n])) for n in names)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    m.dmoe_workspace_init(ws)
    shared = layers(names, ws)
    for _ in range(2):
        for (l, x), (y, idx) in zip(shared, want):
            l.topk_idx.fill_(-7)
            l.y.fill_(5.0)
            assert torch.equal(l.forward(x), y) and torch.equal(l.topk_idx, idx)
            assert not ws[ZEROS].any()
    assert m.dmoe_get_device_error(ws)[0] == 0


# ------------------------------------------------------------------------------ sorts

# pairs: one launch; the first that take two; 148 chunks; chunks of two tiles of a thread's pairs and of many
SORTS = [(128, 8, 256), (1025, 1, 256), (4097, 3, 33), (18944, 8, 256), (18945, 8, 256), (152000, 8, 130)]


def sort(T, k, E, ws, seed=0):
    """A sort on the workspace, held to the order of numpy's stable sort."""
    m = P.dm()
    idx = np.random.default_rng(seed).integers(-1, E, (T, k)).astype(np.int32)
    offsets, rows, pos = (torch.full((n,), 77, dtype=torch.int32, device="cuda") for n in (E + 1, T * k, T * k))
    if isinstance(ws, tuple):
        dev = torch.from_numpy(idx).cuda()
        assert m._lib.dmoe_sort_tokens(T, k, E, dev.data_ptr(), offsets.data_ptr(), rows.data_ptr(),
                                       pos.data_ptr(), *ws, torch.cuda.current_stream().cuda_stream) == 0
    else:
        m.dmoe_sort_tokens(torch.from_numpy(idx).cuda(), E, offsets, rows, pos, workspace=ws)
    key = np.where(idx < 0, E, idx).reshape(-1)
    order = np.argsort(key, kind="stable")
    want = np.empty_like(order)
    want[order] = np.arange(order.size)
    assert np.array_equal(pos.cpu().numpy(), np.where(key == E, ~want, want))
    assert np.array_equal(rows.cpu().numpy(), np.where(key[order] == E, -1, order))
    assert np.array_equal(offsets.cpu().numpy(), np.searchsorted(key[order], np.arange(E + 1)))


@pytest.mark.parametrize("T,k,E", SORTS)
@pytest.mark.parametrize("name", list(SHAPES))
def test_forwards_between_sorts(name, T, k, E):
    m = P.dm()
    (own, x), = layers([name])
    want, routed = own.forward(x).clone(), P.gpu_router(SHAPES[name], layer_inputs(SHAPES[name], seed=3, device="cuda"))
    size = max(m.dmoe_workspace_size(own.desc), m.dmoe_sort_workspace_size(T, k, E))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    m.dmoe_workspace_init(ws)
    (layer, x), = layers([name], ws)
    for seed in range(2):
        sort(T, k, E, ws, seed)
        assert not ws[ZEROS].any()
        layer.topk_idx.fill_(-7)
        layer.y.fill_(5.0)
        assert torch.equal(layer.forward(x), want)
        assert torch.equal(layer.topk_idx, own.topk_idx) and torch.equal(layer.n_unique, own.n_unique)
        sort(T, k, E, ws, seed)
        got = P.gpu_router(SHAPES[name], layer_inputs(SHAPES[name], seed=3, device="cuda"), ws=ws)
        assert all((got[key] == v).all() for key, v in routed.items())
    assert m.dmoe_get_device_error(ws)[0] == 0


def test_routing_between_sorts_on_the_static_scratch():
    m, shape = P.dm(), TINY
    dev = layer_inputs(shape, seed=4, device="cuda", with_weights=False)
    want = P.gpu_router(shape, dev)
    scratch = m.dmoe_no_alloc_scratch()
    for seed in range(2):
        sort(18944, 8, 256, scratch, seed)
        got = torch.full((shape.T, shape.top_k), -7, dtype=torch.int32, device="cuda")
        gate = torch.empty((shape.T, shape.top_k), device="cuda")
        m.dmoe_router_no_alloc(P.desc_of(shape), dev["x"], dev["w_r"], dev["bias"], got, gate)
        assert m.dmoe_router_no_alloc_device_error()[0] == 0
        assert np.array_equal(got.cpu().numpy(), want["idx"])


@pytest.mark.parametrize("most", [0, 1])
def test_sorts_of_chunks_around_16_bits(most):
    """The largest chunks with counts of 16 bits, all pairs of one expert among them, and the next ones."""
    m = P.dm()
    R, E = 148 * 60 * 1024 + most, 3
    idx = torch.full((R, 1), 2, dtype=torch.int32, device="cuda")
    idx[-5] = 0
    idx[R // 2] = -1
    offsets, rows, pos = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (E + 1, R, R))
    m.dmoe_sort_tokens(idx, E, offsets, rows, pos, workspace=m.alloc_sort_workspace(R, 1, E))
    assert offsets.tolist() == [0, 1, 1, R - 1]
    at = torch.arange(R, dtype=torch.int32, device="cuda")
    want = torch.cat([at[-5:-4], at[:R // 2], at[R // 2 + 1:-5], at[-4:], at[:1] - 1])
    assert torch.equal(rows, want)
    assert int(pos[R // 2]) == -R and torch.equal(pos[rows[:-1].long()], at[:-1])


def test_smaller_sorts_on_the_largest_ones_workspace():
    ws = P.dm().alloc_sort_workspace(65536, 8, 256)
    for T, k, E in [(65536, 8, 256), (18944, 8, 256), (18945, 8, 256), (300, 5, 7), (2000, 16, 256), (1, 1, 1)]:
        sort(T, k, E, ws)
