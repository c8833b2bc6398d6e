"""A workspace that calls with different shapes share. What has to be zero when a call begins (the
routing launch's ticket, at decode sizes the expert launch's counters and the published coresets)
lies at one place for every shape, where no call writes anything else: every call gives what it gives
on a workspace of its own."""
import itertools

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
