"""The experts' feed-forward block and its gradients against the formulas in 64 bits."""
import pytest
import torch

import paper_2605_30876_gb300 as dm
from tests import ffn_oracle as O

pytestmark = pytest.mark.gpu

# (experts, d, I, rows of every expert, rows behind the last): one row, ends around the 16 of an MMA,
# the 32 and 64 of a step and the 256 of a unit, experts without rows, widths that are no whole tiles
SHAPES = [
    (1, 64, 64, [1], 0),
    (1, 8, 8, [3], 0),
    (3, 72, 40, [1, 0, 2], 1),
    (4, 256, 128, [15, 16, 17, 33], 0),
    (5, 1000, 344, [0, 64, 65, 127, 0], 9),
    (2, 128, 520, [255, 257], 3),
    (3, 264, 136, [300, 1, 513], 70),
    (1, 512, 256, [777], 0),
    (9, 136, 200, [0, 0, 31, 32, 0, 1, 0, 48, 0], 5),
]
DTYPES = [torch.bfloat16, torch.float16]


def case(dtype, E, d, I, counts, rest, seed=0, stride=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def new(*shape, size=1.0):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0, size, generator=gen)
    R = sum(counts) + rest
    rows = lambda: new(R, d + stride)[:, :d]
    offsets = torch.tensor([0, *torch.tensor(counts).cumsum(0).tolist()], dtype=torch.int32, device="cuda")
    return dict(x=rows(), dy=rows(), offsets=offsets, w_gate=new(E, I, d, size=d ** -0.5),
                w_up=new(E, I, d, size=d ** -0.5), w_down=new(E, d, I, size=I ** -0.5))


def weights(c):
    return c["w_gate"], c["w_up"], c["w_down"]


def filled(shape, dtype, v=7.0):
    return torch.full(shape, v, dtype=dtype, device="cuda")


def run_forward(c, ids=None, zero_rest=False, pre=True, stride=0, stream=None):
    R, d = c["x"].shape
    I, dt = c["w_gate"].shape[1], c["x"].dtype
    pre = filled((R, 2, I), dt) if pre else None
    h, y = filled((R, I), dt), filled((R, d + stride), dt)[:, :d]
    dm.dmoe_expert_ffn(c["x"], c["offsets"], *weights(c), h, y, pre=pre, expert_ids=ids,
                       zero_rest=zero_rest, stream=stream)
    return pre, h, y


def check_forward(c, got, ids=None, zero_rest=False):
    pre, h, y = got
    want = O.forward(c["x"], c["offsets"].tolist(), *weights(c), ids)
    out = torch.isnan(want["y"][0][:, 0])
    if pre is not None:
        O.check("g", pre[:, 0], want["g"])
        O.check("u", pre[:, 1], want["u"])
        assert (pre[out] == 7).all()
    O.check("h", h, want["h"])
    O.check("y", y, want["y"])
    assert (h[out] == 7).all() and (y[out] == (0 if zero_rest else 7)).all()
    assert dm.dmoe_expert_device_error()[0] == 0


def run_backward(c, pre, h, zero_rest=False, stride=0, skip=()):
    R, d = c["x"].shape
    E, I, dt = c["w_gate"].shape[0], c["w_gate"].shape[1], c["x"].dtype
    out = dict(dpre=filled((R, 2, I), dt), dx=filled((R, d + stride), dt)[:, :d],
               dw_gate=filled((E, I, d), dt), dw_up=filled((E, I, d), dt), dw_down=filled((E, d, I), dt))
    out.update({n: None for n in skip})
    dm.dmoe_expert_ffn_backward(c["dy"], c["x"], c["offsets"], *weights(c), pre, h, *out.values(),
                                zero_rest=zero_rest)
    return out


def check_backward(c, pre, h, got, zero_rest=False):
    want = O.backward(c["dy"], c["x"], c["offsets"].tolist(), *weights(c), pre, h)
    out = torch.isnan(want["dx"][0][:, 0])
    if got["dpre"] is not None:
        O.check("dg", got["dpre"][:, 0], want["dg"])
        O.check("du", got["dpre"][:, 1], want["du"])
        assert (got["dpre"][out] == 7).all()
    for n in ("dx", "dw_gate", "dw_up", "dw_down"):
        if got[n] is not None:
            O.check(n, got[n], want[n])
    if got["dx"] is not None:
        assert (got["dx"][out] == (0 if zero_rest else 7)).all()
    assert dm.dmoe_expert_device_error()[0] == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(shape, dtype):
    c = case(dtype, *shape)
    check_forward(c, run_forward(c))
    check_forward(c, run_forward(c, pre=False, zero_rest=True, stride=24), zero_rest=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_backward(shape, dtype):
    c = case(dtype, *shape, seed=1)
    pre, h, _ = run_forward(c)
    check_backward(c, pre, h, run_backward(c, pre, h))
    check_backward(c, pre, h, run_backward(c, pre, h, zero_rest=True, stride=8), zero_rest=True)
