"""Gate and up products that fp16 cannot hold: the forward pass may well be finite (silu of a gate far below zero
is 0), and then the gradients are."""
import pytest
import torch

import paper_2605_30876_gb300 as dm
from paper_2605_30876_gb300.autograd import expert_ffn
from tests import ffn_oracle as O
from tests.test_gpu_expert_ffn import check_backward, run_backward, run_forward, weights

pytestmark = pytest.mark.gpu
MOST = torch.finfo(torch.float16).max
D, I = 64, 40


def case(counts, seed=0):
    """Feature 0 has gates of -102400 .. -89600, feature 1 the same above zero with up products near 0.05, feature
    2 gates near -216 with up products of 89600 .. 102400. x is 7 .. 8 throughout."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    E, R = len(counts), sum(counts)
    new = lambda *s, size: torch.empty(s, dtype=torch.float16, device="cuda").normal_(0, size, generator=gen)
    x = 7 + torch.rand((R, D), device="cuda", generator=gen)
    c = dict(x=x.to(torch.float16), dy=new(R, D, size=0.05),
             offsets=torch.tensor([0, *torch.tensor(counts).cumsum(0).tolist()], dtype=torch.int32, device="cuda"),
             w_gate=new(E, I, D, size=0.02), w_up=new(E, I, D, size=0.02), w_down=new(E, D, I, size=0.1))
    for i, gate, up in ((0, -200, 0.01), (1, 200, 1e-4), (2, -0.45, 200)):
        c["w_gate"][:, i], c["w_up"][:, i] = gate, up
    c["w_down"][:, :, 1] = new(E, D, size=1e-3)
    c["dy"][::7] = 0        # (rows whose loss is masked)
    return c


# few rows, and rows for the tensor cores' form (over 512)
@pytest.mark.parametrize("counts", [[5, 8], [40, 33], [300, 277]], ids=str)
def test_products_beyond_fp16(counts):
    c = case(counts)
    pre, h, y = run_forward(c)
    want = O.forward(c["x"], c["offsets"].tolist(), *weights(c))
    assert (want["g"][0][:, 0] < -MOST).all() and (want["g"][0][:, 1] > MOST).all() and (want["u"][0][:, 2] > MOST).all()
    O.check("h", h, want["h"])
    O.check("y", y, want["y"])
    assert (pre[:, 0, 0] == -MOST).all() and (pre[:, 0, 1] == MOST).all() and (pre[:, 1, 2] == MOST).all()
    got = run_backward(c, pre, h)
    assert all(torch.isfinite(t).all() for t in got.values())
    check_backward(c, pre, h, got)
    # what the unrounded products give: nothing through silu(g) = 0; dg = dh u where silu(g) = g
    dpre = got["dpre"].double()
    assert (dpre[:, :, 0] == 0).all() and (dpre[:, :, 2] == 0).all()
    dh = torch.cat([c["dy"][a:b].double() @ c["w_down"][e].double() for e, (a, b) in
                    enumerate(O.groups(c["offsets"].tolist(), len(y)))])[:, 1]
    dg = dh * want["u"][0][:, 1]
    # (dh's sum of 64 products, u's rounding to fp16 and dg's, a subnormal step of each)
    assert ((dpre[:, 0, 1] - dg).abs() <= 2 * 2.0 ** -11 * dg.abs() + 1e-6).all()
    assert (dpre[::7] == 0).all() and (got["dx"][::7] == 0).all()


def test_products_beyond_fp16_through_autograd():
    c = case([300, 277], seed=1)
    leaves = [c[n].clone().requires_grad_() for n in ("x", "w_gate", "w_up", "w_down")]
    y = expert_ffn(leaves[0], c["offsets"], *leaves[1:])
    assert torch.isfinite(y).all()
    for g in torch.autograd.grad(y, leaves, c["dy"]):
        assert torch.isfinite(g).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("counts", [[5, 8], [300, 277]], ids=str)
def test_what_is_no_number_stays_none(counts, bad):
    c = case(counts, seed=2)
    c["x"][3] = bad
    pre, h, y = run_forward(c)
    assert torch.isnan(h[3]).any() and torch.isnan(y[3]).all()
    if bad != bad:
        assert torch.isnan(pre[3]).all()
    got = run_backward(c, pre, h)
    assert torch.isnan(got["dw_down"][0]).any()
    keep = torch.ones(len(y), dtype=torch.bool, device="cuda")
    keep[3] = False
    assert torch.isfinite(got["dx"][keep]).all() and torch.isfinite(got["dw_down"][1]).all()
    assert dm.dmoe_expert_device_error()[0] == 0
