"""The workspace of the norms' gradients: what a call needs is what it uses."""
import pytest
import torch

import paper_2605_30876_gb300 as dm
from paper_2605_30876_gb300.autograd import norm_residual
from tests.test_gpu_norm import inputs, run

pytestmark = pytest.mark.gpu


def grads(c, d_out, G, ws, dgate=True):
    r, n, stats = torch.empty_like(c["x"]), torch.empty_like(c["x"]), torch.empty((2, len(c["x"])), device="cuda")
    dm.dmoe_norm_residual(*c.values(), r, n, stats=stats, gate_tokens=G)
    out = {"dx": torch.empty_like(r), "dy": torch.empty_like(r),
           "dgate": torch.empty_like(c["gate"]) if dgate else None,
           "dw_post": torch.empty_like(c["w_post"]), "dw_pre": torch.empty_like(c["w_pre"])}
    dm.dmoe_norm_residual_backward(*c.values(), stats, *d_out, *out.values(), gate_tokens=G, workspace=ws)
    return out


def same(a, b):
    return all(v is None or torch.equal(v, b[k]) for k, v in a.items())


@pytest.mark.parametrize("T,d", [(700, 264), (30, 2048)])
def test_a_gate_row_for_each_token(T, d):
    """Without gate_tokens a gate has a row for each token, and so it has with the workspace's sizes."""
    c, d_out = inputs(torch.bfloat16, T, d, 1)
    ws = dm.alloc_norm_workspace(T, d)
    assert same(grads(c, d_out, 0, ws), run(c, d_out, 1))
    x, gate = c["x"].clone().requires_grad_(), c["gate"].clone().requires_grad_()
    w = c["w_pre"].clone().requires_grad_()
    a = torch.autograd.grad(norm_residual(x, c["y"], None, gate, w, gate_tokens=0), [x, gate, w], d_out)
    b = torch.autograd.grad(norm_residual(x, c["y"], None, gate, w), [x, gate, w], d_out)
    assert all(torch.equal(u, v) for u, v in zip(a, b))


@pytest.mark.parametrize("T,d,G", [(700, 264, 7), (3000, 2048, 48), (900, 5120, 9)])
def test_a_gate_whose_gradient_is_not_wanted(T, d, G):
    c, d_out = inputs(torch.bfloat16, T, d, G)
    guard = torch.zeros(dm.dmoe_norm_workspace_size(T, d) + 4096, dtype=torch.uint8, device="cuda")
    got = grads(c, d_out, G, guard[:-4096], dgate=False)
    assert same(got, run(c, d_out, G)) and (guard[-4096:] == 0).all()
