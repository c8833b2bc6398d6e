"""The norms' gradients where a group's run of tokens holds several gate rows and begins and ends inside one: against
the formulas in 64 bits. And the forward pass in place where a run is longer than the rows on their way."""
import pytest
import torch

import paper_2605_30876_gb300 as dm
from tests.test_gpu_norm import compare, inputs, run

pytestmark = pytest.mark.gpu

# (tokens, width, tokens of a gate row, groups of the backward launch: one for each of 152 SMs where rows are wider than
# 2048 elements, two where wider than 1280, and several for each of two CTAs below): runs of T / groups tokens
RUNS = [(4001, 2048, 5, 304), (3300, 4096, 7, 152), (2001, 8192, 5, 152), (1501, 10001, 4, 152), (1501, 16384, 3, 152),
        (4001, 2050, 8, 152), (3301, 2049, 4, 152), (6000, 1536, 7, 304), (60001, 64, 3, 9728), (9001, 512, 3, 1216)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", RUNS, ids=str)
def test_runs_over_several_gate_rows(shape, dtype):
    T, d, G, groups = shape
    a_run = -(-T // groups)
    assert a_run > G and a_run % G and T % G
    c, d_out = inputs(dtype, T, d, G, seed=5)
    compare(c, d_out, G, run(c, d_out, G))


@pytest.mark.parametrize("d,T", [(64, 23000), (2048, 3625), (4096, 3312)])
def test_runs_in_sums_of_their_own(d, T):
    """The sizes at which some of the gradients are compared with all of them, and those with the formulas."""
    c, d_out = inputs(torch.bfloat16, T, d, 16)
    compare(c, d_out, 16, run(c, d_out, 16))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", [(4001, 2048), (3001, 2049), (2500, 8192), (1300, 12000), (30011, 72)])
def test_in_place_over_long_runs(T, d, dtype):
    c, _ = inputs(dtype, T, d, 7, seed=6)
    r, n = torch.empty_like(c["x"]), torch.empty_like(c["x"])
    dm.dmoe_norm_residual(*c.values(), r, n, gate_tokens=7)
    dm.dmoe_norm_residual(*c.values(), c["x"], c["y"], gate_tokens=7)
    assert torch.equal(r, c["x"]) and torch.equal(n, c["y"])
