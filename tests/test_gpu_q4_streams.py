"""Weights that are quantised on a stream of their own: nothing of it waits for, or runs ahead of, what
torch does on the current stream."""
import pytest
import torch

from tests import parity as P
from tests.test_gpu_q4 import make_w

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("more", [False, True])
def test_weights_that_are_not_contiguous_on_another_stream(handle, more):
    """Such weights are copied before they are quantised. The current stream is busy for a while: a copy on
    it would come too late."""
    from paper_2605_30876_gb300.layer import Q4Weight
    m = P.dm()
    w, one = make_w(3, 96, 256), make_w(1, 96, 256, seed=7)[0]
    want = Q4Weight(w, 64, one if more else None)
    wt, ot = w.transpose(1, 2).contiguous().transpose(1, 2), one.t().contiguous().t()
    assert not wt.is_contiguous() and torch.equal(wt, w)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(1 << 28)
    got = Q4Weight(wt, 64, ot if more else None, stream=s.cuda_stream if handle else s)
    out = torch.empty((got.desc.n_experts, 96, 256), dtype=torch.bfloat16, device="cuda")
    m.dmoe_q4_dequantize(got.desc, got.codes, got.scales, out, stream=s)
    s.synchronize()
    values = torch.empty_like(out)
    m.dmoe_q4_dequantize(want.desc, want.codes, want.scales, values)
    torch.cuda.synchronize()
    assert torch.equal(out, values)
