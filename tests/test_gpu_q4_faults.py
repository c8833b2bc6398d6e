"""The 4-bit products' bounded waits that run out, without a GPU fault. With dmoe_q4_set_debug_hold a stage
waits for an arrival that never comes: the issuing warps wait for it to fill, the dequantising and the
loading ones for a slot that does not empty, the epilogue for sums that do not come. Each gives up
after 1 s; the launch records the timeout, gives its tensor memory back and ends, and the next product
is right."""
import time

import pytest
import torch

from tests import parity as P
from tests.test_gpu_q4 import make_w, pack

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16

# stages: fewer than the ring's slots, more, a pair's halves; units: one, of two issuing warps or one,
# several per CTA, of pairs that share none
CASES = {"two stages": (1, 64, 256, [5]), "many stages": (2, 200, 2048, [40, 3]), "96 rows": (1, 8192, 256, [256]),
         "one stage, many units": (40, 640, 128, [7] * 40), "shared": (1, 300, 8192, [20]),
         "pairs apart": (40, 640, 3200, [3] * 40)}


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_waits_that_run_out(name, gated):
    m = P.dm()
    E, N, K, sizes = CASES[name]
    desc, R = m.make_q4_desc(E, N, K, 64), sum(sizes)
    packed = [t for i in range(2 if gated else 1) for t in pack(desc, make_w(E, N, K, i))]
    offsets = torch.tensor([0, *sizes], dtype=torch.int32, device="cuda").cumsum(0).to(torch.int32)
    x = torch.randn((R, K), generator=torch.Generator().manual_seed(0)).to(BF16).cuda()
    call = m.dmoe_q4_swiglu if gated else m.dmoe_q4_linear
    want, y = torch.empty((R, N), dtype=BF16, device="cuda"), torch.empty((R, N), dtype=BF16, device="cuda")
    call(desc, x, offsets, *packed, want)
    assert m.dmoe_q4_device_error() == (0, (0, 0, 0))
    m.dmoe_q4_set_debug_hold(1)
    t0 = time.time()
    call(desc, x, offsets, *packed, y)
    st, info = m.dmoe_q4_device_error()
    elapsed = time.time() - t0
    assert st == 6 and info[:2] == (1, 9), (st, info)          # a wait that ran out, in these products
    assert 0.5 < elapsed < 60, elapsed
    assert m.dmoe_q4_device_error() == (0, (0, 0, 0))          # clear, and the hold with it
    y.zero_()
    call(desc, x, offsets, *packed, y)
    assert m.dmoe_q4_device_error()[0] == 0
    assert torch.equal(y, want)


def test_hold_is_taken_back():
    m = P.dm()
    with pytest.raises(m.DmoeError):
        m.dmoe_q4_set_debug_hold(-1)
    m.dmoe_q4_set_debug_hold(5)
    assert m.dmoe_q4_device_error()[0] == 0                    # no fault was read: the hold stays
    m.dmoe_q4_set_debug_hold(0)
    desc = m.make_q4_desc(1, 64, 128, 64)
    y = torch.empty((3, 64), dtype=BF16, device="cuda")
    m.dmoe_q4_linear(desc, torch.ones((3, 128), dtype=BF16, device="cuda"), None, *pack(desc, make_w(1, 64, 128)), y)
    assert m.dmoe_q4_device_error()[0] == 0
