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
    # the same ends in calls of more rows
    (4, 72, 40, [1, 0, 2, 700], 1),
    (6, 256, 128, [15, 16, 17, 33, 600, 0], 0),
    (7, 1000, 344, [0, 64, 65, 127, 0, 31, 300], 9),
    # whole tiles, and widths a little off 64, 128 and 256
    (2, 256, 384, [257, 300], 0),
    (2, 248, 136, [300, 290], 0),
    (2, 120, 504, [520, 10], 2),
    (1, 192, 320, [600], 0),
    # few rows: groups of up to eight and of more together, long sums, and either side of the sizes
    # at which the kernels change
    (8, 256, 264, [8, 9, 1, 33, 0, 64, 7, 32], 2),
    (2, 4096, 2048, [5, 3], 0),
    (2, 4096, 2048, [5, 4], 0),
    (1, 8192, 64, [8], 0),
    (12, 520, 136, [40] * 12, 32),
    (12, 520, 136, [40] * 12, 33),
    (3, 1024, 1024, [100, 4, 24], 0),
    (3, 1024, 1024, [100, 4, 25], 0),
    (40, 136, 1040, [3, 0, 1, 5] * 10, 0),
    # few units with long sums (several pairs share one): over the width, and over the rows, where some
    # have none
    (1, 1096, 1544, [100], 3),
    (1, 4096, 64, [300], 0),
    (1, 72, 4104, [290], 1),
    (1, 264, 136, [2500], 5),
    (3, 136, 72, [4000, 0, 50], 0),
    (2, 136, 520, [3001, 3], 7),
    (1, 8, 8, [3000], 0),
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


def test_expert_ids():
    """Groups in any order, an expert in two groups, ids that are no expert's."""
    c = case(torch.bfloat16, 6, 136, 72, [20, 5, 0, 40, 33, 2], 4)
    ids = torch.tensor([5, 0, 3, 5, -1, 6], dtype=torch.int32, device="cuda")
    check_forward(c, run_forward(c, ids), ids)
    check_forward(c, run_forward(c, ids, zero_rest=True), ids, zero_rest=True)
    # more groups than experts
    few = dict(c, w_gate=c["w_gate"][:2].contiguous(), w_up=c["w_up"][:2].contiguous(),
               w_down=c["w_down"][:2].contiguous())
    ids = torch.tensor([1, 0, 0, 1, 0, 1], dtype=torch.int32, device="cuda")
    check_forward(few, run_forward(few, ids), ids)


@pytest.mark.parametrize("rows", [1, 2])
def test_as_many_groups_as_there_can_be(rows):
    """512 groups of the same few experts; the call's rows are few and more than that."""
    c = case(torch.bfloat16, 3, 72, 40, [0, 0, 0], 512 * rows)
    c["offsets"] = torch.arange(513, dtype=torch.int32, device="cuda") * rows
    ids = (torch.arange(512, device="cuda") * 7 % 4).to(torch.int32)     # (3 is no expert)
    check_forward(c, run_forward(c, ids, zero_rest=True), ids, zero_rest=True)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("counts", [[5, 3, 0], [40, 9, 30]], ids=str)
def test_few_rows_keep_to_themselves(counts, bad):
    """A row's values are its own: other rows of its group, and rows of no group, may hold anything."""
    c = case(torch.bfloat16, 3, 264, 136, counts, 2)
    want = run_forward(c)
    c["x"][1] = bad
    c["x"][-2:] = bad
    got = run_forward(c)
    keep = torch.ones(sum(counts) + 2, dtype=torch.bool, device="cuda")
    keep[1] = False
    assert all(torch.equal(a[keep], b[keep]) for a, b in zip(got, want))


def test_one_expert_of_all_rows():
    c = case(torch.float16, 1, 200, 104, [71], 0)
    want = run_forward(c)
    dense = dict(c, offsets=None)
    for a, b in zip(run_forward(dense), want):
        assert torch.equal(a, b)
    got, same = run_backward(dense, *want[:2]), run_backward(c, *want[:2])
    assert all(torch.equal(got[n], same[n]) for n in got)


@pytest.mark.parametrize("offsets", [[-7, 10, 30, 99], [0, 30, 10, 50], [50, 50, 60, 7], [3, 3, 20, 41]])
def test_offsets_that_are_cut(offsets):
    c = case(torch.bfloat16, 3, 72, 72, [10, 20, 20], 0)
    c["offsets"] = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    got = run_forward(c)
    if offsets != [0, 30, 10, 50]:         # (two groups share rows there: either's values)
        check_forward(c, got)
        check_backward(c, *got[:2], run_backward(c, *got[:2]))
    else:
        run_backward(c, *got[:2])
        assert dm.dmoe_expert_device_error()[0] == 0


def test_groups_that_overlap_in_calls_of_few_units():
    """More units than rows that are apart would make, where several pairs of CTAs share a unit's sum."""
    c = case(torch.bfloat16, 3, 2048, 264, [600, 0, 0], 0)
    c["offsets"] = torch.tensor([0, 600, 10, 600], dtype=torch.int32, device="cuda")
    pre, h, y = run_forward(c)
    got = run_backward(c, pre, h)
    assert dm.dmoe_expert_device_error()[0] == 0
    want = O.forward(c["x"][:10], [0, 10, 10, 10], *weights(c))       # (rows that one group has alone)
    O.check("h", h[:10], want["h"])
    O.check("y", y[:10], want["y"])
    assert all(torch.isfinite(t).all() for t in (h, y, got["dx"], got["dw_gate"], got["dw_down"]))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_other_experts_rows_and_weights_stay_out(bad):
    """Rows of other groups, rows of none and other experts' weights do not reach a group's results."""
    c = case(torch.bfloat16, 3, 136, 72, [21, 35, 70], 10)
    pre, h, y = run_forward(c)
    want = run_backward(c, pre, h)
    for where in ("rows", "weights"):
        b = {k: v.clone() for k, v in c.items()}
        if where == "rows":
            b["x"][21:56] = bad
            b["dy"][21:56] = bad
            b["x"][126:] = bad
            b["dy"][126:] = bad
        else:
            for n in ("w_gate", "w_up", "w_down"):
                b[n][1] = bad
        pre2, h2, y2 = run_forward(b)
        keep = torch.ones(136, dtype=torch.bool, device="cuda")
        keep[21:56] = False
        for a, z in ((pre, pre2), (h, h2), (y, y2)):
            assert torch.equal(a[keep], z[keep])
        got = run_backward(b, pre2, h2)
        assert torch.equal(got["dx"][keep], want["dx"][keep])
        for n in ("dw_gate", "dw_up", "dw_down"):
            assert torch.equal(got[n][[0, 2]], want[n][[0, 2]])


@pytest.mark.parametrize("skip", [("dx",), ("dw_gate", "dw_up"), ("dw_down",), ("dx", "dw_gate", "dw_up", "dpre"),
                                  ("dw_gate", "dw_up", "dw_down")])
def test_some_of_the_gradients(skip):
    c = case(torch.bfloat16, 2, 72, 136, [40, 13], 0)
    pre, h, _ = run_forward(c)
    whole, got = run_backward(c, pre, h), run_backward(c, pre, h, skip=skip)
    assert all(got[n] is None or torch.equal(got[n], whole[n]) for n in got)


def test_no_rows():
    c = case(torch.bfloat16, 2, 72, 136, [0, 0], 0)
    pre, h, y = run_forward(c)
    got = run_backward(c, pre, h)
    assert y.shape == (0, 72) and all((got[n] == 0).all() for n in ("dw_gate", "dw_up", "dw_down"))
    c = case(torch.bfloat16, 2, 72, 136, [0, 0], 5)            # rows, but none of an expert
    pre, h, y = run_forward(c, zero_rest=True)
    got = run_backward(c, pre, h, zero_rest=True)
    assert (y == 0).all() and (h == 7).all() and all((v == 0).all() for n, v in got.items() if n != "dpre")


def test_rows_and_offsets_beyond_32_bits():
    """Elements of h, pre and x further than 2^31 from their bases."""
    d, I, R = 1096, 520, 2100000
    gen = torch.Generator(device="cuda").manual_seed(5)
    new = lambda *s, size=1.0: torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(0, size, generator=gen)
    x, w = new(R, d), (new(2, I, d, size=0.03), new(2, I, d, size=0.03), new(2, d, I, size=0.04))
    offsets = torch.tensor([0, R - 300, R], dtype=torch.int32, device="cuda")
    pre, h, y = (torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in ((R, 2, I), (R, I), (R, d)))
    dm.dmoe_expert_ffn(x, offsets, *w, h, y, pre=pre)
    last = slice(R - 300, R)
    c = dict(x=x[last], offsets=torch.tensor([0, 0, 300], dtype=torch.int32, device="cuda"), w_gate=w[0],
             w_up=w[1], w_down=w[2], dy=x[:300])
    check_forward(c, (pre[last], h[last], y[last]))
    dpre, dx = torch.empty_like(pre), torch.empty_like(x)
    dw = [torch.empty_like(t) for t in w]
    dy = y
    dy[last] = x[:300]
    dm.dmoe_expert_ffn_backward(dy, x, offsets, *w, pre, h, dpre, dx, *dw)
    want = O.backward(dy[last], x[last], [0, 0, 300], *w, pre[last], h[last])
    O.check("dx", dx[last], want["dx"])
    O.check("dg", dpre[last, 0], want["dg"])
    for n, v in zip(("dw_gate", "dw_up", "dw_down"), dw):
        O.check(n, v[1], (want[n][0][1], want[n][1][1]))


def test_same_call_same_bits_on_any_stream():
    c = case(torch.bfloat16, 5, 264, 136, [33, 0, 260, 7, 100], 3)
    want = run_forward(c)
    grads = run_backward(c, *want[:2])
    torch.cuda.synchronize()
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        a = run_forward(c)
    with torch.cuda.stream(other):
        b = run_forward(c)
        more = run_backward(c, *want[:2])
    torch.cuda.synchronize()
    d = run_forward(c, stream=side)
    torch.cuda.synchronize()
    for got in (a, b, d):
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert all(torch.equal(more[n], grads[n]) for n in grads)


def test_captured_and_replayed():
    c = case(torch.float16, 3, 264, 136, [33, 70, 7], 3)
    R, d, I = 113, 264, 136
    new = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda")
    pre, h, y, dpre, dx = new(R, 2, I), new(R, I), new(R, d), new(R, 2, I), new(R, d)
    dw = [torch.zeros_like(t) for t in weights(c)]

    def both():
        dm.dmoe_expert_ffn(c["x"], c["offsets"], *weights(c), h, y, pre=pre, zero_rest=True)
        dm.dmoe_expert_ffn_backward(c["dy"], c["x"], c["offsets"], *weights(c), pre, h, dpre, dx, *dw,
                                    zero_rest=True)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    c["x"].mul_(-0.5)
    c["offsets"].copy_(torch.tensor([0, 50, 50, 110], dtype=torch.int32))
    both()
    want = [t.clone() for t in (pre[:110], h[:110], y, dpre[:110], dx, *dw)]
    for t in (pre, h, y, dpre, dx, *dw):
        t.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((pre[:110], h[:110], y, dpre[:110], dx, *dw), want))


# (the form for few rows has no waits; in the second shape several pairs of CTAs share a sum)
@pytest.mark.parametrize("shape", [(2, 264, 136, [433, 270], 0), (1, 2048, 264, [600], 0)], ids=str)
def test_waits_that_run_out_are_recorded(shape):
    c = case(torch.bfloat16, *shape)
    pre, h, y = run_forward(c)
    torch.cuda.synchronize()
    dm.dmoe_expert_set_debug_hold(1)
    run_forward(c)
    status, (code, where, _) = dm.dmoe_expert_device_error()
    assert status == 6 and code == 1 and where == 10
    assert dm.dmoe_expert_device_error()[0] == 0      # read and cleared, and the hold with it
    check_forward(c, run_forward(c))
    check_backward(c, pre, h, run_backward(c, pre, h))
