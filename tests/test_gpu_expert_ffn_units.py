"""The feed-forward block where a pair of CTAs has many units, in the tensor cores' form of the forward pass (calls of
more than 512 rows), and in calls of which every element is known exactly."""
import pytest
import torch

import paper_2605_30876_gb300 as dm
from tests import ffn_oracle as O
from tests.test_gpu_expert_ffn import case, check_backward, check_forward, run_backward, run_forward, weights

pytestmark = pytest.mark.gpu
BAD = [float("nan"), float("inf")]
# ends inside tiles of every kind: groups of rows, widths off 128 and 256, rows of no group
MORE = ([210, 35, 400], 10)
E, D, I, R = 3, 136, 72, 655


def more(dtype=torch.bfloat16, seed=0):
    return case(dtype, E, D, I, *MORE, seed=seed)


def test_which_form_runs():
    """The sizes of this file take the form with waits, of which the debug hold makes the first run out; a few
    rows take the other."""
    for c, waits in ((more(), True), (case(torch.bfloat16, 1, D, I, [R], 0), True), (case(torch.bfloat16, E, D, I, [5, 8, 0], 0), False)):
        torch.cuda.synchronize()
        dm.dmoe_expert_set_debug_hold(1)
        run_forward(c)
        status = dm.dmoe_expert_device_error()[0]
        dm.dmoe_expert_set_debug_hold(0)
        assert (status == 6) == waits


def test_weights_gradients_behind_the_rows_gradient():
    """The weights' gradients read what the first of three launches wrote: over many units, with what the memory held
    before of no account, they are those of a call without the launch between."""
    c = case(torch.bfloat16, 40, 520, 264, [(37 * i) % 211 for i in range(40)], 5, seed=3)
    pre, h, _ = run_forward(c)
    want = run_backward(c, pre, h, skip=("dx",))
    got = run_backward(c, pre, h)
    args = (c["dy"], c["x"], c["offsets"], *weights(c), pre, h)
    for i in range(30):
        for t in got.values():
            t.fill_(float("nan"))
        dm.dmoe_expert_ffn_backward(*args, *got.values())
        for n in ("dw_gate", "dw_up", "dw_down"):
            assert torch.equal(got[n], want[n]), (i, n)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_many_units_of_mixed_widths(dtype):
    """Seven units and more for each pair in every product, of 32 to 256 columns and of none."""
    gen = torch.Generator().manual_seed(7)
    counts = torch.randint(0, 301, (192,), generator=gen)
    counts[::17] = 0
    c = case(dtype, 192, 520, 1096, counts.tolist(), 33, seed=4)
    got = run_forward(c)
    check_forward(c, got)
    check_forward(c, run_forward(c, pre=False, zero_rest=True, stride=24), zero_rest=True)
    check_backward(c, *got[:2], run_backward(c, *got[:2], zero_rest=True, stride=8), zero_rest=True)


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("where", ["group", "row", "weights"])
def test_others_stay_out(where, bad):
    c = more(seed=1)
    pre, h, y = run_forward(c, zero_rest=True)
    want = run_backward(c, pre, h, zero_rest=True)
    b = {k: v.clone() for k, v in c.items()}
    off = {"group": slice(210, 245), "row": slice(300, 301), "weights": slice(210, 245)}[where]
    if where == "weights":
        for n in ("w_gate", "w_up", "w_down"):
            b[n][1] = bad
    else:
        for n in ("x", "dy"):
            b[n][off] = bad
            b[n][645:] = bad
    keep = torch.ones(R, dtype=torch.bool, device="cuda")
    keep[off] = False
    got = run_forward(b, zero_rest=True)
    for v, w in zip(got, (pre, h, y)):
        assert torch.equal(v[keep], w[keep])
    back = run_backward(b, *got[:2], zero_rest=True)
    assert torch.equal(back["dx"][keep], want["dx"][keep])
    others = [0, 1] if where == "row" else [0, 2]
    for n in ("dw_gate", "dw_up", "dw_down"):
        assert torch.equal(back[n][others], want[n][others])


@pytest.mark.parametrize("offsets", [[-7, 300, 330, 999], [655, 655, 660, 7], [3, 3, 20, 641], [0, 0, 655, 655], [600, 20, 610, 640]])
def test_offsets_that_are_cut(offsets):
    c = more(seed=2)
    c["offsets"] = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    pre, h, y = run_forward(c, zero_rest=True)
    check_forward(c, (pre, h, y), zero_rest=True)
    check_backward(c, pre, h, run_backward(c, pre, h, zero_rest=True), zero_rest=True)


def test_groups_by_ids():
    c = more(seed=5)
    ids = torch.tensor([2, 7, 0], dtype=torch.int32, device="cuda")
    check_forward(c, run_forward(c, ids, zero_rest=True), ids, zero_rest=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_one_expert_of_all_rows(dtype):
    c = case(dtype, 1, D, I, [R], 0, seed=6)
    want = run_forward(c)
    check_forward(c, want)
    dense = dict(c, offsets=None)
    assert all(torch.equal(a, b) for a, b in zip(run_forward(dense), want))
    got, same = run_backward(dense, *want[:2]), run_backward(c, *want[:2])
    assert all(torch.equal(got[n], same[n]) for n in got)


def test_same_bits_on_any_stream():
    c = more(seed=7)
    want = run_forward(c)
    grads = run_backward(c, *want[:2])
    torch.cuda.synchronize()
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):                      # two calls at once
        with torch.cuda.stream(side):
            a, more_a = run_forward(c), run_backward(c, *want[:2])
        with torch.cuda.stream(other):
            b, more_b = run_forward(c), run_backward(c, *want[:2])
    torch.cuda.synchronize()
    d = run_forward(c, stream=side)
    torch.cuda.synchronize()
    for got in (a, b, d):
        assert all(torch.equal(v, w) for v, w in zip(got, want))
    for got in (more_a, more_b):
        assert all(torch.equal(got[n], grads[n]) for n in grads)


def test_captured_and_replayed():
    c = more(torch.float16, seed=8)
    new = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda")
    pre, h, y, dpre, dx = new(R, 2, I), new(R, I), new(R, D), new(R, 2, I), new(R, D)
    dw = [torch.zeros_like(t) for t in weights(c)]

    def both():
        dm.dmoe_expert_ffn(c["x"], c["offsets"], *weights(c), h, y, pre=pre, zero_rest=True)
        dm.dmoe_expert_ffn_backward(c["dy"], c["x"], c["offsets"], *weights(c), pre, h, dpre, dx, *dw, zero_rest=True)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for offsets in ([0, 300, 300, 640], [0, 1, 17, 655], [0, 0, 0, 0]):
        c["x"].mul_(-0.5)
        c["offsets"].copy_(torch.tensor(offsets, dtype=torch.int32))
        n = offsets[-1]
        both()
        want = [t.clone() for t in (pre[:n], h[:n], y, dpre[:n], dx, *dw)]
        for t in (pre, h, y, dpre, dx, *dw):
            t.fill_(3)
        for _ in range(2):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((pre[:n], h[:n], y, dpre[:n], dx, *dw), want))


def test_dx_in_the_place_of_what_is_not_read():
    """h is an input for dw_down alone: without it dx may take its memory."""
    c = case(torch.bfloat16, E, D, D, *MORE, seed=10)
    pre, h, _ = run_forward(c)
    want = run_backward(c, pre, h, skip=("dw_down",))
    got = dict(want, dx=h, **{n: torch.empty_like(want[n]) for n in ("dpre", "dw_gate", "dw_up")})
    args = (c["dy"], c["x"], c["offsets"], *weights(c), pre, h)
    dm.dmoe_expert_ffn_backward(*args, *got.values())
    assert torch.equal(h[:645], want["dx"][:645]) and torch.equal(got["dw_gate"], want["dw_gate"])
    with pytest.raises(dm.DmoeError):
        dm.dmoe_expert_ffn_backward(*args, *dict(got, dw_down=torch.empty_like(c["w_down"])).values())


def units(shape, gen):
    """-1, 0 and 1."""
    return torch.randint(-1, 2, shape, dtype=torch.int8, device="cuda", generator=gen).to(torch.bfloat16)


def one_each(E, n, m, gen, size):
    """[E, n, m] with one element of -size or size in every row, not in the first column."""
    w = torch.zeros((E, n, m), dtype=torch.bfloat16, device="cuda")
    at = torch.randint(1, m, (E, n, 1), device="cuda", generator=gen)
    sign = torch.randint(0, 2, (E, n, 1), device="cuda", generator=gen) * 2 - 1
    return w.scatter_(2, at, (sign * size).to(torch.bfloat16))


def products(x, w):
    """x w^T exactly: whole numbers below 2^24."""
    return x.float() @ w.float().t()


# rows whose offsets pass 2^31 elements; the widest experts, with one row, with a few and with more than one unit has; the
# most experts
EXACT = [(1096, 520, [0, 1200007, 1200020, 2099990], 10), (16384, 16384, [0, 1], 0), (16384, 16384, [0, 5, 5, 300], 1),
         (8, 16384, [0, 700], 3), (16384, 8, [0, 30, 1030], 0), (136, 72, [7 * i for i in range(513)], 9)]


@pytest.mark.parametrize("d,I,ends,rest", EXACT, ids=lambda v: str(v)[:24])
def test_every_element(d, I, ends, rest):
    """Values of which every product and sum is exact: x is 1 in its first column and -1, 0 or 1 in the others, w_gate
    64 in the first and 0 elsewhere, so that g = 64, silu(g) = 64 and its derivative 1 (exp(-64) is less than half a
    step of 1 in fp32). w_up and w_down have one element of size 1 a row: u is -1, 0 or 1, h and du are multiples of
    64, all sums are whole numbers below 2^24."""
    E = len(ends) - 1
    gen = torch.Generator(device="cuda").manual_seed(9)
    R = ends[-1] + rest
    x, dy = units((R, d), gen), units((R, d), gen)
    x[:, 0] = 1
    w_gate = torch.zeros((E, I, d), dtype=torch.bfloat16, device="cuda")
    w_gate[:, :, 0] = 64
    w_up, w_down = one_each(E, I, d, gen, 1), one_each(E, d, I, gen, 1)
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    new = lambda *s: torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda")
    pre, h, y, dpre, dx = new(R, 2, I), new(R, I), new(R, d), new(R, 2, I), new(R, d)
    dw = [torch.full_like(t, 7.0) for t in (w_gate, w_up, w_down)]
    dm.dmoe_expert_ffn(x, offsets, w_gate, w_up, w_down, h, y, pre=pre, zero_rest=True)
    dm.dmoe_expert_ffn_backward(dy, x, offsets, w_gate, w_up, w_down, pre, h, dpre, dx, *dw, zero_rest=True)
    assert dm.dmoe_expert_device_error()[0] == 0
    assert (y[ends[-1]:] == 0).all() and (dx[ends[-1]:] == 0).all()
    assert all((t[ends[-1]:] == 7).all() for t in (pre, h, dpre))
    tf32 = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        for e in range(E):
            sums = [torch.zeros(t.shape[1:], dtype=torch.float64, device="cuda") for t in dw]
            for lo in range(ends[e], ends[e + 1], 1 << 17):
                at = slice(lo, min(lo + (1 << 17), ends[e + 1]))
                u, dh = products(x[at], w_up[e]), products(dy[at], w_down[e].t())
                assert (pre[at, 0] == 64).all() and torch.equal(pre[at, 1], u.bfloat16())
                assert torch.equal(h[at], (64 * u).bfloat16())
                assert torch.equal(y[at], products(64 * u, w_down[e]).bfloat16())
                assert dh.abs().max() <= 256                             # (exact in bf16)
                dg, du = (dh * u).bfloat16(), (64 * dh).bfloat16()
                assert torch.equal(dpre[at, 0], dg) and torch.equal(dpre[at, 1], du)
                assert torch.equal(dx[at], (products(dg, w_gate[e].t()) + products(du, w_up[e].t())).bfloat16())
                for s, a, b in zip(sums, (dg, du, dy[at]), (x[at], x[at], h[at])):
                    s += products(a.t(), b.t()).double()
            for got, s in zip(dw, sums):
                assert torch.equal(got[e], s.float().bfloat16())
    finally:
        torch.backends.cuda.matmul.allow_tf32 = tf32


def test_a_sum_that_takes_longer_than_a_second():
    """dw_down of 2^28 + 77 rows of one expert (of more than share a sum): a wait is bounded by what it waits for. Sums of
    -1, 0 and 1, exact in fp32."""
    E, d, I, R = 37, 8, 8, (1 << 28) + 77
    gen = torch.Generator(device="cuda").manual_seed(11)
    dy, h = units((R, d), gen), units((R, I), gen)
    offsets = torch.tensor([0] + [R] * E, dtype=torch.int32, device="cuda")
    w = [torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((E, I, d), (E, I, d), (E, d, I))]
    dw_down = torch.full((E, d, I), 7.0, dtype=torch.bfloat16, device="cuda")
    dm.dmoe_expert_ffn_backward(dy, None, offsets, *w, None, h, None, None, None, None, dw_down)
    assert dm.dmoe_expert_device_error()[0] == 0
    want = torch.zeros((d, I), dtype=torch.float64, device="cuda")
    for lo in range(0, R, 1 << 22):
        at = slice(lo, lo + (1 << 22))
        want += products(dy[at].t(), h[at].t()).double()       # (whole numbers up to 2^22)
    assert torch.equal(dw_down[0], want.float().bfloat16()) and (dw_down[1:] == 0).all()
