"""Tokens sorted by expert, their rows gathered and combined, and the gradients, against the plain
forms in 64 bits."""
import numpy as np
import pytest
import torch

from tests import parity as P
from tests import rows_oracle as O

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
I32 = torch.int32


def i32(n, fill=None):
    return torch.full((n,), fill, dtype=I32, device="cuda") if fill is not None else torch.empty(
        n, dtype=I32, device="cuda")


def make_idx(T, k, E, masked, seed=0, skew=False):
    rng = np.random.default_rng(seed + T * 131 + k)
    idx = rng.integers(0, E, (T, k)) if not skew else np.minimum(
        rng.geometric(0.3, (T, k)) - 1, E - 1)
    if masked == "all":
        idx[:] = -1
    elif masked:
        idx[rng.random((T, k)) < masked] = -1
        idx[rng.random(T) < masked] = -(2 ** 31)
    return idx.astype(np.int32)


def sort(idx, E, ws=None):
    m = P.dm()
    T, k = idx.shape
    if ws is None:
        ws = m.alloc_sort_workspace(T, k, E)
    out = i32(E + 1, 77), i32(T * k, 77), i32(T * k, 77)
    m.dmoe_sort_tokens(torch.from_numpy(idx).cuda(), E, *out, workspace=ws)
    return out, ws


@pytest.mark.parametrize("T,k,E", [(0, 4, 7), (1, 1, 1), (1, 16, 256), (3, 5, 9), (32, 8, 256), (512, 8, 256),
                                   (4096, 1, 33), (4097, 1, 33), (1031, 6, 255), (9000, 16, 64),
                                   (65536, 8, 256), (152000, 4, 130)])
@pytest.mark.parametrize("masked", [0, 0.3, "all"])
@pytest.mark.parametrize("skew", [False, True])
def test_sort(T, k, E, masked, skew):
    idx = make_idx(T, k, E, masked, skew=skew)
    out, ws = sort(idx, E)
    for a, b in zip(out, O.sort_tokens(idx, E)):
        assert np.array_equal(a.cpu().numpy(), b)
    assert P.dm().dmoe_get_device_error(ws)[0] == 0


def test_sort_records_ids_that_are_no_expert():
    for T in (40, 5000):
        idx = make_idx(T, 4, 16, 0.1)
        idx[T // 2, 1] = 16
        idx[T // 3, 0] = 2 ** 31 - 1
        out, ws = sort(idx, 16)
        for a, b in zip(out, O.sort_tokens(idx, 16)):     # such a slot counts as one without
            assert np.array_equal(a.cpu().numpy(), b)
        st, info = P.dm().dmoe_get_device_error(ws)
        assert st == 5 and info[2] in (T // 2 * 4 + 1, T // 3 * 4)
        again, _ = sort(make_idx(T, 4, 16, 0.1), 16, ws)
        assert P.dm().dmoe_get_device_error(ws)[0] == 0


def test_sort_agrees_with_the_dispatch():
    m = P.dm()
    rng = np.random.default_rng(3)
    T, k, E = 96, 8, 256
    idx = np.stack([rng.permutation(40)[:k] for _ in range(T)]).astype(np.int32)
    (offsets, rows, pos), _ = sort(idx, E)
    desc = m.make_desc(256, E, k, 128, 0, T, 1, mode=m.DMOE_ROUTE_TOKEN)
    out = i32(1), i32(E), i32(E + 1), i32(T * k), i32(T * k)
    m.dmoe_dispatch(desc, torch.from_numpy(idx).cuda(), *out, workspace=m.alloc_workspace(desc))
    assert torch.equal(out[3], rows) and torch.equal(out[4], pos)
    u = int(out[0])
    assert torch.equal(out[2][:u], offsets[out[1][:u].long()])


# ------------------------------------------------------------------------------ rows

SHAPES = [(1, 1, 1), (1, 8, 2048), (3, 2, 7), (37, 3, 1001), (64, 8, 512), (130, 16, 136), (257, 9, 66),
          (2, 10, 8200), (300, 6, 33)]


def rows_of(n, d, dtype, seed, gap=0, shift=0):
    """[n, d] normal values whose rows are d + gap elements apart, `shift` elements off the base;
    and the whole buffer."""
    gen = torch.Generator().manual_seed(seed)
    buf = torch.randn(shift + n * (d + gap), generator=gen).to(dtype).cuda()
    return buf[shift:].view(n, d + gap)[:, :d], buf


def f64(t):
    return t.double().cpu().numpy()


def setup(T, k, masked, seed=0):
    idx = make_idx(T, k, 13, masked, seed)
    return O.sort_tokens(idx, 13)[2]


def layouts(d):
    # contiguous; rows apart by whole pieces and by odd ones; off the 16-byte boundary
    return [(0, 0), (8, 8), (1, 3), (2, 2)]


@pytest.mark.parametrize("T,k,d", SHAPES)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("masked", [0, 0.3, "all"])
def test_gather(T, k, d, dtype, masked):
    m, t = P.dm(), TYPES[dtype]
    pos = setup(T, k, masked)
    pd = torch.from_numpy(pos).cuda()
    for gap, shift in layouts(d):
        x, _ = rows_of(T, d, t, 1, gap, shift)
        xs, buf = rows_of(T * k, d, t, 2, gap, shift)
        before = buf.clone()
        m.dmoe_gather_rows(x, pd, xs)
        assert np.array_equal(f64(xs), O.gather(f64(x), pos, k))
        keep = torch.ones_like(buf, dtype=torch.bool)
        keep[shift:].view(T * k, d + gap)[:, :d] = False
        assert torch.equal(buf[keep], before[keep])


def bound(exact, mag, terms, t):
    """fp32 sums of `terms` products in any order, then one rounding to t (half a step of it, and
    half the smallest subnormal one). Higher orders of 2^-24 are below a hundredth of the first."""
    u = 2.0 ** -24
    acc = 1.01 * (terms + 1) * u * mag
    half = torch.finfo(t).eps / 2
    tiny = torch.finfo(t).tiny * torch.finfo(t).eps
    return acc + half * (np.abs(exact) + acc) + tiny


@pytest.mark.parametrize("T,k,d", SHAPES)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("masked", [0, 0.3, "all"])
def test_combine_and_gather_backward(T, k, d, dtype, masked):
    m, t = P.dm(), TYPES[dtype]
    pos = setup(T, k, masked)
    pd = torch.from_numpy(pos).cuda()
    gates = torch.rand(T, k, generator=torch.Generator().manual_seed(5))
    gates[torch.from_numpy(pos).view(T, k) < 0] = float("nan")      # not looked at
    for gap, shift in layouts(d):
        ys, _ = rows_of(T * k, d, t, 1, gap, shift)
        for i, p in enumerate(pos):
            if p < 0:
                ys[~p] = float("inf")                                # nor these rows
        add, _ = rows_of(T, d, t, 2, gap, shift)
        for g, a in ((gates, add), (gates, None), (None, add), (None, None)):
            y, buf = rows_of(T, d, t, 3, gap, shift)
            before = buf.clone()
            if g is None and a is None:
                m.dmoe_gather_rows_backward(ys, pd, y)
            else:
                m.dmoe_combine_rows(ys, pd, None if g is None else g.cuda(), a, y)
            want, mag = O.combine(f64(ys), pos, None if g is None else f64(g),
                                  None if a is None else f64(a), T)
            assert (np.abs(f64(y) - want) <= bound(want, mag, k + 1, t)).all()
            keep = torch.ones_like(buf, dtype=torch.bool)
            keep[shift:].view(T, d + gap)[:, :d] = False
            assert torch.equal(buf[keep], before[keep])
        y = add.clone()                                              # in place of the addend
        m.dmoe_combine_rows(ys, pd, gates.cuda(), y, y)
        out = torch.empty_like(y)
        m.dmoe_combine_rows(ys, pd, gates.cuda(), add, out)
        assert torch.equal(y, out)


@pytest.mark.parametrize("T,k,d", SHAPES)
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("masked", [0, 0.3, "all"])
def test_combine_backward(T, k, d, dtype, masked):
    m, t = P.dm(), TYPES[dtype]
    pos = setup(T, k, masked)
    pd = torch.from_numpy(pos).cuda()
    gates = torch.rand(T, k, generator=torch.Generator().manual_seed(5)).cuda()
    for gap, shift in layouts(d):
        dy, _ = rows_of(T, d, t, 1, gap, shift)
        ys, _ = rows_of(T * k, d, t, 2, gap, shift)
        for i, p in enumerate(pos):
            if p < 0:
                ys[~p] = float("nan")
        dys, buf = rows_of(T * k, d, t, 3, gap, shift)
        before = buf.clone()
        dg = torch.full((T, k), 7.0, device="cuda")
        m.dmoe_combine_rows_backward(dy, ys, pd, gates, dys, dg)
        want, wg, mag = O.combine_backward(f64(dy), f64(ys), pos, f64(gates))
        assert (np.abs(f64(dys) - want) <= bound(want, np.abs(want), 1, t)).all()
        assert (np.abs(f64(dg).reshape(-1) - wg) <= bound(wg, mag, d, torch.float32)).all()
        keep = torch.ones_like(buf, dtype=torch.bool)
        keep[shift:].view(T * k, d + gap)[:, :d] = False
        assert torch.equal(buf[keep], before[keep])
        # one of the two alone, and without gates
        only, og = torch.full_like(dys, 9.0), torch.full_like(dg, 9.0)
        m.dmoe_combine_rows_backward(dy, None, pd, gates, only, None)
        m.dmoe_combine_rows_backward(dy, ys, pd, gates, None, og)
        assert torch.equal(only, dys) and torch.equal(og, dg)
        m.dmoe_combine_rows_backward(dy, ys, pd, None, dys, dg)
        want, wg, mag = O.combine_backward(f64(dy), f64(ys), pos, None)
        assert np.array_equal(f64(dys), want)
        assert torch.equal(og, dg)


def test_bad_positions_are_not_followed():
    m = P.dm()
    T, k, d = 9, 4, 64
    x, _ = rows_of(T, d, torch.bfloat16, 0)
    ys, _ = rows_of(T * k, d, torch.bfloat16, 1)
    for bad in (2 ** 31 - 1, -2 ** 31, T * k, -T * k - 1):
        pos = setup(T, k, 0)
        pos[::3] = bad
        pd = torch.from_numpy(pos).cuda()
        xs = torch.zeros(T * k, d, dtype=torch.bfloat16, device="cuda")
        m.dmoe_gather_rows(x, pd, xs)
        named = np.where(np.arange(T * k) % 3 == 0, -1, pos)
        assert np.array_equal(f64(xs), O.gather(f64(x), named, k))
        y = torch.empty(T, d, dtype=torch.float32, device="cuda").to(torch.bfloat16)
        m.dmoe_combine_rows(ys, pd, None, None, y)
        want, mag = O.combine(f64(ys), named, None, None, T)
        assert (np.abs(f64(y) - want) <= bound(want, mag, k + 1, torch.bfloat16)).all()
        dg = torch.empty(T, k, device="cuda")
        xs.zero_()
        m.dmoe_combine_rows_backward(x, ys, pd, None, xs, dg)
        assert np.array_equal(f64(xs), O.gather(f64(x), named, k))
        assert (f64(dg).reshape(-1)[::3] == 0).all()


def test_no_tokens():
    m = P.dm()
    e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
    pos = i32(0)
    m.dmoe_gather_rows(e(0, 8), pos, e(0, 8))
    m.dmoe_gather_rows_backward(e(0, 8), pos, e(0, 8))
    m.dmoe_combine_rows(e(0, 8), pos, None, None, e(0, 8))
    m.dmoe_combine_rows_backward(e(0, 8), e(0, 8), pos, None, e(0, 8), None)
    torch.cuda.synchronize()


def test_infinities_and_nans_stay_in_their_rows():
    m = P.dm()
    T, k, d = 6, 2, 40
    pos = setup(T, k, 0)
    pd = torch.from_numpy(pos).cuda()
    ys, _ = rows_of(T * k, d, torch.float32, 0)
    ys[int(pos[0])] = float("inf")
    ys[int(pos[5])] = float("nan")
    y = torch.empty(T, d, device="cuda")
    m.dmoe_combine_rows(ys, pd, torch.ones(T, k, device="cuda"), None, y)
    assert torch.isinf(y[0]).all() and torch.isnan(y[2]).all()
    assert torch.isfinite(y[[1, 3, 4, 5]]).all()


def test_on_another_stream_and_replayed():
    m = P.dm()
    T, k, d, E = 200, 8, 256, 64
    s = torch.cuda.Stream()
    idx = torch.from_numpy(make_idx(T, k, E, 0.2)).cuda()
    ws = m.alloc_sort_workspace(T, k, E)
    offsets, rows, pos = i32(E + 1), i32(T * k), i32(T * k)
    x, _ = rows_of(T, d, torch.bfloat16, 0)
    xs = torch.empty(T * k, d, dtype=torch.bfloat16, device="cuda")
    y = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    g = torch.rand(T, k, device="cuda")
    dys, dg = torch.empty_like(xs), torch.empty_like(g)

    def step(stream=None):
        m.dmoe_sort_tokens(idx, E, offsets, rows, pos, workspace=ws, stream=stream)
        m.dmoe_gather_rows(x, pos, xs, stream=stream)
        m.dmoe_combine_rows(xs, pos, g, x, y, stream=stream)
        m.dmoe_combine_rows_backward(y, xs, pos, g, dys, dg, stream=stream)
        m.dmoe_gather_rows_backward(dys, pos, y, stream=stream)

    torch.cuda.synchronize()
    step(s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2):
        idx.copy_(torch.from_numpy(make_idx(T, k, E, 0.2, seed)))
        x.copy_(rows_of(T, d, torch.bfloat16, seed)[0])
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (offsets, rows, pos, xs, dys, dg, y)]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (offsets, rows, pos, xs, dys, dg, y)):
            assert torch.equal(a, b)
        want = O.sort_tokens(idx.cpu().numpy(), E)
        assert np.array_equal(got[2].cpu().numpy(), want[2])
        assert np.array_equal(f64(got[3]), O.gather(f64(x), want[2], k))


def test_offsets_past_32_bits():
    """Rows so far apart that the last ones lie behind 2^31 elements: the same values as close together."""
    m = P.dm()
    T, k, d, E = 6, 2, 80, 5
    idx = make_idx(T, k, E, 0)
    idx[4, 1] = -1
    pos = sort(idx, E)[0][2]
    gen = torch.Generator(device="cuda").manual_seed(3)
    far_t, far_r, far_o = (torch.empty((n, 1 << 28 << (n == T)), dtype=torch.bfloat16, device="cuda")[:, :d]
                           for n in (T, T * k, T * k))
    x, ys, dy = (torch.randn((n, d), generator=gen, device="cuda").to(torch.bfloat16)
                 for n in (T, T * k, T))
    gates = torch.rand((T, k), generator=gen, device="cuda")

    near = torch.empty_like(ys)
    m.dmoe_gather_rows(x, pos, near)
    far_t.copy_(x)
    m.dmoe_gather_rows(far_t, pos, far_r)
    assert torch.equal(far_r, near)

    near = torch.empty_like(x)
    m.dmoe_combine_rows(ys, pos, gates, None, near)
    far_r.copy_(ys)
    m.dmoe_combine_rows(far_r, pos, gates, None, far_t)
    assert torch.equal(far_t, near)

    near, dgates, far_gates = torch.empty_like(ys), torch.empty_like(gates), torch.empty_like(gates)
    m.dmoe_combine_rows_backward(dy, ys, pos, gates, near, dgates)
    far_t.copy_(dy)
    m.dmoe_combine_rows_backward(far_t, far_r, pos, gates, far_o, far_gates)
    assert torch.equal(far_o, near) and torch.equal(far_gates, dgates)


@pytest.mark.parametrize("d", [64, 33])
def test_rows_that_no_position_names_are_not_written(d):
    """Entries that are not followed, and two that name one row (with the same token's values)."""
    m = P.dm()
    T, k = 9, 4
    x, _ = rows_of(T, d, torch.bfloat16, 0)
    pos = setup(T, k, 0)
    pos[::5] = T * k
    pos[2] = pos[1]
    pos[7] = ~pos[7]                                       # named, by a slot without an expert
    pd = torch.from_numpy(pos).cuda()
    named = np.zeros(T * k, bool)
    want = np.full((T * k, d), 5.0)
    for i, p in enumerate(pos):
        if p < T * k:
            named[p if p >= 0 else ~p] = True
            want[p if p >= 0 else ~p] = f64(x)[i // k] if p >= 0 else 0.0
    assert not named.all()
    xs = torch.full((T * k, d), 5.0, dtype=torch.bfloat16, device="cuda")
    m.dmoe_gather_rows(x, pd, xs)
    assert np.array_equal(f64(xs), want)
    xs.fill_(5.0)
    m.dmoe_combine_rows_backward(x, None, pd, None, xs, None)
    assert np.array_equal(f64(xs), want)
