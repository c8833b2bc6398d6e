"""4-bit expert matrices: quantising, the values that come back, and the products, against the
plain forms in 64 bits."""
import numpy as np
import pytest
import torch

from tests import parity as P
from tests import rows_oracle as O

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def f64(t):
    return t.double().cpu().numpy()


def make_w(E, N, K, seed=0):
    gen = torch.Generator().manual_seed(seed)
    w = torch.randn((E, N, K), generator=gen) * 0.02
    w[..., 0] *= 20
    return w.to(BF16).cuda()


def pack(desc, w):
    m = P.dm()
    codes, scales = m.alloc_q4(desc, "cuda")
    codes.fill_(0xA5)
    scales.fill_(0x7F)            # (NaNs, if any were left)
    m.dmoe_q4_quantize(desc, w, codes, scales)
    return codes, scales


@pytest.mark.parametrize("E,N,K", [(1, 1, 128), (3, 17, 128), (2, 16, 256), (2, 40, 384), (1, 130, 2048),
                                   (256, 8, 128)])
@pytest.mark.parametrize("g", [32, 64, 128])
def test_quantize_gives_the_defined_values(E, N, K, g):
    m = P.dm()
    w = make_w(E, N, K)
    w[0, 0, :g] = 0                                            # a group of zeros
    w[-1, -1, -g:] = torch.arange(g).to(BF16) - 3              # whole numbers: ties in abundance
    desc = m.make_q4_desc(E, N, K, g)
    out = torch.full_like(w, 5.0)
    m.dmoe_q4_dequantize(desc, *pack(desc, w), out)
    assert np.array_equal(f64(out), O.q4_values(f64(w), g)[2])


@pytest.mark.parametrize("K,g", [(32, 32), (96, 32), (64, 64), (192, 64), (160, 32)])
def test_quantize_widths_that_end_inside_a_tile(K, g):
    m = P.dm()
    w = make_w(2, 19, K)
    desc = m.make_q4_desc(2, 19, K, g)
    out = torch.empty_like(w)
    m.dmoe_q4_dequantize(desc, *pack(desc, w), out)
    assert np.array_equal(f64(out), O.q4_values(f64(w), g)[2])


def test_quantize_every_bf16_magnitude():
    """Every positive bf16 as the largest of its group, with fractions of it beside it."""
    m = P.dm()
    bits = torch.arange(0, 0x7F80, dtype=torch.int32)
    top = bits.to(torch.int16).view(BF16)
    g = 32
    frac = torch.linspace(-1, 1, g, dtype=torch.float64)
    w = (top.double()[:, None] * frac[None]).to(BF16)
    w[:, 0] = top
    w = w.cuda().contiguous()
    n = w.shape[0]                      # 32640 rows of one group
    desc = m.make_q4_desc(1, n, g, g)
    out = torch.empty_like(w)
    m.dmoe_q4_dequantize(desc, *pack(desc, w), out)
    assert np.array_equal(f64(out), O.q4_values(f64(w), g)[2], equal_nan=True)


def test_quantize_marks_groups_that_are_not_finite():
    m = P.dm()
    w = make_w(1, 16, 256)
    w[0, 3, 70] = float("inf")
    w[0, 9, 255] = float("nan")
    w[0, 10, 0] = float("-inf")
    desc = m.make_q4_desc(1, 16, 256, 64)
    out = torch.empty_like(w)
    m.dmoe_q4_dequantize(desc, *pack(desc, w), out)
    bad = torch.zeros(16, 4, dtype=torch.bool)
    bad[3, 1] = bad[9, 3] = bad[10, 0] = True
    assert torch.equal(out.isnan().view(16, 4, 64).all(-1).cpu(), bad)
    assert torch.equal(out.isnan().view(16, 4, 64).any(-1).cpu(), bad)


# ------------------------------------------------------------------------------ products

def group_sizes(kind, G, rng):
    if kind == "even":
        return np.full(G, 4)
    if kind == "one":
        n = np.zeros(G, int)
        n[G // 2] = 1
        return n
    n = rng.integers(0, 5, G)
    n[rng.integers(0, G)] = 70          # more than a tile, ragged
    n[rng.integers(0, G)] = 0
    n[0] = 17
    return n


def bounds(y, mag, K, t):
    """fp32 sums of K products (the tensor cores round a sum of several toward zero: a whole step
    of 2^-23 each), then one rounding to t."""
    acc = 1.01 * (K + 16) * 2.0 ** -23 * mag
    return acc, acc + torch.finfo(t).eps / 2 * (np.abs(y) + acc) + 1e-37


def swiglu_bounds(a, am, b, bm, K, t):
    """h = silu(a) b from a, b with the errors above: |silu'| <= 1.1, |silu(a)| <= |a|; silu itself
    is off by at most 2^-20 of its value (exp to 2 ulp of its argument's scale, one division), a
    quotient and a product by 2^-23."""
    ea, eb = bounds(a, am, K, t)[0], bounds(b, bm, K, t)[0]
    # exp(-a) is evaluated as 2^x: an error of |a| 2^-23 relative, on top of its own 2^-21
    silu = a / (1 + np.exp(-a))
    h = silu * b
    err = 1.1 * ea * (np.abs(b) + eb) + np.abs(silu) * eb
    err += np.abs(h) * (2.0 ** -20 + np.abs(a) * 2.0 ** -22)
    return h, err + torch.finfo(t).eps / 2 * (np.abs(h) + err) + 1e-37


def check_products(E, N, K, g, sizes, ids=None, rows_from=None, k=1, ydt=BF16, gated=False, gap=0,
                   seed=0):
    m = P.dm()
    rng = np.random.default_rng(seed)
    G = len(sizes)
    R = int(sizes.sum()) + 3             # three rows behind the last group's
    offsets = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    desc = m.make_q4_desc(E, N, K, g)
    ws = [make_w(E, N, K, seed + i) for i in range(2 if gated else 1)]
    vals = [O.q4_values(f64(w), g)[2] for w in ws]
    packed = [t for w in ws for t in pack(desc, w)]
    gen = torch.Generator().manual_seed(seed + 9)
    T = R if rows_from is None else rows_from
    xbuf = torch.randn((T, K + gap), generator=gen).to(BF16).cuda()
    x = xbuf[:, :K]
    rows = None
    src = np.arange(R)
    if rows_from is not None:
        rows = rng.integers(-k, T * k + 2 * k, R).astype(np.int32)     # some outside
        src = np.where((rows >= 0) & (rows // k < T), rows // k, -1)
    y = torch.full((R, N + gap), 3.0, dtype=ydt, device="cuda")
    call = m.dmoe_q4_swiglu if gated else m.dmoe_q4_linear
    call(desc, x, torch.from_numpy(offsets).cuda(), *packed, y[:, :N],
         rows=None if rows is None else torch.from_numpy(rows).cuda(), k=k,
         expert_ids=None if ids is None else torch.from_numpy(ids).cuda())
    experts = np.arange(G) if ids is None else ids
    ok = [i for i in range(G) if 0 <= experts[i] < E]
    live = np.zeros(R, bool)
    for i in ok:
        live[offsets[i]:offsets[i + 1]] = True
    safe = np.where((experts >= 0) & (experts < E), experts, 0)
    both = [O.q4_products(f64(x), src, offsets, safe, v) for v in vals]
    got = f64(y)
    if gated:
        want, tol = swiglu_bounds(*both[0], *both[1], K, ydt)
    else:
        want, tol = both[0][0], bounds(*both[0], K, ydt)[1]
    err = np.abs(got[:, :N] - want)
    assert (err[live] <= tol[live]).all(), (err / tol)[live].max()
    assert (got[~live] == 3.0).all() and (got[:, N:] == 3.0).all()      # left as they were
    return x, y


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("kind", ["even", "one", "ragged"])
@pytest.mark.parametrize("E,N,K,g", [(9, 48, 256, 64), (5, 33, 96, 32), (4, 1, 128, 128), (3, 200, 1024, 64),
                                     (2, 128, 2048, 128), (6, 130, 320, 32)])
def test_products(E, N, K, g, kind, gated):
    sizes = group_sizes(kind, E, np.random.default_rng(E))
    check_products(E, N, K, g, sizes, gated=gated)
    check_products(E, N, K, g, sizes, gated=gated, ydt=torch.float32, rows_from=11, k=3, gap=8)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows", [1, 2, 7, 8, 9, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 200, 256, 257, 530])
def test_rows_of_a_group(rows, gated):
    check_products(3, 80, 192, 64, np.array([rows, 0, 5]), gated=gated, seed=rows)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows", [1, 20, 70, 90, 128, 300])
@pytest.mark.parametrize("K", [2944, 3200, 8192])        # 23 stages (a CTA's), 25 and 64 (a pair's)
def test_long_sums_over_several_tiles(rows, K, gated):
    """More inputs than any ring of stages holds, many times over; the same result every time."""
    sizes = np.array([rows, 3])
    _, y = check_products(2, 300, K, 128, sizes, gated=gated, seed=rows, gap=8)
    for _ in range(3):
        assert torch.equal(check_products(2, 300, K, 128, sizes, gated=gated, seed=rows, gap=8)[1], y)


def test_long_sums_of_more_units_than_pairs():
    check_many_units(40, 640, 3200, 64, np.full(40, 3), True)
    check_many_units(40, 640, 3200, 64, np.full(40, 3), False)


def check_many_units(E, N, K, g, sizes, gated, seed=0):
    """The products of more units than CTAs, against torch in 64 bits on the dequantised weights (which
    tests of their own hold to the definition)."""
    m = P.dm()
    desc = m.make_q4_desc(E, N, K, g)
    R = int(sizes.sum())
    gen = torch.Generator(device="cuda").manual_seed(seed)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(sizes)]), dtype=torch.int32, device="cuda")
    packed, vals = [], []
    for _ in range(2 if gated else 1):
        w = torch.empty((E, N, K), dtype=BF16, device="cuda")
        for e in range(E):
            w[e] = torch.randn((N, K), generator=gen, device="cuda") * 0.02
        packed += pack(desc, w)
        m.dmoe_q4_dequantize(desc, packed[-2], packed[-1], w)
        vals.append(w)
    x = torch.randn((R, K), generator=gen, device="cuda").to(BF16)
    y = torch.full((R, N), 3.0, dtype=BF16, device="cuda")
    (m.dmoe_q4_swiglu if gated else m.dmoe_q4_linear)(desc, x, offsets, *packed, y)
    for e in np.flatnonzero(sizes):
        lo, hi = int(offsets[e]), int(offsets[e + 1])
        xe = x[lo:hi].double()
        s = [(xe @ v[e].double().T, xe.abs() @ v[e].double().abs().T) for v in vals]
        s = [(a.cpu().numpy(), b.cpu().numpy()) for a, b in s]
        if gated:
            want, tol = swiglu_bounds(*s[0], *s[1], K, BF16)
        else:
            want, tol = s[0][0], bounds(*s[0], K, BF16)[1]
        assert (np.abs(f64(y[lo:hi]) - want) <= tol).all(), e
    assert m.dmoe_q4_device_error()[0] == 0


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("K", [128, 256, 384, 1408])     # one stage a unit, two, three, eleven
@pytest.mark.parametrize("most", [5, 50, 90, 250])       # up to 16, 64, 96 rows a unit; several units
def test_more_units_than_ctas(K, most, gated):
    rng = np.random.default_rng(K + most)
    sizes = rng.integers(0, 6, 100)
    sizes[rng.integers(0, 100, 5)] = rng.integers(most // 2, most + 1, 5)
    check_many_units(100, 320, K, 64, sizes, gated, seed=K)


def test_more_units_than_a_cta_looks_up_at_once():
    check_many_units(256, 32768, 128, 128, np.full(256, 1), False)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("n,N,K", [(30, 320, 128), (61, 320, 256), (3, 4224, 256), (12, 8192, 128),
                                   (1, 4224, 3200), (1, 8192, 3200)])
def test_groups_between_the_two_limits(n, N, K, gated):
    """Groups of 65 to 96 rows, of one unit or two for each tile of outputs, in one turn of the CTAs or
    more, and in pairs."""
    check_many_units(n, N, K, 64, np.random.default_rng(n).integers(65, 97, n), gated, seed=n)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("ydt", [BF16, torch.float32])
@pytest.mark.parametrize("N,K,g", [(1, 256, 64), (33, 256, 128), (64, 512, 64), (65, 224, 32), (97, 1280, 32),
                                   (130, 2048, 128), (200, 1472, 64)])
def test_few_units(N, K, g, ydt, gated):
    """Fewer units than CTAs: widths of part of a tile, sums that end inside a block, groups of one row to
    several units."""
    for sizes in ([1], [3, 0, 33], [16, 17, 15], [80]):
        check_products(len(sizes), N, K, g, np.array(sizes), rows_from=7, k=3, ydt=ydt, gated=gated, gap=8)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows", [1, 31, 32, 33, 64, 65])
@pytest.mark.parametrize("N", [4096, 4864, 4992, 9728, 9792])
def test_about_as_many_units_as_ctas(rows, N, gated):
    """On 152 SMs: one turn or two, units of 64 rows or 96, with pairs of CTAs and without."""
    for K in (256, 384, 3328):
        check_many_units(1, N, K, 64, np.array([rows]), gated, seed=rows)


@pytest.mark.parametrize("gated", [False, True])
def test_groups_with_their_own_experts(gated):
    ids = np.array([3, 3, -1, 0, 6, 2, 2 ** 31 - 1], np.int32)         # twice the same; three left out
    sizes = np.array([5, 2, 4, 0, 3, 40, 6])
    check_products(6, 64, 128, 32, sizes, ids=ids, gated=gated)


def test_as_many_groups_as_there_can_be():
    check_many_units(512, 48, 128, 64, np.arange(512) % 3, True)
    ids = np.random.default_rng(0).integers(-1, 8, 512).astype(np.int32)
    check_products(7, 40, 128, 32, np.arange(512) % 3, ids=ids)


@pytest.mark.parametrize("R", [1, 3, 40, 300])
def test_dense(R):
    m = P.dm()
    N, K, g = 100, 512, 64
    w = make_w(1, N, K)
    desc = m.make_q4_desc(1, N, K, g)
    x = torch.randn(R, K, generator=torch.Generator().manual_seed(R)).to(BF16).cuda()
    y = torch.empty(R, N, dtype=BF16, device="cuda")
    m.dmoe_q4_linear(desc, x, None, *pack(desc, w), y)
    want, mag = O.q4_products(f64(x), np.arange(R), [0, R], [0], O.q4_values(f64(w), g)[2])
    assert (np.abs(f64(y) - want) <= bounds(want, mag, K, BF16)[1]).all()


def test_offsets_outside_the_rows_are_cut():
    m = P.dm()
    E, N, K = 3, 32, 64
    desc = m.make_q4_desc(E, N, K, 64)
    w = make_w(E, N, K)
    packed = pack(desc, w)
    x = torch.randn(8, K, generator=torch.Generator().manual_seed(0)).to(BF16).cuda()
    y = torch.full((8, N), 3.0, dtype=BF16, device="cuda")
    off = torch.tensor([-5, 4, 2, 2 ** 31 - 1], dtype=torch.int32, device="cuda")   # 0..4, none, 2..8
    m.dmoe_q4_linear(desc, x, off, *packed, y)
    vals = O.q4_values(f64(w), 64)[2]
    want, mag = O.q4_products(f64(x), np.arange(8), [0, 4], [0], vals)
    ok = np.abs(f64(y) - want) <= bounds(want, mag, K, BF16)[1]
    assert ok[:2].all()
    want, mag = O.q4_products(f64(x), np.arange(8), [4, 8], [2], vals)
    assert (np.abs(f64(y) - want) <= bounds(want, mag, K, BF16)[1])[4:].all()


def test_infinities_stay_in_their_rows():
    m = P.dm()
    desc = m.make_q4_desc(1, 48, 128, 64)
    w = make_w(1, 48, 128)
    packed = pack(desc, w)
    for R in (5, 150):
        x = torch.randn(R, 128, generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
        clean, y = (torch.empty(R, 48, dtype=BF16, device="cuda") for _ in range(2))
        m.dmoe_q4_linear(desc, x, None, *packed, clean)
        x[3] = float("inf")
        x[1, 7] = float("nan")
        m.dmoe_q4_linear(desc, x, None, *packed, y)
        rest = [i for i in range(R) if i not in (1, 3)]
        assert torch.equal(y[rest], clean[rest])
        assert y[1].isnan().all() and not torch.isfinite(y[3]).any()


def test_no_rows():
    m = P.dm()
    desc = m.make_q4_desc(2, 32, 64, 64)
    packed = pack(desc, make_w(2, 32, 64))
    x = torch.empty(0, 64, dtype=BF16, device="cuda")
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    m.dmoe_q4_linear(desc, x, off, *packed, torch.empty(0, 32, dtype=BF16, device="cuda"))
    y = torch.full((4, 32), 3.0, dtype=BF16, device="cuda")            # rows, but none in a group
    x = torch.empty(4, 64, dtype=BF16, device="cuda")
    m.dmoe_q4_swiglu(desc, x, off, *packed, *packed, y)
    assert bool((y == 3.0).all())


def test_products_after_the_dispatch():
    """The unique experts' list and offsets of dmoe_dispatch as the groups."""
    m = P.dm()
    T, k, E, N, K = 24, 4, 32, 48, 256
    rng = np.random.default_rng(0)
    idx = np.stack([rng.permutation(9)[:k] for _ in range(T)]).astype(np.int32) * 3
    i32 = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")
    ld = m.make_desc(K, E, k, 128, 0, T, 1, mode=m.DMOE_ROUTE_TOKEN)
    nu, ids, off, rows, pos = i32(1), i32(E), i32(E + 1), i32(T * k), i32(T * k)
    m.dmoe_dispatch(ld, torch.from_numpy(idx).cuda(), nu, ids, off, rows, pos,
                    workspace=m.alloc_workspace(ld))
    desc = m.make_q4_desc(E, N, K, 64)
    w = make_w(E, N, K)
    x = torch.randn(T, K, generator=torch.Generator().manual_seed(0)).to(BF16).cuda()
    y = torch.empty(T * k, N, dtype=BF16, device="cuda")
    m.dmoe_q4_linear(desc, x, off, *pack(desc, w), y, rows=rows, k=k, expert_ids=ids)
    offs, rows_, _ = O.sort_tokens(idx, E)
    want, mag = O.q4_products(f64(x), rows_ // k, offs, np.arange(E), O.q4_values(f64(w), 64)[2])
    assert (np.abs(f64(y) - want) <= bounds(want, mag, K, BF16)[1]).all()


def test_on_another_stream_and_replayed():
    m = P.dm()
    E, N, K, R = 4, 64, 256, 90
    desc = m.make_q4_desc(E, N, K, 64)
    packed = pack(desc, make_w(E, N, K)) + pack(desc, make_w(E, N, K, 1))
    x = torch.randn(R, K, generator=torch.Generator().manual_seed(0)).to(BF16).cuda()
    off = torch.tensor([0, 3, 40, 40, 90], dtype=torch.int32, device="cuda")
    y = torch.empty(R, N, dtype=BF16, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    m.dmoe_q4_swiglu(desc, x, off, *packed, y, stream=s)
    s.synchronize()
    first = y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.dmoe_q4_swiglu(desc, x, off, *packed, y)
    y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, first)
    x.copy_(x.flip(0))
    off.copy_(torch.tensor([0, 0, 64, 70, 80], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    again = y.clone()
    m.dmoe_q4_swiglu(desc, x, off, *packed, y)
    assert torch.equal(y, again)


def test_offsets_past_32_bits():
    """Matrices whose last one lies behind 2^31 bytes of codes, and rows behind 2^31 elements: the same
    values as alone and close together."""
    m = P.dm()
    E, N, K, g, R = 20, 16384, 16384, 64, 12
    desc, one = m.make_q4_desc(E, N, K, g), m.make_q4_desc(1, N, K, g)
    gen = torch.Generator(device="cuda").manual_seed(5)
    w = torch.zeros((E, N, K), dtype=BF16, device="cuda")
    w[-1] = torch.randn((N, K), generator=gen, device="cuda", dtype=BF16) * 0.02
    packed, alone = pack(desc, w), pack(one, w[-1:])
    values = torch.empty_like(w[-1:])
    m.dmoe_q4_dequantize(one, *alone, values)
    m.dmoe_q4_dequantize(desc, *packed, w)
    assert torch.equal(w[-1:], values) and not w[:-1].any()
    del w, values
    x = torch.randn((R, K), generator=gen, device="cuda").to(BF16)
    near = torch.empty((R, N), dtype=BF16, device="cuda")
    far_x, far_y = (torch.empty((R, 1 << 28), dtype=BF16, device="cuda")[:, :n] for n in (K, N))
    far_x.copy_(x)
    ids = torch.tensor([E - 1], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, R], dtype=torch.int32, device="cuda")
    m.dmoe_q4_linear(one, x, None, *alone, near)
    m.dmoe_q4_linear(desc, far_x, offsets, *packed, far_y, expert_ids=ids)
    assert near.any() and torch.equal(far_y, near)
    assert m.dmoe_q4_device_error()[0] == 0
