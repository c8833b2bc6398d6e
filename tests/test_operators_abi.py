"""Sorting, gathering, combining and the 4-bit matrices without a GPU: sizes, exports, and the
refusals that come before any launch."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from tests import rows_oracle as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p
FAKE = 1 << 40     # aligned, never dereferenced: the checks return first


@pytest.fixture(scope="module")
def dm():
    import paper_2605_30876_gb300 as dm
    return dm


@pytest.fixture(scope="module")
def lib(dm):
    return dm._lib


def test_every_declared_call_is_exported_and_bound(dm):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "dmoe.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(dmoe_[a-z0-9_]+)\s*\(", text))
    assert {"dmoe_sort_tokens", "dmoe_gather_rows", "dmoe_combine_rows_backward", "dmoe_q4_linear",
            "dmoe_q4_swiglu", "dmoe_q4_quantize"} <= names
    for n in names:
        assert hasattr(dm._lib, n), n
    for n in dm.__all__:
        assert hasattr(dm, n), n


def test_sort_workspace(dm):
    assert dm.dmoe_sort_workspace_size(0, 1, 1) >= 16
    assert dm.dmoe_sort_workspace_size(32, 8, 256) < 1024
    # the counts of at most 148 chunks, whatever the number of tokens
    assert dm.dmoe_sort_workspace_size(2 ** 27, 8, 256) <= 256 + 148 * 257 * 4


@pytest.mark.parametrize("T,k,E,status", [
    (-1, 8, 256, 1), (4, 0, 256, 1), (4, 8, 0, 1), (4, 17, 256, 2), (4, 8, 257, 2),
    (2 ** 27 + 1, 8, 256, 2), (2 ** 62, 16, 256, 2)])
def test_sort_refusals(dm, lib, T, k, E, status):
    with pytest.raises(dm.DmoeError) as ei:
        dm.dmoe_sort_workspace_size(T, k, E)
    assert ei.value.status == status
    f = [P(FAKE)] * 5
    assert lib.dmoe_sort_tokens(T, k, E, *f, 1 << 30, None) == status


def test_sort_pointer_refusals(dm, lib):
    n = dm.dmoe_sort_workspace_size(4, 8, 256)
    good = [P(FAKE)] * 5
    for i in range(5):
        for bad in (None, P(FAKE + 4)):
            a = list(good)
            a[i] = bad
            assert lib.dmoe_sort_tokens(4, 8, 256, *a, n, None) == 1
    assert lib.dmoe_sort_tokens(4, 8, 256, *good[:4], P(FAKE + 16), n, None) == 1
    assert lib.dmoe_sort_tokens(4, 8, 256, *good, n - 1, None) == 3


def rows_calls(lib):
    """name -> a call of (dtype, T, k, d, pointers by name, strides by name)."""
    def ptrs(p, names):
        return [P(p[n]) if p[n] else None for n in names]

    def gather(t, T, k, d, p, s):
        a, b, c = ptrs(p, ("x", "pos", "out"))
        return lib.dmoe_gather_rows(t, T, k, d, a, s["x"], b, c, s["out"], None)

    def gather_backward(t, T, k, d, p, s):
        a, b, c = ptrs(p, ("x", "pos", "out"))
        return lib.dmoe_gather_rows_backward(t, T, k, d, a, s["x"], b, c, s["out"], None)

    def combine(t, T, k, d, p, s):
        a, b, g, add, c = ptrs(p, ("x", "pos", "gates", "add", "out"))
        return lib.dmoe_combine_rows(t, T, k, d, a, s["x"], b, g, add, s["add"], c, s["out"], None)

    def combine_backward(t, T, k, d, p, s):
        a, y, b, g, c, dg = ptrs(p, ("x", "add", "pos", "gates", "out", "dgates"))
        return lib.dmoe_combine_rows_backward(t, T, k, d, a, s["x"], y, s["add"], b, g, c, s["out"],
                                              dg, None)
    return dict(gather=gather, gather_backward=gather_backward, combine=combine,
                combine_backward=combine_backward)


@pytest.mark.parametrize("name", ["gather", "gather_backward", "combine", "combine_backward"])
def test_row_refusals(lib, name):
    call = rows_calls(lib)[name]
    p = {n: FAKE + i * 4096 for i, n in enumerate(("x", "pos", "gates", "add", "out", "dgates"))}
    s = dict(x=64, add=64, out=64)
    assert call(0, 0, 8, 64, dict.fromkeys(p), s) == 0                # no tokens: nothing to do
    for args, status in [((3, 4, 8, 64), 1), ((-1, 4, 8, 64), 1), ((0, -1, 8, 64), 1),
                         ((0, 4, 0, 64), 1), ((0, 4, 8, 0), 1), ((0, 4, 17, 64), 2),
                         ((0, 2 ** 27 + 1, 8, 64), 2), ((0, 4, 8, 2 ** 20 + 1), 2)]:
        assert call(*args, p, s) == status, args
    for need in ("x", "pos", "out"):
        if not (name == "combine_backward" and need == "out"):
            assert call(0, 4, 8, 64, dict(p, **{need: None}), s) == 1, need
    for odd in ("x", "out"):                                          # off an element's boundary
        assert call(0, 4, 8, 64, dict(p, **{odd: FAKE + 1}), s) == 1, odd
        assert call(2, 4, 8, 64, dict(p, **{odd: FAKE + 2}), s) == 1, odd
        assert call(0, 4, 8, 64, p, dict(s, **{odd: 63})) == 1, odd
    assert call(0, 4, 8, 64, dict(p, pos=FAKE + 4), s) == 1
    assert call(0, 4, 8, 64, dict(p, out=p["x"]), s) == 1             # in place
    if name.startswith("combine"):
        assert call(0, 4, 8, 64, dict(p, gates=FAKE + 4), s) == 1
        assert call(0, 4, 8, 64, p, dict(s, add=63)) == 1
    if name == "combine":
        assert call(0, 4, 8, 64, dict(p, add=p["out"]), dict(s, add=72)) == 1
    if name == "combine_backward":
        assert call(0, 4, 8, 64, dict(p, out=None, dgates=None), s) == 1
        assert call(0, 4, 8, 64, dict(p, add=None), s) == 1           # dgates without ys
        assert call(0, 4, 8, 64, dict(p, dgates=p["gates"]), s) == 1


@pytest.mark.parametrize("kw,status", [
    (dict(n_experts=0), 1), (dict(n_out=0), 1), (dict(n_in=0), 1), (dict(group=0), 1),
    (dict(group=16), 2), (dict(group=96), 2), (dict(n_in=96, group=64), 2),
    (dict(n_in=16384 + 64), 2), (dict(n_experts=513), 2), (dict(n_out=65537), 2)])
def test_q4_desc_refusals(dm, lib, kw, status):
    a = dict(n_experts=4, n_out=24, n_in=128, group=64)
    a.update(kw)
    desc = dm.make_q4_desc(**a)
    with pytest.raises(dm.DmoeError) as ei:
        dm.dmoe_q4_size(desc)
    assert ei.value.status == status
    f = P(FAKE)
    assert lib.dmoe_q4_quantize(ctypes.byref(desc), f, f, f, None) == status
    assert lib.dmoe_q4_dequantize(ctypes.byref(desc), f, f, f, None) == status
    assert lib.dmoe_q4_linear(ctypes.byref(desc), 4, 1, f, 1 << 20, 4, f, 1, f, f, f, f, P(FAKE * 2),
                              1 << 20, 0, None) == status


def test_q4_sizes(dm):
    # 4 bits a weight and 16 a group, where rows are whole 32s and inputs whole 128s
    assert dm.dmoe_q4_size(dm.make_q4_desc(3, 32, 512, 64)) == (3 * 32 * 256, 3 * 32 * 8 * 2)
    # 33 rows: 64; 160 inputs: 256
    assert dm.dmoe_q4_size(dm.make_q4_desc(1, 33, 160, 32)) == (64 * 128, 64 * 8 * 2)


def test_q4_product_refusals(dm, lib):
    desc = dm.make_q4_desc(4, 24, 128, 64)

    def call(fn="linear", desc=desc, R=8, groups=4, x=FAKE, ldx=128, T_x=8, rows=None, k=1,
             offsets=FAKE, ids=None, w=None, y=FAKE * 2, ldy=24, ydt=0):
        n = 4 if fn == "swiglu" else 2
        w = [FAKE * 3 + 4096 * i for i in range(n)] if w is None else w
        p = lambda v: None if v is None else P(v)
        return getattr(lib, "dmoe_q4_" + fn)(
            ctypes.byref(desc), R, groups, p(x), ldx, T_x, p(rows), k, p(offsets), p(ids),
            *[p(v) for v in w], p(y), ldy, ydt, None)
    for fn, n in (("linear", 2), ("swiglu", 4)):
        assert call(fn, R=0) == 0                     # no rows: nothing to do
        assert call(fn, R=-1) == 1
        assert call(fn, groups=0) == 1
        assert call(fn, groups=513, ids=FAKE) == 2
        assert call(fn, groups=5) == 1                # more groups than experts, without ids
        assert call(fn, groups=2, offsets=None) == 1
        assert call(fn, k=0) == 1
        assert call(fn, k=17) == 2
        assert call(fn, ldx=127) == 1
        assert call(fn, ldx=132) == 1                 # rows off the 16-byte boundaries
        assert call(fn, x=FAKE + 8) == 1
        assert call(fn, x=None) == 1
        assert call(fn, T_x=7) == 1                   # fewer rows of x than R, without a list
        assert call(fn, T_x=-1) == 1
        assert call(fn, T_x=0, rows=FAKE) == 1        # no row of x at all
        assert call(fn, T_x=2 ** 31) == 2
        assert call(fn, ldx=2 ** 39) == 2
        assert call(fn, ldy=23) == 1
        assert call(fn, ydt=1) == 1
        assert call(fn, y=None) == 1
        assert call(fn, y=FAKE) == 1                  # in place
        assert call(fn, y=FAKE * 2 + 2, ydt=2) == 1
        assert call(fn, R=2 ** 30 + 1, T_x=2 ** 30 + 1) == 2
        # more units than 32 bits count
        assert call(fn, R=2 ** 30, T_x=2 ** 30, groups=256, ids=FAKE) == 2
        for a in ("rows", "offsets", "ids"):
            assert call(fn, **{a: FAKE + 4}) == 1
        for i in range(n):
            for bad in (None, FAKE + 8):
                w = [FAKE * 3 + 4096 * j for j in range(n)]
                w[i] = bad
                assert call(fn, w=w) == 1


def test_binding_refuses_host_tensors_and_wrong_shapes(dm):
    x, pos = torch.zeros(4, 8), torch.zeros(8, dtype=torch.int32)
    with pytest.raises(ValueError):
        dm.dmoe_gather_rows(x, pos, torch.zeros(8, 8))
    with pytest.raises(ValueError):
        dm.dmoe_combine_rows(torch.zeros(8, 8), pos, None, None, x)
    with pytest.raises(ValueError):
        dm.dmoe_gather_rows(x, torch.zeros(9, dtype=torch.int32), torch.zeros(9, 8))
    with pytest.raises(TypeError):
        dm.dmoe_gather_rows(x.double(), pos, torch.zeros(8, 8))
    with pytest.raises(TypeError):
        dm.dmoe_sort_tokens(torch.zeros(8, dtype=torch.int32), 4, None, None, None,
                            workspace=torch.zeros(256, dtype=torch.uint8))
    with pytest.raises(ValueError):
        dm.dmoe_q4_linear(dm.make_q4_desc(1, 16, 64, 64), torch.zeros(1, 64, dtype=torch.bfloat16),
                          None, torch.zeros(1, dtype=torch.uint8), None,
                          torch.zeros(1, 16, dtype=torch.bfloat16))


# ---------------------------------------------------------------- the oracle's own pins

def test_oracle_sort_by_hand():
    offsets, rows, pos = O.sort_tokens(np.array([[2, 0], [-1, 2], [0, 9]]), 3)
    assert offsets.tolist() == [0, 2, 2, 4]
    assert rows.tolist() == [1, 4, 0, 3, -1, -1]
    assert pos.tolist() == [2, 0, -5, 3, 1, -6]


def test_oracle_combine_is_the_transpose_of_gather():
    rng = np.random.default_rng(0)
    idx = rng.integers(-1, 5, (7, 3))
    _, _, pos = O.sort_tokens(idx, 5)
    x, ys = rng.normal(size=(7, 4)), rng.normal(size=(21, 4))
    assert np.isclose((O.gather(x, pos, 3) * ys).sum(), (O.combine(ys, pos, None, None, 7)[0] * x).sum())


def test_oracle_combine_backward_by_differences():
    rng = np.random.default_rng(1)
    _, _, pos = O.sort_tokens(rng.integers(-1, 4, (5, 2)), 4)
    ys, g, dy = rng.normal(size=(10, 3)), rng.normal(size=(5, 2)), rng.normal(size=(5, 3))
    dys, dg, _ = O.combine_backward(dy, ys, pos, g)
    f = lambda ys, g: (O.combine(ys, pos, g, None, 5)[0] * dy).sum()
    h = 1e-6
    for i in range(10):
        e = np.zeros(10)
        e[i] = h
        num = (f(ys, g + e.reshape(5, 2)) - f(ys, g - e.reshape(5, 2))) / (2 * h)
        assert abs(num - dg[i]) < 1e-8
        for j in range(3):
            e = np.zeros((10, 3))
            e[i, j] = h
            assert abs((f(ys + e, g) - f(ys - e, g)) / (2 * h) - dys[i, j]) < 1e-8


def test_oracle_q4_error_is_at_most_half_a_step():
    rng = np.random.default_rng(2)
    w = torch.from_numpy(rng.normal(size=(6, 256))).to(torch.bfloat16).double().numpy()
    for g in (32, 64, 128):
        c, s, v = O.q4_values(w, g)
        assert np.abs(c).max() <= 7
        # the largest weight is 7 s within a factor of 1 +- 2^-5: at most 0.25 s beyond 7 s
        assert (np.abs(w - v) <= 0.5 * np.repeat(s, g, -1) + 1e-300).all()
        exact = torch.from_numpy(v).to(torch.bfloat16).double().numpy()
        assert (exact == v).all()
        assert (np.frexp(s)[0] * 32 % 1 == 0).all()


# ---------------------------------------------------------------- one workspace for sorts of many sizes

def test_sort_workspace_never_shrinks(dm):
    """By the pairs, over every step in which they are cut into chunks, and by the experts."""
    for E in (1, 64, 256):
        last = 0
        around = {n * p * 1024 + i for n in (144, 148) for p in range(1, 70) for i in (-1024, 0, 1, 1024)}
        for R in sorted({0, 1, 1024, 1025, 2 ** 30} | around | {int(1.07 ** i) for i in range(300)}):
            size = dm.dmoe_sort_workspace_size(R, 1, E)
            assert size >= last, R
            last = size
    for R in (1, 1025, 151552, 151553, 524288, 2 ** 27):
        sizes = [dm.dmoe_sort_workspace_size(R, 8, E) for E in range(1, 257)]
        assert sizes == sorted(sizes)


def test_sort_of_a_smaller_batch_is_taken(dm, lib):
    """The workspace of 65536 x 8 pairs is not refused for 18944 x 8 (148 chunks, where the larger has 128):
    the call gets past the check of its size, to the launch, which has no device here."""
    if torch.cuda.is_available():
        pytest.skip("would run on addresses that are not there")
    n = dm.dmoe_sort_workspace_size(65536, 8, 256)
    for T in (18944, 18945, 1000, 8):
        assert lib.dmoe_sort_tokens(T, 8, 256, *[P(FAKE)] * 5, n, None) == 4


def test_binding_refuses_slots_cut_another_way(dm):
    """Gates or positions [T, k] beside rows of another number of tokens, which divides the slots as well."""
    T, k, d = 4, 2, 8
    bf = lambda n: torch.zeros(n, d, dtype=torch.bfloat16, device="meta")
    pos, gates = torch.zeros(T * k, dtype=torch.int32), torch.zeros(T, k)

    def refusal(f, *a):
        with pytest.raises(ValueError) as ei:
            f(*a)
        return str(ei.value)
    for n in (2, 8):
        assert refusal(dm._gates, gates, "gates", n, T * k // n, 0).startswith("gates: expected shape")
        two = pos.view(T, k)
        assert "slots" in refusal(dm.dmoe_gather_rows, bf(n), two, bf(8))
        assert "slots" in refusal(dm.dmoe_gather_rows_backward, bf(8), two, bf(n))
        assert "slots" in refusal(dm.dmoe_combine_rows, bf(8), two, None, None, bf(n))
        assert "slots" in refusal(dm.dmoe_combine_rows_backward, bf(n), None, two, None, bf(8), None)
    assert "device" in refusal(dm._gates, gates, "gates", T, k, 0)      # the right split, on the host
    assert dm._slots(T, pos.view(T, k)) == k and dm._slots(T, pos) == k and dm._gates(None, "g", T, k, 0) is None


def test_q4_hold_refusal(dm, lib):
    assert lib.dmoe_q4_set_debug_hold(-1) == 1
    dm.dmoe_q4_set_debug_hold(0)
