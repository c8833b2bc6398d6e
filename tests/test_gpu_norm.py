"""The norms around a block, with gate and residual, and their gradients against the formulas in 64 bits."""
import pytest
import torch

import paper_2605_30876_gb300 as dm
from tests import norm_oracle as O

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16, torch.float32]
# (tokens, width, tokens to a gate's row: 0 none): every number of threads to a row and both widths of
# a piece, gate rows that end inside a run, hold many runs, or are a token's
SHAPES = [(1, 1, 0), (3, 7, 1), (5, 8, 2), (33, 64, 33), (700, 100, 7), (257, 129, 64), (40, 1001, 0),
          (611, 2048, 32), (613, 2050, 700), (90, 4096, 48), (311, 8192, 5), (9, 10001, 4), (7, 16384, 7),
          (4000, 24, 1000), (20011, 16, 3),
          # rows of whole warps that are no power of two, several to a CTA and one
          (900, 1280, 7), (1201, 768, 100), (700, 2560, 33), (333, 5120, 50), (411, 2056, 4), (600, 644, 9)]


def rows(gen, n, d, dtype, size, pad=0):
    return torch.empty((n, d + pad), device="cuda").normal_(0, size, generator=gen).to(dtype)[:, :d]


def inputs(dtype, T, d, G, post=True, pre=True, seed=0, pad=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    vec = lambda: 1 + 0.3 * torch.empty(d, device="cuda").normal_(generator=gen)
    return dict(x=rows(gen, T, d, dtype, 2.0, pad), y=rows(gen, T, d, dtype, 0.7, pad),
                w_post=vec() if post else None,
                gate=rows(gen, -(-T // G), d, dtype, 0.5, pad) if G else None,
                w_pre=vec() if pre else None), (rows(gen, T, d, dtype, 1.0, pad), rows(gen, T, d, dtype, 1.0, pad))


def filled(t, pad=0):
    return None if t is None else torch.full((t.shape[0], t.shape[1] + pad), 7.0, dtype=t.dtype,
                                             device="cuda")[:, :t.shape[1]] if t.dim() == 2 else torch.full_like(t, 7.0)


def run(c, d_out, G, scale=1.0, eps=1e-6, pad=0, skip=()):
    """Everything by name, through the calls with out-tensors."""
    x = c["x"]
    T, d = x.shape
    r, n = filled(x, pad), filled(x, pad) if c["w_pre"] is not None else None
    stats = torch.empty((2, T), device="cuda")
    dm.dmoe_norm_residual(*c.values(), r, n, stats=stats, scale=scale, eps=eps, gate_tokens=G)
    dr, dn = d_out
    grads = {"dx": filled(x, pad), "dy": filled(c["y"], pad), "dgate": filled(c["gate"], pad),
             "dw_post": filled(c["w_post"]), "dw_pre": filled(c["w_pre"])}
    grads.update({k: None for k in skip})
    ws = dm.alloc_norm_workspace(T, d, G)
    ws.fill_(0xff)      # (NaNs: nothing is read that the call has not written)
    dm.dmoe_norm_residual_backward(*c.values(), stats, dr, dn if n is not None else None, *grads.values(),
                                   scale=scale, gate_tokens=G, workspace=ws)
    return dict(r=r, n=n, **grads)


def compare(c, d_out, G, got, scale=1.0, eps=1e-6):
    dn = d_out[1] if c["w_pre"] is not None else None
    want = O.norm_residual(*c.values(), scale, eps, G, d_out[0], dn)
    for k, v in got.items():
        if v is not None:
            O.check(k, v, want[k])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_both_directions(shape, dtype):
    T, d, G = shape
    c, d_out = inputs(dtype, T, d, G)
    compare(c, d_out, G, run(c, d_out, G))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("post,pre", [(False, True), (True, False), (False, False)])
def test_without_a_norm(post, pre, dtype):
    for T, d, G in ((50, 264, 8), (50, 263, 0)):
        c, d_out = inputs(dtype, T, d, G, post, pre, seed=1)
        compare(c, d_out, G, run(c, d_out, G, scale=0.7, eps=1e-3), scale=0.7, eps=1e-3)


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_and_gaps(dtype):
    for T, d, G, pad in ((70, 256, 9, 8), (70, 256, 9, 3), (1, 64, 1, 5)):
        c, d_out = inputs(dtype, T, d, G, pad=pad, seed=2)
        got = run(c, d_out, G, pad=pad)
        compare(c, d_out, G, got)
        for k in ("r", "n", "dx", "dy", "dgate"):
            gaps = torch.as_strided(got[k], (got[k].shape[0], pad), (d + pad, 1), d)
            assert (gaps == 7).all(), k


def test_off_16_bytes():
    c, d_out = inputs(torch.bfloat16, 20, 65, 4, seed=3)
    c = {k: v[:, 1:] if v is not None and v.dim() == 2 else None if v is None else v[:64].contiguous()
         for k, v in c.items()}
    d_out = [v[:, 1:] for v in d_out]
    compare(c, d_out, 4, run(c, d_out, 4))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_in_place(dtype):
    c, _ = inputs(dtype, 77, 200, 10)
    r, n = torch.empty_like(c["x"]), torch.empty_like(c["x"])
    dm.dmoe_norm_residual(*c.values(), r, n, gate_tokens=10)
    dm.dmoe_norm_residual(*c.values(), c["x"], c["y"], gate_tokens=10)
    assert torch.equal(r, c["x"]) and torch.equal(n, c["y"])


def test_without_a_block():
    """The norm before a first block alone: n, its gradient, and r not wanted."""
    c, (dr, dn) = inputs(torch.bfloat16, 50, 136, 0, post=False)
    n, stats = torch.empty_like(c["x"]), torch.empty((2, 50), device="cuda")
    dm.dmoe_norm_residual(c["x"], None, None, None, c["w_pre"], None, n, stats=stats)
    dx, dw = torch.empty_like(n), torch.empty_like(c["w_pre"])
    dm.dmoe_norm_residual_backward(c["x"], None, None, None, c["w_pre"], stats, None, dn, dx, None, None, None,
                                   dw, workspace=dm.alloc_norm_workspace(50, 136))
    want = O.norm_residual(c["x"], None, None, None, c["w_pre"], 1.0, 1e-6, 0, None, dn)
    for k, v in (("n", n), ("dx", dx), ("dw_pre", dw)):
        O.check(k, v, want[k])


@pytest.mark.parametrize("none", ["dr", "dn"])
def test_one_of_the_two_gradients(none):
    c, (dr, dn) = inputs(torch.float32, 90, 136, 4)
    d_out = (None, dn) if none == "dr" else (dr, None)
    got = run(c, d_out, 4)
    want = O.norm_residual(*c.values(), 1.0, 1e-6, 4, *d_out)
    for k in ("dx", "dy", "dgate", "dw_post", "dw_pre"):
        O.check(k, got[k], want[k])


@pytest.mark.parametrize("d", [64, 2048, 4096])
def test_some_of_the_gradients(d):
    c, d_out = inputs(torch.bfloat16, 20000 // (d // 64) + 3000, d, 16)     # (runs over several gate rows)
    whole = run(c, d_out, 16)
    names = ("dx", "dy", "dgate", "dw_post", "dw_pre")
    for keep in names:
        got = run(c, d_out, 16, skip=[k for k in names if k != keep])
        assert torch.equal(got[keep], whole[keep]), keep


def test_no_tokens():
    c, d_out = inputs(torch.bfloat16, 0, 64, 4)
    got = run(c, d_out, 4)
    assert (got["dw_post"] == 0).all() and (got["dw_pre"] == 0).all() and got["r"].shape == (0, 64)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_bad_row_stays_in_its_row(bad):
    c, d_out = inputs(torch.bfloat16, 100, 72, 10)
    want = run(c, d_out, 10)
    c["y"][33] = bad
    d_out[0][50] = bad
    got = run(c, d_out, 10)
    keep = torch.ones(100, dtype=torch.bool, device="cuda")
    keep[33] = keep[50] = False
    for k in ("r", "n", "dx", "dy"):
        assert torch.equal(got[k][keep], want[k][keep]), k
    rows = torch.tensor([i for i in range(10) if i not in (3, 5)], device="cuda")
    assert torch.equal(got["dgate"][rows], want["dgate"][rows])


def test_rows_of_zeros():
    c, d_out = inputs(torch.float32, 20, 72, 5)
    c["x"][3:9] = 0
    c["y"][5:12] = 0
    compare(c, d_out, 5, run(c, d_out, 5))


def test_rows_beyond_32_bits():
    T, d = 270001, 8192
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, y = (torch.empty((T, d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    w = torch.rand(d, device="cuda", generator=gen) + 0.5
    gate = torch.rand((27, d), device="cuda", generator=gen).to(torch.bfloat16)
    r, n, stats = torch.empty_like(x), torch.empty_like(x), torch.empty((2, T), device="cuda")
    dm.dmoe_norm_residual(x, y, w, gate, w, r, n, stats=stats, gate_tokens=10001)
    dx, dy = torch.empty_like(x), torch.empty_like(x)
    dm.dmoe_norm_residual_backward(x, y, w, gate, w, stats, y, x, dx, dy, None, None, None, gate_tokens=10001)
    part = slice(26 * 10001, T)
    want = O.norm_residual(x[part], y[part], w, gate[26:], w, 1.0, 1e-6, 10001, y[part], x[part])
    for k, v in (("r", r), ("n", n), ("dx", dx), ("dy", dy)):
        O.check(k, v[part], want[k])


def test_same_call_same_bits_on_any_stream_and_replayed():
    c, d_out = inputs(torch.bfloat16, 1000, 520, 48)
    want = run(c, d_out, 48)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = run(c, d_out, 48)
    torch.cuda.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in want)
    x = c["x"]
    outs = [torch.empty_like(t) for t in (x, x, x, c["y"], c["gate"], c["w_post"], c["w_pre"])]
    stats, ws = torch.empty((2, 1000), device="cuda"), dm.alloc_norm_workspace(1000, 520, 48)

    def both():
        dm.dmoe_norm_residual(*c.values(), *outs[:2], stats=stats, gate_tokens=48)
        dm.dmoe_norm_residual_backward(*c.values(), stats, *d_out, *outs[2:], gate_tokens=48, workspace=ws)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for t in outs:
        t.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want.values()))
