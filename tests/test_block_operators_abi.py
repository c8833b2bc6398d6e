"""The experts' feed-forward block and the norms around it without a GPU: sizes, and the refusals that
come before any launch."""
import ctypes

import pytest
import torch

P = ctypes.c_void_p
FAKE = 1 << 40     # aligned, never dereferenced: the checks return first


@pytest.fixture(scope="module")
def dm():
    import paper_2605_30876_gb300 as dm
    return dm


def at(name, names):
    return FAKE + 65536 * names.index(name)


FFN = ("x", "offsets", "ids", "w_gate", "w_up", "w_down", "pre", "h", "y")
BACK = ("dy", "x", "offsets", "w_gate", "w_up", "w_down", "pre", "h", "dpre", "dx", "dw_gate", "dw_up", "dw_down")


def ffn(dm, desc=(0, 4, 64, 64), R=8, n=4, ldx=64, ldy=64, **change):
    p = {k: at(k, FFN) for k in FFN}
    p.update(change)
    v = {k: P(a) if a else None for k, a in p.items()}
    d = dm.ExpertDesc(*desc) if desc else None
    return dm._lib.dmoe_expert_ffn(ctypes.byref(d) if d else None, R, n, v["x"], ldx, v["offsets"], v["ids"],
                                   v["w_gate"], v["w_up"], v["w_down"], v["pre"], v["h"], v["y"], ldy, 0, None)


def ffn_backward(dm, desc=(0, 4, 64, 64), R=8, lddy=64, ldx=64, lddx=64, **change):
    p = {k: at(k, BACK) for k in BACK}
    p.update(change)
    v = {k: P(a) if a else None for k, a in p.items()}
    d = dm.ExpertDesc(*desc) if desc else None
    return dm._lib.dmoe_expert_ffn_backward(
        ctypes.byref(d) if d else None, R, v["dy"], lddy, v["x"], ldx, v["offsets"], v["w_gate"], v["w_up"],
        v["w_down"], v["pre"], v["h"], v["dpre"], v["dx"], lddx, v["dw_gate"], v["dw_up"], v["dw_down"], 0, None)


DESCS = [((2, 4, 64, 64), 1), ((-1, 4, 64, 64), 1), ((0, 0, 64, 64), 1), ((0, 4, 0, 64), 1),
         ((0, 4, 64, 0), 1), ((0, 513, 64, 64), 2), ((0, 4, 60, 64), 2), ((0, 4, 64, 4), 2),
         ((0, 4, 16392, 64), 2), ((0, 4, 64, 16392), 2)]


@pytest.mark.parametrize("desc,status", DESCS)
def test_expert_sizes(dm, desc, status):
    assert ffn(dm, desc, n=1, ids=None) == status or (desc[1] == 0 and status == 1)
    assert ffn_backward(dm, desc) == status


def test_expert_refusals(dm):
    assert ffn(dm, None) == 1 and ffn_backward(dm, None) == 1
    assert ffn(dm, R=0, **dict.fromkeys(FFN[3:])) == 0                  # no rows: nothing to do
    assert ffn(dm, R=-1) == 1 and ffn_backward(dm, R=-1) == 1
    assert ffn(dm, R=2 ** 30 + 1) == 2 and ffn_backward(dm, R=2 ** 30 + 1) == 2
    assert ffn(dm, n=0) == 1 and ffn(dm, n=513) == 2
    assert ffn(dm, n=5, ids=None) == 1                                   # more groups than experts
    assert ffn(dm, offsets=None) == 1 and ffn_backward(dm, offsets=None) == 1   # groups without offsets
    # units, whatever the offsets hold, are counted in 32 bits
    assert ffn(dm, (0, 512, 16384, 16384), R=2 ** 30, n=512, ldx=16384, ldy=16384) == 2
    for k in ("x", "w_gate", "w_up", "w_down", "h", "y"):
        assert ffn(dm, **{k: None}) == 1, k
    for k in FFN:
        assert ffn(dm, **{k: at(k, FFN) + 8}) == 1, k                    # off 16 bytes
    for ld in (56, 68, 0, -64):
        assert ffn(dm, ldx=ld) == 1 and ffn(dm, ldy=ld) == 1
    x = at("x", FFN)
    assert ffn(dm, y=x) == 1 and ffn(dm, h=x) == 1 and ffn(dm, pre=x) == 1
    assert ffn(dm, h=at("y", FFN)) == 1 and ffn(dm, pre=at("h", FFN)) == 1


def test_expert_backward_refusals(dm):
    for k in ("dy", "x", "w_gate", "w_up", "w_down", "pre", "h", "dpre"):
        assert ffn_backward(dm, **{k: None}) == 1, k
    for k in BACK:
        assert ffn_backward(dm, **{k: at(k, BACK) + 8}) == 1, k
    assert ffn_backward(dm, dx=None, dw_gate=None, dw_up=None, dw_down=None) == 1
    assert ffn_backward(dm, dw_gate=None) == 1 and ffn_backward(dm, dw_up=None) == 1
    assert ffn_backward(dm, dw_up=at("dw_gate", BACK)) == 1
    for ld in (56, 68):
        assert ffn_backward(dm, lddy=ld) == 1 and ffn_backward(dm, ldx=ld) == 1
        assert ffn_backward(dm, lddx=ld) == 1
    assert ffn_backward(dm, dpre=at("pre", BACK)) == 1
    assert ffn_backward(dm, dx=at("dy", BACK)) == 1 and ffn_backward(dm, dx=at("x", BACK)) == 1


def test_expert_outputs_that_overlap(dm):
    for k in ("h", "dy", "x", "dx", "pre"):
        assert ffn_backward(dm, dpre=at(k, BACK)) == 1, k
    for a, b in (("dw_gate", "dw_up"), ("dw_gate", "dw_down"), ("dw_up", "dw_down")):
        assert ffn_backward(dm, **{a: at(b, BACK)}) == 1, (a, b)


def test_expert_hold(dm):
    assert dm._lib.dmoe_expert_set_debug_hold(-1) == 1
    assert dm._lib.dmoe_expert_set_debug_hold(0) == 0


def test_expert_binding_refusals(dm):
    """What the binding refuses before it asks the library."""
    t = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)
    w = (t(2, 16, 8), t(2, 16, 8), t(2, 8, 16))
    with pytest.raises(TypeError):
        dm.dmoe_expert_ffn(t(4, 8, dtype=torch.float32), None, *w, t(4, 16), t(4, 8))
    with pytest.raises(TypeError):
        dm.dmoe_expert_ffn(t(4, 8, 1), None, *w, t(4, 16), t(4, 8))
    with pytest.raises(TypeError):
        dm.dmoe_expert_ffn(t(4, 8), None, w[0][0], w[1], w[2], t(4, 16), t(4, 8))
    with pytest.raises(ValueError):
        dm.dmoe_expert_ffn(t(4, 8), None, w[0], w[1], t(2, 16, 8), t(4, 16), t(4, 8))
    with pytest.raises(ValueError):                                       # not on a GPU
        dm.dmoe_expert_ffn(t(4, 8), None, *w, t(4, 16), t(4, 8))


NORM = ("x", "y", "w_post", "gate", "w_pre", "r", "n", "stats")
NORM_BACK = ("x", "y", "w_post", "gate", "w_pre", "stats", "dr", "dn", "dx", "dy", "dgate", "dw_post", "dw_pre", "ws")
NDESC = dict(dtype=0, d=64, T=8, G=2, scale=1.0, eps=1e-6)


def ndesc(dm, change):
    v = dict(NDESC, **change)
    return dm.NormDesc(v["dtype"], v["d"], v["T"], v["G"], v["scale"], v["eps"])


def norm(dm, desc={}, ld={}, **change):
    p = {k: at(k, NORM) for k in NORM}
    p.update(change)
    v = {k: P(a) if a else None for k, a in p.items()}
    s = lambda k: ld.get(k, 64)
    return dm._lib.dmoe_norm_residual(
        ctypes.byref(ndesc(dm, desc)), v["x"], s("x"), v["y"], s("y"), v["w_post"], v["gate"], s("gate"),
        v["w_pre"], v["r"], s("r"), v["n"], s("n"), v["stats"], None)


def norm_backward(dm, desc={}, ld={}, nbytes=1 << 40, **change):
    p = {k: at(k, NORM_BACK) for k in NORM_BACK}
    p.update(change)
    v = {k: P(a) if a else None for k, a in p.items()}
    s = lambda k: ld.get(k, 64)
    return dm._lib.dmoe_norm_residual_backward(
        ctypes.byref(ndesc(dm, desc)), v["x"], s("x"), v["y"], s("y"), v["w_post"], v["gate"], s("gate"),
        v["w_pre"], v["stats"], v["dr"], s("dr"), v["dn"], s("dn"), v["dx"], s("dx"), v["dy"], s("dy"),
        v["dgate"], s("dgate"), v["dw_post"], v["dw_pre"], v["ws"], nbytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), 1), (dict(dtype=-1), 1), (dict(d=0), 1), (dict(T=-1), 1), (dict(G=-1), 1),
    (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(d=16385), 2), (dict(T=2 ** 30 + 1), 2)])
def test_norm_sizes(dm, change, status):
    assert norm(dm, change) == status and norm_backward(dm, change) == status
    n = ctypes.c_size_t(0)
    assert dm._lib.dmoe_norm_workspace_size(ctypes.byref(ndesc(dm, change)), ctypes.byref(n)) == status


def test_norm_workspace(dm):
    size = dm.dmoe_norm_workspace_size
    assert size(0, 64) == 0
    assert 0 < size(1, 64) <= size(1, 64, 1) <= size(100, 64, 1) <= size(100, 128, 1) <= size(10 ** 6, 128, 1)
    assert size(2 ** 30, 2048, 32) == size(10 ** 6, 2048, 1)
    assert dm._lib.dmoe_norm_workspace_size(ctypes.byref(ndesc(dm, {})), None) == 1


def test_norm_refusals(dm):
    assert norm(dm, dict(T=0), **dict.fromkeys(NORM)) == 0
    assert dm._lib.dmoe_norm_residual(None, *[None, 0] * 2, None, None, 0, None, None, 0, None, 0, None, None) == 1
    assert norm(dm, x=None) == 1
    assert norm(dm, y=None) == 1 and norm(dm, y=None, gate=None) == 1 and norm(dm, y=None, w_post=None) == 1
    assert norm(dm, n=None) == 1 and norm(dm, w_pre=None) == 1          # one without the other
    assert norm(dm, r=None, n=None, w_pre=None) == 1                     # nothing wanted
    assert norm(dm, dict(G=0)) == 1                                      # a gate for how many tokens?
    for k in ("x", "y", "gate", "r", "n"):
        assert norm(dm, **{k: at(k, NORM) + 1}) == 1, k
        assert norm(dm, dict(dtype=2), **{k: at(k, NORM) + 2}) == 1, k
        assert norm(dm, ld={k: 63}) == 1, k
    for k in ("w_post", "w_pre", "stats"):
        assert norm(dm, **{k: at(k, NORM) + 4}) == 1, k
    # in place only r over x and n over y, with the same strides
    x, y, g = (at(k, NORM) for k in ("x", "y", "gate"))
    assert norm(dm, r=y) == 1 and norm(dm, n=x) == 1 and norm(dm, r=g) == 1 and norm(dm, n=g) == 1
    assert norm(dm, n=at("r", NORM)) == 1
    assert norm(dm, ld=dict(x=2 ** 30)) == 2 and norm_backward(dm, ld=dict(dx=2 ** 30)) == 2
    assert norm(dm, r=x, ld=dict(x=72)) == 1 and norm(dm, n=y, ld=dict(n=72)) == 1


def test_norm_backward_refusals(dm):
    outs = ("dx", "dy", "dgate", "dw_post", "dw_pre")
    assert norm_backward(dm, **dict.fromkeys(outs)) == 1
    assert norm_backward(dm, dict(T=0), **dict.fromkeys(outs)) == 1
    assert norm_backward(dm, x=None) == 1 and norm_backward(dm, stats=None) == 1
    assert norm_backward(dm, dr=None, dn=None) == 1
    assert norm_backward(dm, w_pre=None, dw_pre=None) == 1               # dn without w_pre
    assert norm_backward(dm, w_pre=None, dn=None) == 1                   # dw_pre without w_pre
    assert norm_backward(dm, w_post=None) == 1 and norm_backward(dm, gate=None) == 1
    assert norm_backward(dm, y=None, gate=None, w_post=None, dgate=None, dw_post=None) == 1
    for k in ("x", "y", "gate", "dr", "dn", "dx", "dy", "dgate"):
        assert norm_backward(dm, **{k: at(k, NORM_BACK) + 1}) == 1, k
        assert norm_backward(dm, ld={k: 63}) == 1, k
    for k in ("w_post", "w_pre", "stats", "dw_post", "dw_pre", "ws"):
        assert norm_backward(dm, **{k: at(k, NORM_BACK) + 4}) == 1, k
    assert norm_backward(dm, ws=None) == 1
    need = dm.dmoe_norm_workspace_size(8, 64, 2)
    assert norm_backward(dm, nbytes=need - 1) == 3
    assert norm_backward(dm, dw_post=at("dw_pre", NORM_BACK)) == 1
    for k in ("dx", "dy", "dgate"):
        for o in ("x", "y", "gate", "dr", "dn"):
            assert norm_backward(dm, **{k: at(o, NORM_BACK)}) == 1, (k, o)
    assert norm_backward(dm, dy=at("dx", NORM_BACK)) == 1


def test_norm_binding_refusals(dm):
    t = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)
    with pytest.raises(TypeError):
        dm.dmoe_norm_residual(t(4, 8, dtype=torch.int32), None, None, None, None, t(4, 8), None)
    with pytest.raises(ValueError):                                       # not on a GPU
        dm.dmoe_norm_residual(t(4, 8), None, None, None, None, t(4, 8), None)
