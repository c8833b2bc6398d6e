"""The experts' feed-forward block in 64 bits, group by group, with a bound of every element's error.

Bounds count, for sums of K products in fp32, K * 2^-23 of the sum of the products' sizes (the tensor
cores may cut the addends instead of rounding them), half a step of the type for every rounding to it
(and half a subnormal step), and 2^-20 of a value for the exponential, the quotient and the few
products around it in fp32.
"""
import torch

FN = 2.0 ** -20


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def acc(K):
    return K * 2.0 ** -23


def rounding(v, dtype):
    return half_step(dtype) * v.abs() + tiny(dtype)


def groups(offsets, R):
    """[(first, last)] of every group, cut to [0, R]."""
    o = [min(max(int(v), 0), R) for v in offsets]
    return [(a, max(a, b)) for a, b in zip(o, o[1:])]


def forward(x, offsets, w_gate, w_up, w_down, ids=None):
    """{name: (value, bound)} of g, u, h, y in float64 on x's device; NaN in rows of no group."""
    dt, (R, d), I = x.dtype, x.shape, w_gate.shape[1]
    nan = lambda n: torch.full((R, n), float("nan"), dtype=torch.float64, device=x.device)
    out = {n: (nan(k), nan(k)) for n, k in (("g", I), ("u", I), ("h", I), ("y", d))}
    for g, (lo, hi) in enumerate(groups(offsets, R)):
        e = g if ids is None else int(ids[g])
        if lo == hi or not 0 <= e < w_gate.shape[0]:
            continue
        X = x[lo:hi].double()
        G, U, D = (w[e].double() for w in (w_gate, w_up, w_down))
        g_, u_ = X @ G.t(), X @ U.t()
        eg, eu = acc(d) * (X.abs() @ G.abs().t()), acc(d) * (X.abs() @ U.abs().t())
        s = torch.sigmoid(g_)
        h = g_ * s * u_
        # |silu'| <= 1.1, |silu''| <= 0.5
        eh = ((1.1 * eg + eg * eg) * (u_.abs() + eu) + (g_ * s).abs() * eu + FN * h.abs())
        ehr = eh + rounding(h.abs() + eh, dt)
        y = h @ D.t()
        ey = ehr @ D.abs().t() + acc(I) * ((h.abs() + ehr) @ D.abs().t())
        for n, v, b in (("g", g_, eg), ("u", u_, eu), ("h", h, eh), ("y", y, ey)):
            out[n][0][lo:hi] = v
            out[n][1][lo:hi] = b + rounding(v.abs() + b, dt)
    return out


def backward(dy, x, offsets, w_gate, w_up, w_down, pre, h, off=None):
    """The same of dpre (gate, up), dx and the three weights' gradients, from pre and h as given; off: how
    far the kernel's g, u and h may be from those, rows by rows."""
    dt, (R, d), (E, I) = x.dtype, x.shape, w_gate.shape[:2]
    nan = lambda n: torch.full((R, n), float("nan"), dtype=torch.float64, device=x.device)
    out = {n: (nan(k), nan(k)) for n, k in (("dg", I), ("du", I), ("dx", d))}
    for n, w in (("dw_gate", w_gate), ("dw_up", w_up), ("dw_down", w_down)):
        out[n] = tuple(torch.zeros(w.shape, dtype=torch.float64, device=x.device) for _ in range(2))
    for e, (lo, hi) in enumerate(groups(offsets, R)):
        if lo == hi:
            continue
        n = hi - lo
        X, DY, H = x[lo:hi].double(), dy[lo:hi].double(), h[lo:hi].double()
        g, u = pre[lo:hi, 0].double(), pre[lo:hi, 1].double()
        G, U, D = (w[e].double() for w in (w_gate, w_up, w_down))
        dh, edh = DY @ D, acc(d) * (DY.abs() @ D.abs())
        s = torch.sigmoid(g)
        fg, fu = u * s * (1 + g * (1 - s)), g * s
        # (1 + g (1 - s) can cancel: its parts count)
        part = u.abs() * s * (1 + g.abs() * (1 - s))
        dg, du = dh * fg, dh * fu
        edg = edh * (fg.abs() + FN * part) + FN * dh.abs() * part
        edu = edh * fu.abs() * (1 + FN) + FN * du.abs()
        eh = torch.zeros_like(H)
        if off is not None:      # |s'| = |(silu)'| <= 1.1, |silu''| <= 0.5
            og, ou, eh = (o[lo:hi] for o in off)
            edg = edg + (dh.abs() + edh) * (1.1 * ou + 0.5 * og * (u.abs() + ou))
            edu = edu + (dh.abs() + edh) * 1.1 * og
        rdg, rdu = edg + rounding(dg.abs() + edg, dt), edu + rounding(du.abs() + edu, dt)
        dx = dg @ G + du @ U
        size = (dg.abs() + rdg) @ G.abs() + (du.abs() + rdu) @ U.abs()
        edx = rdg @ G.abs() + rdu @ U.abs() + acc(2 * I) * size
        for name, v, b in (("dg", dg, edg), ("du", du, edu), ("dx", dx, edx)):
            out[name][0][lo:hi] = v
            out[name][1][lo:hi] = b + rounding(v.abs() + b, dt)
        none, zero = torch.zeros_like(X), torch.zeros_like(DY)
        for name, a, ea, b, eb in (("dw_gate", dg, rdg, X, none), ("dw_up", du, rdu, X, none),
                                   ("dw_down", DY, zero, H, eh)):
            v = a.t() @ b
            size = (a.abs() + ea).t() @ (b.abs() + eb)
            err = ea.t() @ (b.abs() + eb) + a.abs().t() @ eb + acc(n) * size
            out[name][0][e] = v
            out[name][1][e] = err + rounding(v.abs() + err, dt)
    return out


def check(name, got, want):
    """got against (value, bound); rows whose value is NaN are in no group and are not looked at."""
    v, b = want
    off = (got.double() - v).abs()
    bad = ~(off <= b) & ~torch.isnan(v)
    if bad.any():
        at = tuple(torch.nonzero(bad)[0].tolist())
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} off, first at {at}: "
                             f"{got[at].item()} for {v[at].item()}, bound {b[at].item()}")
