"""The norms around a block in 64 bits, with a bound of every element's error.

F = 2^-24 is a rounding in fp32. A row's sum is added up in at most 64 steps (32 elements of a thread,
5 exchanges, 16 warps), a sum over T tokens in at most T / 304 + 80 (a run of tokens, the groups of a
CTA, the CTAs in 32 strips): that many F of the sum of the sizes. A value from a handful of products
counts 16 F of the sum of its terms' sizes.
"""
import torch

F = 2.0 ** -24
ROW, FEW = 64 * F, 16 * F


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rounding(v, dtype):
    return half_step(dtype) * v.abs() + torch.finfo(dtype).smallest_normal * half_step(dtype)


def norm_residual(x, y, w_post, gate, w_pre, scale, eps, gate_tokens, dr=None, dn=None):
    """{name: (value, bound)} of r, n and, with dr or dn, dx, dy, dgate, dw_post, dw_pre (None where
    there is no such thing)."""
    dt, (T, d) = x.dtype, x.shape
    X = x.double()
    zero, one = torch.zeros_like(X), torch.ones_like(X)
    Y = zero if y is None else y.double()
    W = None if w_post is None else w_post.double()
    C = one if gate is None else gate.double()[torch.arange(T, device=x.device) // gate_tokens]
    eps = torch.tensor(eps, dtype=torch.float32).double().item()      # (the values that fp32 holds)
    scale = torch.tensor(scale, dtype=torch.float32).double().item()
    ry, e_ry = one[:, :1], 0.0
    if W is not None:
        ry = ((Y * Y).mean(1, keepdim=True) + eps) ** -0.5
        e_ry = ROW / 2 + FEW                                # relative
        C = C * W
    yh = Y * ry
    r = scale * X + C * yh
    size = (scale * X).abs() + (C * yh).abs()
    e_r = size * (e_ry + FEW)
    out = {"r": (r, e_r + rounding(r.abs() + e_r, dt)), "n": None}
    rr, e_rr = one[:, :1], 0.0
    if w_pre is not None:
        P = w_pre.double()
        ms = (r * r).mean(1, keepdim=True) + eps
        rr = ms ** -0.5
        e_rr = ((r.abs() + e_r) * e_r).mean(1, keepdim=True) / ms * 1.01 + ROW / 2 + FEW
        n = r * rr * P
        e_n = P.abs() * rr * (e_r + (r.abs() + e_r) * e_rr) * (1 + FEW) + FEW * n.abs()
        out["n"] = (n, e_n + rounding(n.abs() + e_n, dt))
    if dr is None and dn is None:
        return out
    DR = zero if dr is None else dr.double()
    A = zero if dn is None else dn.double() * w_pre.double()
    rh, size_rh = r * rr, size * rr
    mean = lambda v: v.mean(1, keepdim=True)
    m1 = mean(A * rh)
    q = DR + rr * (A - rh * m1)
    size_q = DR.abs() + rr * (A.abs() + size_rh * mean(A.abs() * size_rh))
    # rr, ry and rh (which holds both) stand in every term at most four times
    rel = 4 * (e_rr + e_ry) + ROW + 4 * FEW
    out["dx"] = _with(scale * q, abs(scale) * size_q * rel, dt)
    for k in ("dy", "dgate", "dw_post", "dw_pre"):
        out[k] = None
    if y is not None:
        v = q * C
        if W is not None:
            s2 = mean(size_q * C.abs() * yh.abs())
            out["dy"] = _with(ry * (v - yh * mean(v * yh)), ry * (size_q * C.abs() + yh.abs() * s2) * (rel + ROW), dt)
        else:
            out["dy"] = _with(v, size_q * C.abs() * rel, dt)
    tokens = rel + (T / 304 + 80) * F
    if gate is not None:
        p = yh if W is None else yh * W
        runs = torch.arange(T, device=x.device) // gate_tokens
        by = lambda v: torch.zeros(gate.shape, dtype=torch.float64, device=x.device).index_add_(0, runs, v)
        out["dgate"] = _with(by(q * p), by(size_q * p.abs() * tokens), dt)
    if W is not None:
        g = C / W
        out["dw_post"] = _with((q * g * yh).sum(0), (size_q * (g * yh).abs() * tokens).sum(0), torch.float32)
    if w_pre is not None:
        D = zero if dn is None else dn.double()
        out["dw_pre"] = _with((D * rh).sum(0), (D.abs() * size_rh * tokens).sum(0), torch.float32)
    return out


def _with(v, e, dtype):
    return v, e + rounding(v.abs() + e, dtype)


def check(name, got, want):
    v, b = want
    off = (got.double() - v).abs()
    bad = ~(off <= b)
    if bad.any():
        at = tuple(torch.nonzero(bad)[0].tolist())
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} off, first at {at}: "
                             f"{got[at].item()} for {v[at].item()}, bound {b[at].item()}")
