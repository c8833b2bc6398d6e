"""A MoE block's experts and norms for training and serving, as cases that can be timed and compared.

Two operators, each through the package's public entry points (``own = True``) or in its plain form
of elementary torch operations (``own = False``):

* ``ffn``   the gated feed-forward block of the experts on rows sorted by expert,
            y[r] = Wd_e (silu(Wg_e x[r]) * (Wu_e x[r])) for the rows of every expert e
            (``dmoe_expert_ffn``); a training pass computes the gradients by x and by the three
            weights, too (``dmoe_expert_ffn_backward``). One expert of all rows is a dense block.
            Rows behind the last expert's (slots without an expert) have zeros in y and in dx.
* ``norm``  what stands around such a block: the norm of its output, gated, added to the scaled
            residual, and the norm before the next block,
                p = y * rstd(y) * w_post,  r = scale * x + gate * p,  n = r * rstd(r) * w_pre,
                rstd(v) = 1 / sqrt(mean(v^2) + eps)
            in one pass (``dmoe_norm_residual``), and its gradients by x, y, the gate and both
            weights (``dmoe_norm_residual_backward``). A row of the gate holds for ``gate`` tokens
            (0: there is no gate).

Sizes: ``R`` rows, ``E`` experts of which ``U`` have rows, width ``d``, inner width ``I``; for the
norms ``T`` tokens.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_EPS = 1e-6


def _ffn(name, **kw):
    return dict(dict(name=name, op="ffn", train=False, E=256, d=2048, I=512, dtype="bf16", masked=0.0), **kw)


def _norm(name, **kw):
    return dict(dict(name=name, op="norm", train=False, d=2048, dtype="bf16", gate=0, post=True, pre=True,
                     scale=1.0), **kw)


def listed():
    return [
        # one token through its eight experts: what a single user waits for
        _ffn("ffn_token", R=8, U=8),
        # a decoding block under block top-k: 32 rows for each of eight experts
        _ffn("ffn_block", R=256, U=8),
        # a prompt of 2048 tokens, eight experts each, through all of them
        _ffn("ffn_prompt", R=16384, U=256),
        # a dense block of its own sizes, not whole tiles, on a ragged batch in half precision
        _ffn("ffn_dense", R=2031, U=1, E=1, d=2048, I=2744, dtype="fp16"),
        # a training micro-batch of 8192 tokens, eight experts each, a tenth of the slots masked
        _ffn("ffn_train", train=True, R=65536, U=256, masked=0.1),
        # a small model's training step: odd widths, few rows for some experts and none for others
        _ffn("ffn_train_odd", train=True, R=6186, U=41, E=48, d=1000, I=344, dtype="fp16", masked=0.2),
        # between two blocks of a decoding step of one block of 32 tokens: all latency
        _norm("norm_step", T=32, gate=32),
        # between two blocks of a long prompt, a learned gate per channel
        _norm("norm_prompt", T=16384, gate=16384),
        # a wide model, a gate for every sequence of 700 tokens, half precision
        _norm("norm_wide", T=4197, d=8192, gate=700, dtype="fp16", scale=0.5),
        # a training micro-batch, a gate for every diffusion block of 32 tokens
        _norm("norm_train", train=True, T=16384, gate=32),
        # a ragged batch of odd width in single precision, gates that end inside the batch
        _norm("norm_train_odd", train=True, T=2111, d=1001, gate=48, dtype="fp32", scale=0.7),
        # the norm before the first block alone, with its gradients (no norm after, no gate)
        _norm("norm_train_plain", train=True, T=8192, d=4096, post=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.5:
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        d = _log(rng, 64, 8192)
        if rng.random() < 0.7:
            d = (d + 7) // 8 * 8
        T = min(_log(rng, 1, 65536), 16384 * 2048 // (d * (2 if dtype == "fp32" else 1)))
        gate = rng.choice([0, 1, _log(rng, 1, 4096), _log(rng, 8, 512), T])
        return dict(op="norm", train=rng.random() < 0.5, T=T, d=d, dtype=dtype, gate=gate,
                    post=rng.random() < 0.7, pre=rng.random() < 0.8, scale=rng.choice([1.0, 0.5, 1.25]))
    train = rng.random() < 0.5
    d, I = 8 * _log(rng, 8, 512), 8 * _log(rng, 8, 512)
    E = 1 if rng.random() < 0.25 else min(_log(rng, 1, 256), max(1, 2 ** 28 // (d * I)))
    R = min(_log(rng, 1, 65536), max(1, 2 ** 36 // (d * I)))
    U = min(E, R, _log(rng, max(1, E // 4), E))
    return dict(op="ffn", train=train, R=R, U=U, E=E, d=d, I=I, dtype=rng.choice(["bf16", "bf16", "fp16"]),
                masked=rng.choice([0.0, 0.0, 0.05, 0.3]) if R > 4 * U else 0.0)


# ------------------------------------------------------------------------------ inputs

def _randn(gen, shape, dtype, size=1.0):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, size, generator=gen)


def _counts(gen, case):
    """int64 [E]: rows of every expert, some far more popular than others; U of them have rows."""
    E, U = case["E"], case["U"]
    rows = max(U, int(case["R"] * (1 - case["masked"])))
    pop = torch.arange(1, U + 1, device="cuda", dtype=torch.float32) ** -0.5
    pick = torch.multinomial(pop, rows - U, replacement=True, generator=gen) if rows > U else None
    used = torch.ones(U, dtype=torch.int64, device="cuda")
    if pick is not None:
        used = used + torch.bincount(pick, minlength=U)
    counts = torch.zeros(E, dtype=torch.int64, device="cuda")
    counts[torch.randperm(E, generator=gen, device="cuda")[:U]] = used
    return counts


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, d = _DTYPES[case["dtype"]], case["d"]
    if case["op"] == "norm":
        T, G = case["T"], case["gate"]
        s = {"x": _randn(gen, (T, d), dt, 2.0), "y": _randn(gen, (T, d), dt, 0.7),
             "w_post": 1 + 0.2 * _randn(gen, (d,), torch.float32) if case["post"] else None,
             "w_pre": 1 + 0.2 * _randn(gen, (d,), torch.float32) if case["pre"] else None,
             "gate": (0.5 + 0.3 * _randn(gen, (-(-T // G), d), torch.float32)).to(dt) if G else None}
        if case["train"]:
            s["dr"] = _randn(gen, (T, d), dt)
            s["dn"] = _randn(gen, (T, d), dt) if case["pre"] else None
        return s
    R, E, I = case["R"], case["E"], case["I"]
    counts = _counts(gen, case)
    s = {"offsets": torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32),
         "x": _randn(gen, (R, d), dt),
         "w_gate": _randn(gen, (E, I, d), dt, d ** -0.5),
         "w_up": _randn(gen, (E, I, d), dt, d ** -0.5),
         "w_down": _randn(gen, (E, d, I), dt, I ** -0.5)}
    if case["train"]:
        s["dy"] = _randn(gen, (R, d), dt)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    like = torch.empty_like
    if case["op"] == "norm":
        # outputs and what a training program keeps between its forward and its backward pass
        s["r"], s["n"] = like(s["x"]), like(s["x"]) if case["pre"] else None
        s["stats"], s["ws"] = None, None
        if case["train"]:
            s["stats"] = torch.empty((2, case["T"]), dtype=torch.float32, device="cuda")
            s["grads"] = [None if t is None else like(t)
                          for t in (s["x"], s["y"], s["gate"], s["w_post"], s["w_pre"])]
        return s
    R, I = case["R"], case["I"]
    # where each expert's rows begin, on the host: the plain form goes through the experts there
    s["first"] = s["offsets"].tolist()
    new = lambda *shape: torch.empty(shape, dtype=s["x"].dtype, device="cuda")
    s["h"], s["y"] = new(R, I), like(s["x"])
    s["pre"] = None
    if case["train"]:
        s["pre"], s["dpre"] = new(R, 2, I), new(R, 2, I)
        s["grads"] = [like(s[n]) for n in ("x", "w_gate", "w_up", "w_down")]
    return s


# ------------------------------------------------------------------------------ one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2605_30876_gb300 as dmoe
    case = s["case"]
    if case["op"] == "norm":
        if case["train"] and s["ws"] is None:   # once for a program's sizes
            s["ws"] = dmoe.alloc_norm_workspace(case["T"], case["d"], case["gate"], "cuda")
        a = (s["x"], s["y"], s["w_post"], s["gate"], s["w_pre"])
        dmoe.dmoe_norm_residual(*a, s["r"], s["n"], stats=s["stats"], scale=case["scale"], eps=_EPS,
                                gate_tokens=case["gate"])
        if case["train"]:
            dmoe.dmoe_norm_residual_backward(*a, s["stats"], s["dr"], s["dn"], *s["grads"],
                                             scale=case["scale"], gate_tokens=case["gate"],
                                             workspace=s["ws"])
            return [s["r"], s["n"], *s["grads"]]
        return [s["r"], s["n"]]
    w = (s["w_gate"], s["w_up"], s["w_down"])
    dmoe.dmoe_expert_ffn(s["x"], s["offsets"], *w, s["h"], s["y"], pre=s["pre"], zero_rest=True)
    if not case["train"]:
        return s["y"]
    dmoe.dmoe_expert_ffn_backward(s["dy"], s["x"], s["offsets"], *w, s["pre"], s["h"], s["dpre"],
                                  *s["grads"], zero_rest=True)
    return [s["y"], *s["grads"]]


def _run_plain(s):
    return _plain_norm(s) if s["case"]["op"] == "norm" else _plain_ffn(s)


def _rstd(v):
    return 1 / torch.sqrt((v * v).mean(1, keepdim=True) + _EPS)


def _by_gate(v, G):
    """Sums of v's rows over runs of G of them."""
    T, d = v.shape
    n = -(-T // G)
    full = torch.zeros((n * G, d), device=v.device)
    full[:T] = v
    return full.view(n, G, d).sum(1)


def _plain_norm(s):
    case, dt = s["case"], s["x"].dtype
    G, T = case["gate"], case["T"]
    x, y = s["x"].float(), s["y"].float()
    p = y
    if case["post"]:
        ry = _rstd(y)
        yhat = y * ry
        p = yhat * s["w_post"]
    gate = s["gate"].float().repeat_interleave(G, 0)[:T] if G else None
    r = case["scale"] * x + (gate * p if G else p)
    n = None
    if case["pre"]:
        rr = _rstd(r)
        rhat = r * rr
        n = (rhat * s["w_pre"]).to(dt)
    if not case["train"]:
        return [r.to(dt), n]
    g = s["dr"].float()
    dw_pre = dw_post = dgate = None
    if case["pre"]:
        dn = s["dn"].float()
        dw_pre = (dn * rhat).sum(0)
        dn = dn * s["w_pre"]
        g = g + rr * (dn - rhat * (dn * rhat).mean(1, keepdim=True))
    dy = g
    if G:
        dgate = _by_gate(g * p, G).to(dt)
        dy = g * gate
    if case["post"]:
        dw_post = (dy * yhat).sum(0)
        dy = dy * s["w_post"]
        dy = ry * (dy - yhat * (dy * yhat).mean(1, keepdim=True))
    return [r.to(dt), n, (case["scale"] * g).to(dt), dy.to(dt), dgate, dw_post, dw_pre]


def _plain_ffn(s):
    case = s["case"]
    first = s["first"]
    y = torch.zeros_like(s["x"])
    if case["train"]:
        dx = torch.zeros_like(s["x"])
        dws = [torch.zeros_like(s[n]) for n in ("w_gate", "w_up", "w_down")]
    for e in range(case["E"]):
        lo, hi = first[e], first[e + 1]
        if lo == hi:
            continue
        x = s["x"][lo:hi].float()
        wg, wu, wd = (s[n][e].float() for n in ("w_gate", "w_up", "w_down"))
        g, u = x @ wg.t(), x @ wu.t()
        sig = 1 / (1 + torch.exp(-g))
        h = g * sig * u
        y[lo:hi] = (h @ wd.t()).to(y.dtype)
        if case["train"]:
            dy = s["dy"][lo:hi].float()
            dh = dy @ wd
            dg, du = dh * u * sig * (1 + g * (1 - sig)), dh * g * sig
            dx[lo:hi] = (dg @ wg + du @ wu).to(dx.dtype)
            for dw, v in zip(dws, (dg.t() @ x, du.t() @ x, dy.t() @ h)):
                dw[e] = v.to(dw.dtype)
    return [y, dx, *dws] if case["train"] else y


# ------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    return _exact_norm(case, s) if case["op"] == "norm" else _exact_ffn(case, s)


def _leaf(t):
    return None if t is None else t.double().requires_grad_()


def _exact_norm(case, s):
    x, y, gate, w_post, w_pre = (_leaf(s[n]) for n in ("x", "y", "gate", "w_post", "w_pre"))
    power = lambda v: (v.square().sum(1) / v.shape[1] + _EPS)[:, None]
    p = y if w_post is None else y * power(y) ** -0.5 * w_post
    if gate is not None:
        p = p * gate[torch.arange(case["T"], device="cuda") // case["gate"]]
    r = x * case["scale"] + p
    n = None if w_pre is None else r * power(r) ** -0.5 * w_pre
    if not case["train"]:
        return [r.detach(), None if n is None else n.detach()]
    loss = (r * s["dr"].double()).sum()
    if n is not None:
        loss = loss + (n * s["dn"].double()).sum()
    leaves = [t for t in (x, y, gate, w_post, w_pre) if t is not None]
    grads = iter(torch.autograd.grad(loss, leaves))
    return [r.detach(), None if n is None else n.detach(),
            *(None if t is None else next(grads) for t in (x, y, gate, w_post, w_pre))]


def _exact_ffn(case, s):
    if case["R"] * case["d"] * case["I"] * (3 if case["train"] else 1) > 2 ** 38:
        return None
    y = torch.zeros(s["x"].shape, dtype=torch.float64, device="cuda")
    names = ("x", "w_gate", "w_up", "w_down")
    grads = [torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in names] if case["train"] else []
    ends = s["offsets"].cpu().numpy()
    for e in range(case["E"]):
        at = slice(int(ends[e]), int(ends[e + 1]))
        if at.start == at.stop:
            continue
        leaves = [_leaf(s["x"][at])] + [_leaf(s[n][e]) for n in names[1:]]
        x, wg, wu, wd = leaves
        with torch.set_grad_enabled(case["train"]):
            a = torch.einsum("rd,id->ri", x, wg)
            out = torch.einsum("ri,di->rd", a * torch.sigmoid(a) * torch.einsum("rd,id->ri", x, wu), wd)
        y[at] = out.detach()
        if case["train"]:
            got = torch.autograd.grad(out, leaves, s["dy"][at].double())
            grads[0][at] = got[0]
            for whole, one in zip(grads[1:], got[1:]):
                whole[e] = one
    return [y, *grads] if case["train"] else y


# ------------------------------------------------------------------------------ work

def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "norm":
        n = case["T"] * case["d"]
        gates = -(-case["T"] // case["gate"]) * case["d"] if case["gate"] else 0
        tensors = 3 + case["pre"] + ((3 + case["pre"]) if case["train"] else 0)
        vectors = 4 * case["d"] * (case["pre"] + case["post"]) * (2 if case["train"] else 1)
        return {"bytes": size * (tensors * n + gates * (2 if case["train"] else 1)) + vectors,
                "flops": (30 if case["train"] else 10) * n}
    rows = max(case["U"], int(case["R"] * (1 - case["masked"])))
    per = case["d"] * case["I"]
    weights = 3 * case["U"] * per
    # (the rows behind the last expert's are written, not read)
    tensors = rows * case["d"] + case["R"] * case["d"]
    if case["train"]:
        return {"bytes": size * (weights + 3 * case["E"] * per + 2 * tensors), "flops": 18 * rows * per}
    return {"bytes": size * (weights + tensors), "flops": 6 * rows * per}
