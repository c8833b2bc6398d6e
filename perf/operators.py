"""Operators around a MoE layer's experts, as cases that can be timed and compared.

Five operators, each through the package's public entry points (``own = True``) or in its plain
form of elementary torch operations (``own = False``):

* ``sort``      tokens sorted by expert (``dmoe_sort_tokens``): where each expert's rows begin,
                which (token, slot) a row is, and which row a (token, slot) has. Slots without an
                expert (masked and padded tokens) stand behind the last expert's rows.
* ``gather``    token rows copied into that order (``dmoe_gather_rows``), and its gradient, which
                sums a token's rows again (``dmoe_gather_rows_backward``).
* ``combine``   the experts' rows back to token order, weighted by the gates, with an optional
                addend such as a shared expert's rows (``dmoe_combine_rows``), and its gradient
                by the rows and by the gates (``dmoe_combine_rows_backward``).
* ``q4``        sorted rows times their experts' 4-bit matrices with a scale per group of
                inputs: plain (``dmoe_q4_linear``) or gate and up with SwiGLU
                (``dmoe_q4_swiglu``). One group without a list of experts is a dense layer.
* ``quantize``  bf16 weights to 4 bits and scales, laid out for the above, and the values that they
                stand for (``dmoe_q4_quantize``, ``dmoe_q4_dequantize``).

Sizes: ``T`` tokens of ``k`` slots, ``E`` experts, width ``d``; for the products ``U`` experts in
use, ``K`` inputs, ``N`` outputs, groups of ``g`` inputs.
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # one decoding block of 32 tokens: the sort is a small part of a step, all latency
        dict(name="sort_step", op="sort", T=32, k=8, E=256, masked=0.0),
        # a training micro-batch of padded sequences, a seventh of the tokens masked
        dict(name="sort_train", op="sort", T=65536, k=8, E=256, masked=0.15),
        # eight users' decoding blocks into expert order
        dict(name="gather_step", op="gather", back=False, T=256, k=8, d=2048, dtype="bf16", masked=0.0),
        # the gradient of a training micro-batch's gather
        dict(name="gather_grad", op="gather", back=True, T=16384, k=8, d=2048, dtype="bf16", masked=0.1),
        # a ragged batch of odd width in half precision, with a shared expert's rows added
        dict(name="combine_odd", op="combine", back=False, T=1031, k=6, d=1001, dtype="fp16", masked=0.2,
             add=True),
        # the gradient of a training micro-batch's combine, by the rows and by the gates
        dict(name="combine_grad", op="combine", back=True, T=16384, k=8, d=2048, dtype="bf16", masked=0.1,
             add=False),
        # one token through its eight experts' gate and up products: what a single user waits for
        dict(name="q4_token", op="q4", gated=True, T=1, k=8, E=256, U=8, K=2048, N=512, g=64),
        # a decoding block under block top-k: 32 rows for each of eight experts
        dict(name="q4_block", op="q4", gated=True, T=32, k=8, E=256, U=8, K=2048, N=512, g=64),
        # the same block routed token by token: the down products of about a hundred experts
        dict(name="q4_routed", op="q4", gated=False, T=32, k=8, E=256, U=104, K=512, N=2048, g=32),
        # a prompt of 2048 tokens through all experts
        dict(name="q4_prompt", op="q4", gated=True, T=2048, k=8, E=256, U=256, K=2048, N=512, g=128),
        # a toy layer's weights, converted in a test
        dict(name="quantize_toy", op="quantize", E=16, K=256, N=128, g=32),
        # one of a layer's three weights, converted at load time
        dict(name="quantize_layer", op="quantize", E=256, K=2048, N=512, g=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sort", "gather", "combine", "q4", "quantize"])
    k = rng.randint(1, 16)
    masked = rng.choice([0.0, 0.05, 0.2, 0.5])
    if op == "sort":
        return dict(op=op, T=min(_log(rng, 1, 131072), 65536 * 8 // k), k=k, E=rng.randint(max(k, 2), 256),
                    masked=masked)
    if op in ("gather", "combine"):
        d = _log(rng, 64, 8192)
        if rng.random() < 0.7:
            d = (d + 7) // 8 * 8
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        most = 16384 * 8 * 2048 // (k * d * (2 if dtype == "fp32" else 1))
        case = dict(op=op, back=rng.random() < 0.5, T=min(_log(rng, 1, 16384), most), k=k, d=d,
                    dtype=dtype, masked=masked)
        if op == "combine":
            case["add"] = not case["back"] and rng.random() < 0.5
        return case
    g = rng.choice([32, 64, 128])
    if op == "quantize":
        K, N = g * _log(rng, 1, 8192 // g), _log(rng, 16, 8192)
        return dict(op=op, E=max(1, min(_log(rng, 1, 256), 256 * 512 * 2048 // (K * N))), K=K, N=N, g=g)
    gated = rng.random() < 0.5
    K, N = g * _log(rng, 2, 8192 // g), _log(rng, 64, 8192)
    if rng.random() < 0.25:      # a dense layer
        T = min(_log(rng, 1, 2048), max(1, 2 ** 34 // (K * N)))
        return dict(op=op, gated=gated, T=T, k=1, E=1, U=1, K=K, N=N, g=g)
    N = min(N, 2 ** 28 // (K * k))
    E = max(k, min(_log(rng, 16, 256), 2 ** 28 // (K * N)))
    T = min(_log(rng, 1, 2048), max(1, 2 ** 34 // (K * N * k)))
    U = max(k, min(E, T * k, _log(rng, k, 256)))
    return dict(op=op, gated=gated, T=T, k=k, E=E, U=U, K=K, N=N, g=g)


# ------------------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(gen, shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def _routing(gen, T, k, E, U):
    """int32 [T, k]: k different experts for each token, some far more popular than others. All of
    the U experts in use have a row."""
    pop = -0.5 * torch.log(torch.arange(1, U + 1, device="cuda", dtype=torch.float32))
    noise = torch.rand((T, U), generator=gen, device="cuda").clamp_(1e-7, 1 - 1e-7)
    idx = torch.topk(pop - torch.log(-torch.log(noise)), k, dim=1).indices
    first = -(-U // k)                       # these tokens go through the experts in turn
    turn = torch.arange(min(first, T) * k, device="cuda").reshape(-1, k) % U
    idx[: turn.shape[0]] = turn
    names = torch.randperm(E, generator=gen, device="cuda")[:U]
    return names[idx].to(torch.int32)


def _mask(gen, idx, share):
    """Whole tokens masked at the end of each of up to 8 padded sequences, and a few single slots."""
    if share <= 0:
        return idx
    T, k = idx.shape
    S = min(8, T)
    length = -(-T // S)
    keep = (1 - 2 * share * torch.rand(S, generator=gen, device="cuda")) * length
    at = torch.arange(T, device="cuda")
    padded = (at % length).float() >= keep[at // length]
    single = torch.rand((T, k), generator=gen, device="cuda") < 0.01
    return torch.where(padded[:, None] | single, -1, idx).to(torch.int32)


def _sorted(idx, E):
    """offsets, rows, pos of the routing (the order that the sort gives)."""
    key = torch.where((idx < 0) | (idx >= E), E, idx).reshape(-1).long()
    order = torch.sort(key, stable=True).indices
    at = torch.arange(key.numel(), device=idx.device)
    pos = torch.empty_like(order)
    pos[order] = at
    pos = torch.where(key == E, -1 - pos, pos)
    rows = torch.where(key[order] == E, -1, order)
    counts = torch.zeros(E + 1, dtype=torch.int64, device=idx.device).scatter_add_(
        0, key, torch.ones_like(key))
    offsets = torch.cat([counts.new_zeros(1), torch.cumsum(counts[:E], 0)])
    return offsets.to(torch.int32), rows.to(torch.int32), pos.to(torch.int32)


def _weights(gen, E, N, K):
    # expert matrices as trained: each of its own size, a few large inputs
    w = torch.empty((E, N, K), dtype=torch.bfloat16, device="cuda")
    size = 0.01 + 0.02 * torch.rand(E, generator=gen, device="cuda")
    for e0 in range(0, E, 32):
        n = min(32, E - e0)
        w[e0:e0 + n] = torch.randn((n, N, K), generator=gen, device="cuda") * size[e0:e0 + n, None, None]
    return w


def _inputs(case, seed):
    gen = _gen(seed)
    op = case["op"]
    if op == "quantize":
        return {"w": _weights(gen, case["E"], case["N"], case["K"])}
    T, k = case["T"], case["k"]
    if op == "q4":
        idx = _routing(gen, T, k, case["E"], case["U"])
        s = {"idx": idx, "x": _randn(gen, (T, case["K"]), torch.bfloat16)}
        s["w"] = [_weights(gen, case["E"], case["N"], case["K"]) for _ in range(2 if case["gated"] else 1)]
        return s
    E = case.get("E", 256)
    idx = _mask(gen, _routing(gen, T, k, E, E), case["masked"])
    if op == "sort":
        return {"idx": idx}
    dtype, d = _DTYPES[case["dtype"]], case["d"]
    s = {"idx": idx}
    if op == "gather":
        s["a"] = _randn(gen, (T * k if case["back"] else T, d), dtype)
        return s
    gates = torch.rand((T, k), generator=gen, device="cuda") + 0.05
    gates = torch.where(idx < 0, 0.0, gates)
    s["gates"] = gates / gates.sum(1, keepdim=True).clamp_min(1e-6)
    s["ys"] = _randn(gen, (T * k, d), dtype)
    if case["back"]:
        s["dy"] = _randn(gen, (T, d), dtype)
    s["add"] = _randn(gen, (T, d), dtype) if case["add"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op = case["op"]
    if own:
        import paper_2605_30876_gb300 as dmoe
    if op == "quantize":
        if own:
            s["desc"] = dmoe.make_q4_desc(case["E"], case["N"], case["K"], case["g"])
            s["codes"], s["scales"] = dmoe.alloc_q4(s["desc"], "cuda")
            s["out"] = torch.empty_like(s["w"])
        return s
    T, k = case["T"], case["k"]
    if op == "sort":
        if own:
            E = case["E"]
            s["ws"] = dmoe.alloc_sort_workspace(T, k, E, "cuda")
            s["out"] = (torch.empty(E + 1, dtype=torch.int32, device="cuda"),
                        torch.empty(T * k, dtype=torch.int32, device="cuda"),
                        torch.empty(T * k, dtype=torch.int32, device="cuda"))
        return s
    E = case.get("E", 256)
    s["offsets"], s["rows"], s["pos"] = _sorted(s.pop("idx"), E)
    if op == "q4":
        s["R"] = T * k
        weights = s.pop("w")
        if own:
            s["desc"] = dmoe.make_q4_desc(E, case["N"], case["K"], case["g"])
            s["w"] = []
            for w in weights:
                codes, scales = dmoe.alloc_q4(s["desc"], "cuda")
                dmoe.dmoe_q4_quantize(s["desc"], w, codes, scales)
                s["w"] += [codes, scales]
            s["out"] = torch.empty((T * k, case["N"]), dtype=torch.bfloat16, device="cuda")
        else:
            s["w"] = [_codes(w, case["g"]) for w in weights]
            s["first"] = s["offsets"].tolist()     # (the plain form goes through the experts on the host)
        return s
    if own:
        new = lambda *shape, t=_DTYPES[case["dtype"]]: torch.empty(shape, dtype=t, device="cuda")
        if op == "gather":
            s["out"] = new(T if case["back"] else T * k, case["d"])
        elif case["back"]:
            s["out"] = (new(T * k, case["d"]), new(T, k, t=torch.float32))
        else:
            s["out"] = new(T, case["d"])
    return s


# ------------------------------------------------------------------------------ one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2605_30876_gb300 as dmoe
    case, op = s["case"], s["case"]["op"]
    if op == "sort":
        dmoe.dmoe_sort_tokens(s["idx"], case["E"], *s["out"], workspace=s["ws"])
    elif op == "gather" and case["back"]:
        dmoe.dmoe_gather_rows_backward(s["a"], s["pos"], s["out"])
    elif op == "gather":
        dmoe.dmoe_gather_rows(s["a"], s["pos"], s["out"])
    elif op == "combine" and case["back"]:
        dmoe.dmoe_combine_rows_backward(s["dy"], s["ys"], s["pos"], s["gates"], *s["out"])
    elif op == "combine":
        dmoe.dmoe_combine_rows(s["ys"], s["pos"], s["gates"], s["add"], s["out"])
    elif op == "q4":
        call = dmoe.dmoe_q4_swiglu if case["gated"] else dmoe.dmoe_q4_linear
        call(s["desc"], s["x"], s["offsets"], *s["w"], s["out"], rows=s["rows"], k=case["k"])
    else:
        dmoe.dmoe_q4_quantize(s["desc"], s["w"], s["codes"], s["scales"])
        dmoe.dmoe_q4_dequantize(s["desc"], s["codes"], s["scales"], s["out"])
    return s["out"]


def _codes(w, g):
    """(int8 [E, N, K], bf16 [E, N, K/g]): codes of -7 .. 7 and scales of five significant bits."""
    E, N, K = w.shape
    codes = torch.empty((E, N, K), dtype=torch.int8, device=w.device)
    scales = torch.empty((E, N, K // g), dtype=torch.bfloat16, device=w.device)
    step = max(1, 2 ** 26 // (N * K))
    for e0 in range(0, E, step):
        v = w[e0:e0 + step].float().reshape(-1, N, K // g, g)
        s = v.abs().amax(-1) / torch.full((), 7.0, device=w.device)
        bits = s.view(torch.int32)
        bits = (bits + 0x3FFFF + ((bits >> 19) & 1)) & ~0x7FFFF      # to nearest, ties to even
        s = bits.view(torch.float32)
        c = torch.round(v / torch.where(s > 0, s, 1.0)[..., None])
        codes[e0:e0 + step] = c.reshape(-1, N, K).to(torch.int8)
        scales[e0:e0 + step] = s.to(torch.bfloat16)
    return codes, scales


def _values(codes, scales, g):
    shape = codes.shape
    v = codes.float().reshape(*shape[:-1], shape[-1] // g, g) * scales.float()[..., None]
    return v.reshape(shape)


def _run_plain(s):
    case, op = s["case"], s["case"]["op"]
    if op == "sort":
        return _sorted(s["idx"], case["E"])
    if op == "quantize":
        return _values(*_codes(s["w"], case["g"]), case["g"]).to(torch.bfloat16)
    if op == "q4":
        src = (s["rows"] // case["k"]).long()
        x = s["x"].float()[src]
        out = torch.empty((s["R"], case["N"]), dtype=torch.bfloat16, device=x.device)
        for e in range(case["E"]):
            lo, hi = s["first"][e], s["first"][e + 1]
            if lo == hi:
                continue
            y = [x[lo:hi] @ _values(c[e], sc[e], case["g"]).t() for c, sc in s["w"]]
            out[lo:hi] = (y[0] / (1 + torch.exp(-y[0])) * y[1] if case["gated"] else y[0]).to(out.dtype)
        return out
    T, k, d = case["T"], case["k"], case["d"]
    pos = s["pos"].long()
    valid = pos >= 0
    at = torch.where(valid, pos, -1 - pos)
    if op == "gather" and not case["back"]:
        a = s["a"]
        out = torch.empty((T * k, d), dtype=a.dtype, device=a.device)
        out[at] = torch.where(valid[:, None], a.repeat_interleave(k, 0), 0)
        return out
    at, valid = at.view(T, k), valid.view(T, k)
    if op == "gather":
        acc = torch.zeros((T, d), device=pos.device)
        for j in range(k):
            acc = acc + torch.where(valid[:, j, None], s["a"][at[:, j]].float(), 0)
        return acc.to(s["a"].dtype)
    g, ys = s["gates"], s["ys"]
    if not case["back"]:
        acc = s["add"].float() if s["add"] is not None else torch.zeros((T, d), device=pos.device)
        for j in range(k):
            acc = acc + torch.where(valid[:, j, None], g[:, j, None] * ys[at[:, j]].float(), 0)
        return acc.to(ys.dtype)
    dy = s["dy"].float()
    dys = torch.empty_like(ys)
    dg = torch.empty_like(g)
    for j in range(k):
        v = valid[:, j, None]
        dys[at[:, j]] = torch.where(v, g[:, j, None] * dy, 0).to(ys.dtype)
        dg[:, j] = torch.where(v, dy * ys[at[:, j]].float(), 0).sum(1)
    return dys, dg


# ------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "sort":
        return tuple(torch.from_numpy(a).cuda() for a in _order_by_hand(s["idx"].cpu().numpy(), case["E"]))
    if op == "quantize":
        return _quantized(s["w"], case["g"])[2]
    T, k = case["T"], case["k"]
    E = case.get("E", 256)
    offsets, rows, pos = _order_by_hand(s["idx"].cpu().numpy(), E)
    if op == "q4":
        out = torch.zeros((T * k, case["N"]), dtype=torch.float64, device="cuda")
        used = np.flatnonzero(np.diff(offsets))
        for e in used:
            r = torch.from_numpy(rows[offsets[e]:offsets[e + 1]] // k).long().cuda()
            xe = s["x"][r].double()
            y = [torch.einsum("rk,nk->rn", xe, _quantized(w[e:e + 1], case["g"])[2][0]) for w in s["w"]]
            if case["gated"]:
                y[0] = y[0] * torch.sigmoid(y[0]) * y[1]
            out[int(offsets[e]):int(offsets[e + 1])] = y[0]
        return out
    # the order as a sparse matrix of ones: P[r, t] = 1 where row r is one of token t's
    live = int(offsets[E])
    token = torch.from_numpy(np.where(rows >= 0, rows // k, 0)).long().cuda()
    slot = torch.from_numpy(np.where(rows >= 0, rows % k, 0)).long().cuda()
    ok = (torch.arange(T * k, device="cuda") < live).double()[:, None]
    if op == "gather":
        a = s["a"].double()
        if not case["back"]:
            return a[token] * ok
        return torch.zeros((T, case["d"]), dtype=torch.float64, device="cuda").index_add_(0, token, a * ok)
    w = s["gates"].double()[token, slot][:, None] * ok
    ys = s["ys"].double()
    if not case["back"]:
        y = torch.zeros((T, case["d"]), dtype=torch.float64, device="cuda").index_add_(0, token, ys * w)
        return y if s["add"] is None else y + s["add"].double()
    dyr = s["dy"].double()[token]
    dg = torch.zeros((T, k), dtype=torch.float64, device="cuda")
    dg[token[:live], slot[:live]] = torch.einsum("rd,rd->r", dyr[:live], ys[:live])
    return dyr * w, dg


def _order_by_hand(idx, E):
    key = idx.reshape(-1).astype(np.int64)
    R = key.size
    dropped = np.flatnonzero((key < 0) | (key >= E))
    kept = np.flatnonzero((key >= 0) & (key < E))
    by = kept[np.lexsort((kept, key[kept]))]
    rows = np.full(R, -1, np.int32)
    pos = np.empty(R, np.int32)
    rows[:by.size] = by
    pos[by] = np.arange(by.size)
    pos[dropped] = -1 - np.arange(by.size, R)
    offsets = np.searchsorted(key[by], np.arange(E + 1), side="left").astype(np.int32)
    return offsets, rows, pos


def _quantized(w, g):
    """codes, scales and values in 64 bits of bf16 weights [E, N, K]."""
    E, N, K = w.shape
    values = torch.empty((E, N, K), dtype=torch.float64, device=w.device)
    codes = scales = None
    for e in range(E):
        v = w[e].double().reshape(N, K // g, g)
        a = v.abs().max(-1).values / 7
        power = (a.view(torch.int64) & (0x7FF << 52)).view(torch.float64)   # of two, at most a
        unit = torch.where(power > 0, power, 1.0) / 16                # five significant bits
        scales = torch.round(a / unit) * unit
        codes = torch.round(v / torch.where(scales > 0, scales, 1.0)[..., None])
        values[e] = (codes * scales[..., None]).reshape(N, K)
    return codes, scales, values


# ------------------------------------------------------------------------------ work

def work(case):
    op = case["op"]
    if op == "quantize":
        n = case["E"] * case["N"] * case["K"]
        return {"bytes": n * (2 + 2 + 2 * (0.5 + 2 / case["g"])), "flops": 4 * n}
    T, k = case["T"], case["k"]
    R = T * k
    if op == "sort":
        return {"bytes": 12 * R + 4 * (case["E"] + 1), "flops": 0}
    if op == "q4":
        m = 2 if case["gated"] else 1
        weights = m * case["U"] * case["N"] * case["K"] * (0.5 + 2 / case["g"])
        return {"bytes": weights + 2 * T * case["K"] + 2 * R * case["N"] + 4 * R,
                "flops": 2 * m * R * case["N"] * case["K"]}
    size, d = (4 if case["dtype"] == "fp32" else 2), case["d"]
    live = R * (1 - case["masked"])
    if op == "gather":
        if case["back"]:
            return {"bytes": (live + T) * d * size + 4 * R, "flops": live * d}
        return {"bytes": (R + T) * d * size + 4 * R, "flops": 0}
    if case["back"]:
        return {"bytes": (live + R + T) * d * size + 12 * R, "flops": 3 * live * d}
    return {"bytes": (live + T * (2 if case["add"] else 1)) * d * size + 8 * R, "flops": 2 * live * d}
