"""Operators on the token side of a training step, as cases that can be timed and compared.

Six kinds of call:

  dispatch           tokens sorted by expert: slot (t, i) of expert e = topk_idx[t, i] has a row where e is one of the E experts held here
                     (first .. first + E - 1) and fewer than `capacity` earlier slots chose it.  Rows are expert-contiguous, in order of slots:
                     rows[row_of[t, i]] = (w[t, i]) x[t].
  dispatch_backward  dx[t] = (base[t] +) sum_i (w[t, i]) drows[row_of[t, i]], and dw[t, i] = <x[t], drows[row_of[t, i]]>.
  collect            back in the tokens' order: y[t] = (residual[t] +) D(sum_i w[t, i] rows[row_of[t, i]]), D being dropout.
  collect_backward   its gradients: v = D(dy), drows[row_of[t, i]] = w[t, i] v[t], dw[t, i] = <v[t], rows[row_of[t, i]]>.
  dropout            y = (residual +) D(x) alone.
  route_backward     gradients of the gate weights w = gate(x W_r^T + bias)[topk_idx]: of x, W_r and bias.

D keeps element n with probability 1 - p and divides by it.  Its mask is a function of (seed, offset, n) alone: the Philox4x32-10 generator (Salmon, Moraes,
Dror and Shaw, 2011) with the seed as key and (n / 8, offset) as counter gives sixteen bits for each of eight elements; those below 65536 p are dropped.

Layer shapes are the repository's own (moe_inputs.PRESETS) or generic.  `skew` is the exponent of the power law that the experts' popularity follows.
Activations ~ N(0, 1), router weights ~ N(0, 1/d), gradients ~ N(0, 1e-2), all bf16.  What no slot's row covers stays as it was: zero, or -1 in a table.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
BF16 = torch.bfloat16

# (d, E, k, gating) of moe_inputs.PRESETS
_SHAPES = {"tiny": (256, 8, 2, 0), "mixtral": (4096, 8, 2, 0), "qwen2moe": (3584, 64, 8, 1), "dsv3": (7168, 256, 8, 0)}


def _tokens(kind, T, d, k, experts, E=None, first=0, capacity=0, weighted=True, skew=0.0, add=False, p=0.0):
    return {"kind": kind, "T": T, "d": d, "k": k, "experts": experts, "E": E or experts, "first": first, "capacity": capacity, "weighted": weighted,
            "skew": skew, "add": add, "p": p}


def _of(kind, shape, T, **more):
    d, experts, k, _ = _SHAPES[shape]
    return _tokens(kind, T, d, k, experts, **more)


def _router(T, d, E, k, gating, skew=0.0):
    return {"kind": "route_backward", "T": T, "d": d, "k": k, "E": E, "gating": gating, "skew": skew}


def listed():
    d3 = _SHAPES["dsv3"]
    named = {
        # One user's decode step: latency of a launch.
        "dispatch, mixtral, 1 token": _of("dispatch", "mixtral", 1, weighted=False),
        # A training batch on the widest model, popular experts cut off at a quarter above the mean: 400 MB of rows, scaled on the way in.
        "dispatch, dsv3, 4096 tokens, capacity 160": _of("dispatch", "dsv3", 4096, capacity=160, skew=0.5),
        # A short odd batch on a GPU that holds a quarter of the experts: some tokens have no row here.
        "dispatch backward, qwen2moe share, 333 tokens": _of("dispatch_backward", "qwen2moe", 333, E=16, first=16),
        # A training batch: the sum of a token's rows' gradients on top of the router's.
        "dispatch backward, dsv3, 4096 tokens": _of("dispatch_backward", "dsv3", 4096, weighted=False, add=True),
        # A decode batch's way back onto the residual stream.
        "collect, mixtral, 64 tokens": _of("collect", "mixtral", 64, add=True),
        # A training batch's, with dropout.
        "collect, dsv3, 4096 tokens, dropout": _of("collect", "dsv3", 4096, add=True, p=0.1),
        # A mid-size batch that is no multiple of anything, experts with a limit.
        "collect backward, qwen2moe, 1999 tokens, dropout": _of("collect_backward", "qwen2moe", 1999, capacity=300, skew=1.0, p=0.1),
        # The largest: rows read and their gradients written, 0.9 GB.
        "collect backward, dsv3, 4096 tokens, dropout": _of("collect_backward", "dsv3", 4096, p=0.1),
        # A handful of elements; an odd number of them.
        "dropout, 1999 x 257": _tokens("dropout", 1999, 257, 1, 1, p=0.1),
        # A batch's hidden states of the widest model.
        "dropout, 4096 x 7168, residual": _tokens("dropout", 4096, 7168, 1, 1, add=True, p=0.25),
        # A ragged batch through a renormalised gate: the gradient has eight entries per token.
        "route backward, qwen2moe, 1999 tokens": _router(1999, 3584, 64, 8, 1),
        # A training batch on the widest model: every expert's logit has a gradient.
        "route backward, dsv3, 4096 tokens": _router(4096, d3[0], d3[1], d3[2], d3[3]),
    }
    return [dict(c, name=n) for n, c in named.items()]


_MOST_BYTES = 2 * 4096 * 7168 + 4 * 4096 * 8 * 7168         # the largest listed case's
_MOST_FLOPS = 6 * 4096 * 256 * 7168


def _log(rng, a, b):
    return math.exp(rng.uniform(math.log(a), math.log(b)))


def draw(rng):
    """One more case: 1 to 16384 tokens over the logarithm, widths of 8 to 8192, 1 to 12 choices out of up to 256 experts of which all or a share are here,
    with or without a limit, weights, something added, and dropout; routers of all three gates."""
    kind = rng.choice(["dispatch", "dispatch_backward", "collect", "collect_backward", "dropout", "route_backward"])
    while True:
        T = round(_log(rng, 1, 16384))
        experts = rng.choice([1, 4, 7, 8, 16, 32, 60, 64, 128, 256])
        k = rng.randint(1, min(experts, rng.choice([2, 8, 8, 12])))
        skew = rng.choice([0.0, 0.0, round(rng.uniform(0.3, 2.0), 2)])
        p = rng.choice([0.0, round(rng.uniform(0.01, 0.6), 3)])
        if kind == "route_backward":
            c = _router(T, 64 * round(_log(rng, 1, 128)), experts, k, rng.randint(0, 2), skew)
        elif kind == "dropout":
            c = _tokens(kind, T, round(_log(rng, 1, 8192)), 1, 1, add=rng.random() < 0.5, p=p or 0.1)
        else:
            d = 8 * round(_log(rng, 1, 1024))
            E = experts if rng.random() < 0.5 else rng.randint(1, experts)
            capacity = 0 if rng.random() < 0.5 else max(1, round(T * k / experts * rng.uniform(0.5, 2.0)))
            c = _tokens(kind, T, d, k, experts, E, rng.randint(0, experts - E), capacity, rng.random() < 0.7, skew,
                        kind in ("collect", "dispatch_backward") and rng.random() < 0.5, p if kind.startswith("collect") else 0.0)
        w = work(c)
        if w["bytes"] <= _MOST_BYTES and w["flops"] <= _MOST_FLOPS and T * k <= 65536:
            return c


# ---- inputs -------------------------------------------------------------------------------------------------------------


def _normal(shape, std, seed, stream, dtype=BF16):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1_000_003 + stream) * 4099)
    t = torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=g)
    return t.mul_(std) if std != 1.0 else t


def _rng(seed):
    """What a training program keeps on the device: a seed, and an offset that it advances with every use."""
    a, b = np.random.default_rng([seed, 5]).integers(0, 1 << 62, size=2)
    return torch.tensor([int(a) * 2 + 1, int(b)], dtype=torch.int64).to(DEV)


def _choices(case, seed):
    """k distinct experts for every token, by popularity, and gate weights that add up to one."""
    T, n, k = case["T"], case["experts"], case["k"]
    rank = np.random.default_rng([seed, 11]).permutation(n) + 1.0
    p = torch.from_numpy(rank ** -float(case["skew"])).expand(T, n)
    g = torch.Generator().manual_seed(seed)
    idx = torch.multinomial(p, k, generator=g)
    w = torch.rand((T, k), generator=g) + 0.1
    return idx.to(torch.int32), w / w.sum(1, keepdim=True)


def _rows_of_slots(case, idx):
    """Host: each slot's row (-1: none), from a count of the slots in front of it."""
    e = idx.numpy().reshape(-1).astype(np.int64) - case["first"]
    E, most = case["E"], case["capacity"] or 1 << 40
    here = (e >= 0) & (e < E)
    at = np.arange(e.size)
    order = np.argsort(np.where(here, e, E), kind="stable")
    n = np.bincount(np.where(here, e, E), minlength=E + 1)
    rank = np.empty(e.size, np.int64)
    rank[order] = at - (np.cumsum(n) - n)[np.where(here, e, E)[order]]
    start = np.concatenate([[0], np.cumsum(np.minimum(n[:E], most))])
    return torch.from_numpy(np.where(here & (rank < most), start[np.minimum(np.maximum(e, 0), E - 1)] + rank, -1).astype(np.int32)).view(case["T"], case["k"])


def _inputs(case, seed):
    kind, T, d, k = (case[n] for n in ("kind", "T", "d", "k"))
    if kind == "route_backward":
        E = case["E"]
        x, w_r = _normal((T, d), 1.0, seed, 0), _normal((E, d), d ** -0.5, seed, 1)
        rank = np.random.default_rng([seed, 11]).permutation(E) + 1.0
        bias = torch.from_numpy(np.log((rank ** -float(case["skew"]))).astype(np.float32)).to(DEV)
        z = x.double() @ w_r.double().t() + bias.double()
        top, idx = torch.topk(z, k, dim=1)
        if case["gating"] == 0:
            w = torch.exp(top - torch.logsumexp(z, 1, keepdim=True))
        else:
            w = torch.softmax(top, 1) if case["gating"] == 1 else torch.sigmoid(top) / torch.sigmoid(top).sum(1, keepdim=True)
        return {"x": x, "w_r": w_r, "bias": bias, "idx": idx.to(torch.int32), "w": w.float(), "g": _normal((T, k), 0.5, seed, 2, torch.float32)}
    i = {"rng": _rng(seed)}
    if kind == "dropout":
        return {**i, "x": _normal((T, d), 1.0, seed, 0), "add": _normal((T, d), 1.0, seed, 1) if case["add"] else None}
    idx, w = _choices(case, seed)
    i["w"] = w.to(DEV) if case["weighted"] else None
    i["add"] = _normal((T, d), 1.0, seed, 2) if case["add"] else None
    if kind == "dispatch":
        return {**i, "x": _normal((T, d), 1.0, seed, 0), "idx": idx.to(DEV)}
    i["row_of"] = _rows_of_slots(case, idx).to(DEV)
    i["rows"] = _normal((T * k, d), 1e-2 if kind == "dispatch_backward" else 1.0, seed, 1)
    if kind == "dispatch_backward":
        i["x"] = _normal((T, d), 1.0, seed, 0) if case["weighted"] else None
    elif kind == "collect_backward":
        i["dy"] = _normal((T, d), 1e-2, seed, 0)
    return i


def prepare(case, seed):
    return {"case": case, **_inputs(case, seed)}


# ---- one pass -----------------------------------------------------------------------------------------------------------


def _buffers(s):
    """What a user's program allocates once: outputs and the workspace."""
    if "out" in s:
        return s["out"]
    import paper_2605_23911_amd as moe
    c = s["case"]
    kind, T, d, k = (c[n] for n in ("kind", "T", "d", "k"))

    def buf(*shape, dtype=BF16, value=0):
        return torch.full(shape, value, dtype=dtype, device=DEV)

    f32, i32 = torch.float32, torch.int32
    if kind == "route_backward":
        cfg = moe.MoEConfig.of(T, d, 64, c["E"], k, c["gating"])
        o = {"cfg": cfg, "dx": buf(T, d), "dw_r": buf(c["E"], d, dtype=f32), "dbias": buf(c["E"], dtype=f32),
             "ws": buf(moe.route_backward_workspace_size(cfg), dtype=torch.uint8)}
    elif kind == "dropout":
        o = {"y": buf(T, d)}
    else:
        cfg = moe.DispatchConfig.of(T, d, k, c["E"], c["first"], c["capacity"])
        o = {"cfg": cfg}
        if kind == "dispatch":
            o.update(counts=buf(c["E"], dtype=i32), offsets=buf(c["E"] + 1, dtype=i32), row_of=buf(T, k, dtype=i32), src_of=buf(T * k, dtype=i32, value=-1),
                     rows=buf(T * k, d), ws=buf(moe.dispatch_workspace_size(cfg), dtype=torch.uint8))
        elif kind == "dispatch_backward":
            o.update(dx=buf(T, d), dw=buf(T, k, dtype=f32) if c["weighted"] else None)
        elif kind == "collect":
            o.update(y=buf(T, d))
        else:
            o.update(drows=buf(T * k, d), dw=buf(T, k, dtype=f32) if c["weighted"] else None)
    s["out"] = o
    return o


def _run_own(s):
    import paper_2605_23911_amd as moe
    c, o = s["case"], _buffers(s)
    kind = c["kind"]
    if kind == "dispatch":
        moe.moe_dispatch(o["cfg"], s["x"], s["idx"], s["w"], o["counts"], o["offsets"], o["row_of"], o["src_of"], o["rows"], o["ws"])
        return {n: o[n] for n in ("counts", "offsets", "row_of", "src_of", "rows")}
    if kind == "dispatch_backward":
        moe.moe_dispatch_backward(o["cfg"], s["rows"], s["row_of"], s["w"], o["dx"], x=s["x"], d_topk_w=o["dw"], base=s["add"])
        return {n: o[n] for n in ("dx", "dw") if o[n] is not None}
    if kind == "collect":
        moe.moe_collect(o["cfg"], s["rows"], s["row_of"], s["w"], o["y"], residual=s["add"], p=c["p"], rng=s["rng"])
        return {"y": o["y"]}
    if kind == "collect_backward":
        moe.moe_collect_backward(o["cfg"], s["dy"], s["rows"] if c["weighted"] else None, s["row_of"], s["w"], o["drows"], d_topk_w=o["dw"], p=c["p"], rng=s["rng"])
        return {n: o[n] for n in ("drows", "dw") if o[n] is not None}
    if kind == "dropout":
        moe.moe_dropout(s["x"], o["y"], c["p"], s["rng"], residual=s["add"])
        return {"y": o["y"]}
    moe.moe_route_backward(o["cfg"], s["x"], s["w_r"], s["bias"], s["idx"], s["w"], s["g"], o["dx"], o["dw_r"], o["dbias"], o["ws"])
    return {n: o[n] for n in ("dx", "dw_r", "dbias")}


def _limit(p):
    """p in steps of 2^-16."""
    return int(math.floor(p * 65536 + 0.5))


def _dropped(v, p, rng):
    """D(v) of v [T, d] in 32 bits.  The generator's products are taken modulo 2^64, where signs do not matter."""
    if p == 0.0:
        return v
    low = 0xFFFFFFFF
    n = v.numel()
    at = torch.arange((n + 7) // 8, device=DEV)
    x0, x1, x2, x3 = at & low, at >> 32, (rng[1] & low).expand_as(at), ((rng[1] >> 32) & low).expand_as(at)
    k0, k1 = rng[0] & low, (rng[0] >> 32) & low
    for _ in range(10):
        a, b = x0 * 0xD2511F53, x2 * 0xCD9E8D57
        x0, x1, x2, x3 = ((b >> 32) & low) ^ x1 ^ k0, b & low, ((a >> 32) & low) ^ x3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([x0, x1, x2, x3], 1)
    bits = torch.stack([words & 0xFFFF, words >> 16], 2).view(-1)[:n].view(v.shape)
    return torch.where(bits >= _limit(p), v * (65536.0 / (65536 - _limit(p))), 0.0)


def _dispatch(s):
    c = s["case"]
    T, k, E = c["T"], c["k"], c["E"]
    e = s["idx"].reshape(-1).long() - c["first"]
    here = (e >= 0) & (e < E)
    key = torch.where(here, e, E)
    slots = torch.arange(T * k, device=DEV)
    order = torch.sort(key, stable=True).indices
    n = (key[:, None] == torch.arange(E + 1, device=DEV)).sum(0)
    rank = torch.empty_like(slots)
    rank[order] = slots - (torch.cumsum(n, 0) - n)[key[order]]
    kept = n[:E].clamp(max=c["capacity"]) if c["capacity"] else n[:E]
    start = torch.cat([torch.zeros_like(n[:1]), torch.cumsum(kept, 0)])
    have = here & (rank < c["capacity"]) if c["capacity"] else here
    row = torch.where(have, start[key.clamp(max=E - 1)] + rank, -1)
    src = torch.full((T * k,), -1, dtype=torch.int32, device=DEV)
    src[row[have]] = slots[have].int()
    rows = torch.zeros((T * k, c["d"]), dtype=BF16, device=DEV)
    x = s["x"].float()[slots[have] // k]
    rows[row[have]] = (x if s["w"] is None else x * s["w"].view(-1)[have][:, None]).to(BF16)
    return {"counts": n[:E].int(), "offsets": start.int(), "row_of": row.int().view(T, k), "src_of": src, "rows": rows}


def _weights(s):
    """Gate weights, zero where a slot has no row, and rows' numbers that can be indexed with."""
    have = s["row_of"] >= 0
    w = torch.where(have, s["w"] if s["w"] is not None else torch.ones_like(have, dtype=torch.float32), 0.0)
    return have, w, s["row_of"].long().clamp(min=0)


def _gathered(s):
    have, w, at = _weights(s)
    total = torch.zeros((s["case"]["T"], s["case"]["d"]), device=DEV)
    for i in range(w.shape[1]):
        total = total + w[:, i, None] * s["rows"][at[:, i]].float()
    return total


def _dots(s, v):
    have, _, at = _weights(s)
    return torch.stack([torch.where(have[:, i], (v * s["rows"][at[:, i]].float()).sum(1), 0.0) for i in range(at.shape[1])], 1)


def _collect_backward(s):
    have, w, at = _weights(s)
    v = _dropped(s["dy"].float(), s["case"]["p"], s["rng"])
    drows = torch.zeros_like(s["rows"])
    for i in range(w.shape[1]):
        drows[at[have[:, i], i]] = (w[:, i, None] * v)[have[:, i]].to(BF16)
    return {"drows": drows, "dw": _dots(s, v)} if s["w"] is not None else {"drows": drows}


def _route_backward(s):
    x, w_r, idx, g = s["x"].float(), s["w_r"].float(), s["idx"].long(), s["g"]
    z = x @ w_r.t() + s["bias"]
    chosen = idx[:, :, None] == torch.arange(z.shape[1], device=DEV)
    if s["case"]["gating"] == 0:
        e = torch.exp(z - z.max(1, keepdim=True).values)
        p = e / e.sum(1, keepdim=True)
        G = (chosen * g[:, :, None]).sum(1)
        dz = p * (G - (p * G).sum(1, keepdim=True))
    else:
        d = s["w"] * (g - (s["w"] * g).sum(1, keepdim=True))
        dz = (chosen * d[:, :, None]).sum(1)
        if s["case"]["gating"] == 2:
            dz = dz / (1 + torch.exp(z))
    return {"dx": (dz @ w_r).to(BF16), "dw_r": dz.t() @ x, "dbias": dz.sum(0)}


def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    kind = c["kind"]
    if kind == "dispatch":
        return _dispatch(s)
    if kind == "collect_backward":
        return _collect_backward(s)
    if kind == "route_backward":
        return _route_backward(s)
    y = s["x"].float() if kind == "dropout" else _gathered(s)
    if kind != "dispatch_backward":
        y = _dropped(y, c["p"], s["rng"])
    y = (y if s["add"] is None else y + s["add"].float()).to(BF16)
    if kind != "dispatch_backward":
        return {"y": y}
    return {"dx": y, "dw": _dots(s, s["x"].float())} if s["w"] is not None else {"dx": y}


# ---- what it costs at least, and what the results are -------------------------------------------------------------------


def _kept(case):
    """Slots with a row, in the mean: an expert's share of the choices, up to its limit."""
    p = np.arange(1, case["experts"] + 1) ** -float(case["skew"])
    n = np.minimum(1.0, p / p.sum() * case["k"]) * case["T"]
    if case["capacity"]:
        n = np.minimum(n, case["capacity"])
    return float(n.sum()) * case["E"] / case["experts"]


def work(case):
    """Each input read once, each output written once; rows that a slot has, in the mean."""
    kind, T, d, k = (case[n] for n in ("kind", "T", "d", "k"))
    if kind == "route_backward":
        products = 6 if case["gating"] != 1 else 4
        return {"bytes": 4 * T * d + 6 * case["E"] * d + 12 * T * k, "flops": products * T * case["E"] * d}
    if kind == "dropout":
        return {"bytes": (6 if case["add"] else 4) * T * d, "flops": 2 * T * d}
    n = min(_kept(case), T * k)
    w = case["weighted"]
    if kind == "dispatch":
        return {"bytes": 2 * T * d + 2 * n * d + (16 if w else 12) * T * k, "flops": n * d}
    if kind == "dispatch_backward":
        return {"bytes": 2 * n * d + 2 * T * d * (1 + w + case["add"]) + (12 if w else 4) * T * k, "flops": (4 if w else 1) * n * d}
    if kind == "collect":
        return {"bytes": 2 * n * d + 2 * T * d * (1 + case["add"]) + (8 if w else 4) * T * k, "flops": 2 * n * d}
    return {"bytes": 2 * T * d + 2 * n * d * (1 + w) + (12 if w else 4) * T * k, "flops": (3 if w else 1) * n * d}


def _kept_exactly(case, i):
    """The mask [T, d], from the generator's definition on unsigned 64-bit numbers of the host."""
    seed, offset = (int(v) for v in i["rng"].cpu())
    T, d = case["T"], case["d"]
    n = T * d
    u = np.uint64
    low = u(0xFFFFFFFF)
    block = np.arange((n + 7) // 8, dtype=np.uint64)
    ctr = [block & low, block >> u(32), np.full_like(block, offset & 0xFFFFFFFF), np.full_like(block, offset >> 32)]
    for r in range(10):
        key = [((seed & 0xFFFFFFFF) + r * 0x9E3779B9) & 0xFFFFFFFF, ((seed >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF]
        first, second = ctr[0] * u(0xD2511F53), ctr[2] * u(0xCD9E8D57)
        ctr = [(second >> u(32)) ^ ctr[1] ^ u(key[0]), second & low, (first >> u(32)) ^ ctr[3] ^ u(key[1]), first & low]
    halves = np.empty((block.size, 8), np.uint16)
    for j in range(8):
        halves[:, j] = (ctr[j // 2] >> u(16 * (j % 2))) & u(0xFFFF)
    return torch.from_numpy(halves.reshape(-1)[:n].reshape(T, d) >= _limit(case["p"])).to(DEV)


def exact(case, seed):
    """The definitions in float64; tables by counting, expert by expert."""
    i = _inputs(case, seed)
    kind, T, d, k = (case[n] for n in ("kind", "T", "d", "k"))
    f64 = torch.float64
    if kind == "route_backward":
        x, w_r, g = i["x"].double(), i["w_r"].double(), i["g"].double()
        z = torch.addmm(i["bias"].double(), x, w_r.t())
        idx = i["idx"].long()
        if case["gating"] == 0:
            logs = torch.log_softmax(z, 1)
            w = torch.gather(logs, 1, idx).exp()
            dz = -(w * g).sum(1, keepdim=True) * logs.exp()
            dz.scatter_add_(1, idx, w * g)
        else:
            w = i["w"].double()
            d_top = w * g - w * (w * g).sum(1, keepdim=True)
            if case["gating"] == 2:
                d_top = d_top * torch.sigmoid(-torch.gather(z, 1, idx))
            dz = torch.zeros_like(z).scatter_add_(1, idx, d_top)
        return {"dx": torch.mm(dz, w_r), "dw_r": torch.mm(dz.t(), x), "dbias": dz.sum(0)}
    scale = 65536.0 / (65536 - _limit(case["p"]))
    keep = _kept_exactly(case, i) if case["p"] else None

    def dropped(v):
        return v if keep is None else v.masked_fill(~keep, 0.0) * scale

    def plus(v):
        return v if i["add"] is None else v + i["add"].double()

    if kind == "dropout":
        return {"y": plus(dropped(i["x"].double()))}
    w = i["w"].double() if i["w"] is not None else torch.ones((T, k), dtype=f64, device=DEV)
    if kind == "dispatch":
        idx, x = i["idx"].reshape(-1), i["x"].double()
        counts, offsets = [], [0]
        row_of = torch.full((T * k,), -1, dtype=torch.int32, device=DEV)
        src_of = torch.full((T * k,), -1, dtype=torch.int32, device=DEV)
        rows = torch.zeros((T * k, d), dtype=f64, device=DEV)
        for e in range(case["E"]):
            slots = (idx == case["first"] + e).nonzero()[:, 0]
            counts.append(slots.numel())
            slots = slots[: case["capacity"]] if case["capacity"] else slots
            a, b = offsets[-1], offsets[-1] + slots.numel()
            offsets.append(b)
            row_of[slots] = torch.arange(a, b, dtype=torch.int32, device=DEV)
            src_of[a:b] = slots.int()
            rows[a:b] = x[slots // k] * w.view(-1)[slots][:, None]
        as_int = {"dtype": torch.int32, "device": DEV}
        return {"counts": torch.tensor(counts, **as_int), "offsets": torch.tensor(offsets, **as_int), "row_of": row_of.view(T, k), "src_of": src_of, "rows": rows}
    flat = i["row_of"].reshape(-1).long()
    slots = (flat >= 0).nonzero()[:, 0]
    token, mine = slots // k, i["rows"].double()[flat[slots]]
    if kind == "collect_backward":
        v = dropped(i["dy"].double())
        o = {"drows": torch.zeros(i["rows"].shape, dtype=f64, device=DEV)}
        o["drows"][flat[slots]] = v[token] * w.view(-1)[slots][:, None]
    else:
        total = torch.zeros((T, d), dtype=f64, device=DEV).index_add_(0, token, mine * w.view(-1)[slots][:, None])
        if kind == "collect":
            return {"y": plus(dropped(total))}
        o = {"dx": plus(total)}
        v = i["x"].double() if i["x"] is not None else None
    if i["w"] is not None:
        dw = torch.zeros(T * k, dtype=f64, device=DEV)
        dw[slots] = torch.linalg.vecdot(mine, v[token])
        o["dw"] = dw.view(T, k)
    return o
