"""Training and adapter operators of the MoE layer, as cases that can be timed and compared.

Five kinds of call:

  ffn_train         the gated feed-forward block over expert-contiguous rows, keeping what its backward pass needs:
                    g = x Wg^T, u = x Wu^T, h = SiLU(g) (.) u, y = h Wd^T.  One expert is a dense (or shared) block.
  ffn_backward      its gradients: dx, dWg, dWu, dWd from x, g, u and dy.
  combine_backward  gradients of y[t] = sum_i w[t,i] p[row_of[t,i]]: of the rows p, and of the gate weights w.
  adapter_linear    y[t] = (base[t] +) x[t] W^T + scale[a] (x[t] A[a]^T) B[a]^T with a = adapter_of[t], the adapter of the
                    request that token t belongs to; an id below zero is a request without one.
  adapter_gated     h = SiLU(gate) (.) up, gate and up being such projections of one input: a feed-forward block's first half.

Layer shapes are the repository's own (moe_inputs.PRESETS) or generic.  `skew` is the exponent of the power law that the
experts' popularity follows.  Activations ~ N(0, 1), weights ~ N(0, 1/fan-in), gradients ~ N(0, 1e-2), all bf16.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
BF16 = torch.bfloat16

# (d, F, E, k) of moe_inputs.PRESETS, and one dense block
_SHAPES = {"tiny": (256, 512, 8, 2), "mixtral": (4096, 14336, 8, 2), "qwen2moe": (3584, 2560, 64, 8), "dsv3": (7168, 2048, 256, 8),
           "dense": (2048, 5632, 1, 1)}


def _layer(kind, shape, T, skew=0.0):
    d, F, E, k = _SHAPES[shape]
    return {"kind": kind, "T": T, "d": d, "F": F, "E": E, "k": k, "skew": skew}


def _adapters(kind, T, K, N, rank, adapters, requests, without=0.0, base=False):
    return {"kind": kind, "T": T, "K": K, "N": N, "rank": rank, "adapters": adapters, "requests": requests, "without": without, "base": base}


def listed():
    named = {
        # A small layer's step: launches and latency.
        "train forward, tiny, 64 tokens": _layer("ffn_train", "tiny", 64),
        # A training step's block with a thousand rows per expert: bound by the matrix cores.
        "train forward, mixtral, 4096 tokens": _layer("ffn_train", "mixtral", 4096),
        # The smallest backward pass.
        "backward, tiny, 64 tokens": _layer("ffn_backward", "tiny", 64),
        # The largest: six products of a training step.
        "backward, mixtral, 4096 tokens": _layer("ffn_backward", "mixtral", 4096),
        # Many mid-size experts, popular and unpopular ones side by side, an odd token count.
        "backward, qwen2moe, 1999 tokens, skew 1": _layer("ffn_backward", "qwen2moe", 1999, 1.0),
        # A dense block (or the expert that all tokens share), a batch that is no multiple of any tile.
        "backward, dense, 2000 tokens": _layer("ffn_backward", "dense", 2000),
        # A short odd batch of eight experts per token.
        "combine backward, qwen2moe, 333 tokens": _layer("combine_backward", "qwen2moe", 333),
        # A training batch on the widest model: 470 MB of rows.
        "combine backward, dsv3, 4096 tokens": _layer("combine_backward", "dsv3", 4096),
        # One user's decode step: a down projection with that user's adapter, added to what the routed experts gave.
        "adapter linear, 1 token": _adapters("adapter_linear", 1, 14336, 4096, 16, 8, 1, base=True),
        # A ragged prefill batch of a few requests, some without an adapter, on the shared expert's down projection.
        "adapter linear, 1999 tokens": _adapters("adapter_linear", 1999, 2048, 7168, 32, 16, 11, without=0.2),
        # A decode batch: every token another request, each with its adapter out of 64.
        "adapter gated, 48 tokens": _adapters("adapter_gated", 48, 4096, 14336, 64, 64, 48),
        # A prefill batch of six prompts on the wide block.
        "adapter gated, 4096 tokens": _adapters("adapter_gated", 4096, 4096, 14336, 16, 8, 6),
    }
    return [dict(c, name=n) for n, c in named.items()]


_MOST_FLOPS = 12 * 4096 * 2 * 4096 * 14336       # the largest listed case
_MOST_WEIGHTS = 3 * 8 * 4096 * 14336


def _log(rng, a, b):
    return math.exp(rng.uniform(math.log(a), math.log(b)))


def draw(rng):
    """One more case: a preset's or a generic shape, 1 to 8192 tokens over the logarithm, routing from uniform to heavily skewed;
    1 to 64 adapters of ranks 8 to 128, requests from one to one per token."""
    kind = rng.choice(["ffn_train", "ffn_backward", "ffn_backward", "combine_backward", "adapter_linear", "adapter_gated"])
    while True:
        T = round(_log(rng, 1, 8192))
        d, F = 64 * round(_log(rng, 4, 112)), 64 * round(_log(rng, 4, 224))
        if kind.startswith("adapter"):
            n = rng.randint(1, 64)
            K, N = (F, d) if kind == "adapter_linear" else (d, F)
            c = _adapters(kind, T, K, N, 8 * rng.choice([1, 2, 2, 3, 4, 8, 8, 16]), n, round(_log(rng, 1, T)),
                          rng.choice([0.0, 0.0, round(rng.random(), 2)]), kind == "adapter_linear" and rng.random() < 0.4)
        else:
            E = rng.choice([1, 1, 4, 7, 8, 16, 32, 60, 64])
            c = {"kind": kind, "T": T, "d": d, "F": F, "E": E, "k": rng.randint(1, min(E, 8)), "skew": rng.choice([0.0, 0.0, round(rng.uniform(0.3, 2.0), 2)])}
            if rng.random() < 0.3:
                c = _layer(kind, rng.choice(["tiny", "mixtral", "qwen2moe", "dense"]), T, c["skew"])
            if 3 * c["E"] * c["d"] * c["F"] > _MOST_WEIGHTS:
                continue
        if work(c)["flops"] <= _MOST_FLOPS:
            return c


# ---- inputs -------------------------------------------------------------------------------------------------------------


def _normal(shape, std, seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1_000_003 + stream) * 4099)
    t = torch.empty(shape, dtype=BF16, device=DEV).normal_(generator=g)
    return t.mul_(std) if std != 1.0 else t


def _routing(case, seed):
    """k distinct experts for every token, by popularity: the rows' order by expert (stable), and how many each expert has."""
    T, E, k = case["T"], case["E"], case["k"]
    rank = np.random.default_rng([seed, 11]).permutation(E) + 1.0
    p = torch.from_numpy(rank ** -float(case["skew"])).expand(T, E)
    g = torch.Generator().manual_seed(seed)
    flat = torch.multinomial(p, k, generator=g).reshape(-1)
    src = torch.sort(flat, stable=True).indices
    row_of = torch.empty_like(src)
    row_of[src] = torch.arange(T * k)
    w = torch.rand((T, k), generator=g) + 0.1
    return torch.bincount(flat, minlength=E).tolist(), row_of.view(T, k), w / w.sum(1, keepdim=True)


def _inputs(case, seed):
    if case["kind"].startswith("adapter"):
        T, K, N, r, n = (case[x] for x in ("T", "K", "N", "rank", "adapters"))
        g = np.random.default_rng([seed, 7])
        # contiguous requests of uneven lengths, each with one adapter or none
        cuts = np.sort(g.choice(T - 1, case["requests"] - 1, replace=False) + 1) if case["requests"] > 1 else np.zeros(0, np.int64)
        of_request = g.permutation(max(n, case["requests"]))[: case["requests"]] % n
        of_request = np.where(g.random(case["requests"]) < case["without"], -1, of_request)
        ids = of_request[np.searchsorted(cuts, np.arange(T), side="right")]
        two = 2 if case["kind"] == "adapter_gated" else 1
        i = {"x": _normal((T, K), 1.0, seed, 0), "adapter_of": torch.from_numpy(ids.astype(np.int32)).to(DEV),
             "scale": torch.from_numpy((0.5 + g.random(n)).astype(np.float32)).to(DEV),
             "W": [_normal((N, K), K ** -0.5, seed, 1 + m) for m in range(two)],
             "A": [_normal((n, r, K), K ** -0.5, seed, 3 + m) for m in range(two)],
             "B": [_normal((n, N, r), r ** -0.5, seed, 5 + m) for m in range(two)],
             "base": _normal((T, N), 1.0, seed, 8) if case["base"] else None}
        return i
    T, d, F, E, k = (case[n] for n in ("T", "d", "F", "E", "k"))
    R = T * k
    counts, row_of, w = _routing(case, seed)
    if case["kind"] == "combine_backward":
        return {"dy": _normal((T, d), 1e-2, seed, 0), "y_perm": _normal((R, d), 1.0, seed, 1),
                "row_of": row_of.to(torch.int32).to(DEV), "topk_w": w.to(DEV)}
    i = {"counts": counts, "offsets": torch.tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).to(DEV),
         "x": _normal((R, d), 1.0, seed, 0), "wg": _normal((E, F, d), d ** -0.5, seed, 2), "wu": _normal((E, F, d), d ** -0.5, seed, 3),
         "wd": _normal((E, d, F), F ** -0.5, seed, 4)}
    if case["kind"] == "ffn_backward":
        i.update(g=_normal((R, F), 1.0, seed, 5), u=_normal((R, F), 1.0, seed, 6), dy=_normal((R, d), 1e-2, seed, 7))
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

    def buf(*shape, dtype=BF16):
        return torch.empty(shape, dtype=dtype, device=DEV)

    if c["kind"].startswith("adapter"):
        cfg = moe.AdapterConfig.of(c["T"], c["N"], c["K"], c["adapters"], c["rank"])
        s["out"] = {"cfg": cfg, "y": buf(c["T"], c["N"]), "ws": buf(moe.adapter_workspace_size(cfg), dtype=torch.uint8)}
        return s["out"]
    cfg = moe.MoEConfig.of(c["T"], c["d"], c["F"], c["E"], c["k"])
    R, d, F, E = c["T"] * c["k"], c["d"], c["F"], c["E"]
    o = {"cfg": cfg}
    if c["kind"] == "combine_backward":
        o.update(dy_perm=buf(R, d), d_topk_w=buf(c["T"], c["k"], dtype=torch.float32))
    elif c["kind"] == "ffn_train":
        o.update(g=buf(R, F), u=buf(R, F), h=buf(R, F), y=buf(R, d), ws=buf(moe.ffn_workspace_size(cfg), dtype=torch.uint8))
    else:
        o.update(dx=buf(R, d), dwg=buf(E, F, d), dwu=buf(E, F, d), dwd=buf(E, d, F), ws=buf(moe.ffn_backward_workspace_size(cfg), dtype=torch.uint8))
    s["out"] = o
    return o


def _run_own(s):
    import paper_2605_23911_amd as moe
    kind, o = s["case"]["kind"], _buffers(s)
    if kind == "ffn_train":
        moe.moe_grouped_ffn_train(o["cfg"], s["x"], s["offsets"], s["wg"], s["wu"], s["wd"], o["g"], o["u"], o["h"], o["y"], o["ws"])
        return {n: o[n] for n in ("g", "u", "h", "y")}
    if kind == "ffn_backward":
        moe.moe_grouped_ffn_backward(o["cfg"], s["x"], s["offsets"], s["wg"], s["wu"], s["wd"], s["g"], s["u"], s["dy"],
                                     o["dx"], o["dwg"], o["dwu"], o["dwd"], o["ws"])
        return {n: o[n] for n in ("dx", "dwg", "dwu", "dwd")}
    if kind == "combine_backward":
        moe.moe_combine_backward(o["cfg"], s["dy"], s["y_perm"], s["row_of"], s["topk_w"], o["dy_perm"], o["d_topk_w"])
        return {n: o[n] for n in ("dy_perm", "d_topk_w")}
    if kind == "adapter_linear":
        moe.moe_adapter_linear(o["cfg"], s["x"], s["W"][0], s["A"][0], s["B"][0], s["scale"], s["adapter_of"], o["y"], o["ws"], base=s["base"])
    else:
        moe.moe_adapter_gated_up(o["cfg"], s["x"], *s["W"], *s["A"], *s["B"], s["scale"], s["adapter_of"], o["y"], o["ws"])
    return {"y": o["y"]}


def _experts(s):
    """(expert, its rows) of the experts that have any."""
    stop = np.cumsum(s["counts"])
    return [(e, slice(int(b) - n, int(b))) for e, (n, b) in enumerate(zip(s["counts"], stop)) if n]


def _ffn_train(s):
    R, F = s["x"].shape[0], s["wg"].shape[1]
    out = {n: torch.empty((R, F), dtype=BF16, device=DEV) for n in ("g", "u", "h")}
    out["y"] = torch.empty_like(s["x"])
    for e, rows in _experts(s):
        x = s["x"][rows].float()
        g, u = x @ s["wg"][e].float().t(), x @ s["wu"][e].float().t()
        h = g / (1 + torch.exp(-g)) * u
        out["g"][rows], out["u"][rows], out["h"][rows] = g, u, h
        out["y"][rows] = h @ s["wd"][e].float().t()
    return out


def _ffn_backward(s):
    out = {"dx": torch.empty_like(s["x"]), "dwg": torch.zeros_like(s["wg"]), "dwu": torch.zeros_like(s["wu"]), "dwd": torch.zeros_like(s["wd"])}
    for e, rows in _experts(s):
        x, dy, g, u = (s[n][rows].float() for n in ("x", "dy", "g", "u"))
        sig = 1 / (1 + torch.exp(-g))
        dh = dy @ s["wd"][e].float()
        dg, du = dh * u * sig * (1 + g * (1 - sig)), dh * g * sig
        out["dx"][rows] = dg @ s["wg"][e].float() + du @ s["wu"][e].float()
        out["dwg"][e] = dg.t() @ x
        out["dwu"][e] = du.t() @ x
        out["dwd"][e] = dy.t() @ (g * sig * u)
    return out


def _combine_backward(s):
    T, k = s["topk_w"].shape
    rows, dy = s["row_of"].reshape(-1).long(), s["dy"].float()
    dy_perm = torch.empty_like(s["y_perm"])
    dy_perm[rows] = (s["topk_w"][:, :, None] * dy[:, None, :]).reshape(T * k, -1).to(BF16)
    return {"dy_perm": dy_perm, "d_topk_w": (s["y_perm"].float()[rows].view(T, k, -1) * dy[:, None, :]).sum(2)}


def _project(s, x, m):
    """x W^T + scale (x A^T) B^T: products with all adapters at once, of which each token keeps its own."""
    A, B, ids = s["A"][m].float(), s["B"][m].float(), s["adapter_of"].long()
    n, r, K = A.shape
    mine = (ids[:, None] == torch.arange(n, device=DEV)) * s["scale"]
    v = (x @ A.view(n * r, K).t()).view(-1, n, r) * mine[:, :, None]
    return x @ s["W"][m].float().t() + v.view(-1, n * r) @ B.transpose(1, 2).reshape(n * r, -1)


def run(s):
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    if kind == "ffn_train":
        return _ffn_train(s)
    if kind == "ffn_backward":
        return _ffn_backward(s)
    if kind == "combine_backward":
        return _combine_backward(s)
    x = s["x"].float()
    if kind == "adapter_linear":
        y = _project(s, x, 0)
        return {"y": (y if s["base"] is None else y + s["base"].float()).to(BF16)}
    g, u = _project(s, x, 0), _project(s, x, 1)
    return {"y": (g / (1 + torch.exp(-g)) * u).to(BF16)}


# ---- what it costs at least, and what the results are -------------------------------------------------------------------


def work(case):
    """Each input read once (weights of experts and adapters that are hit, in the mean), each output written once."""
    if case["kind"].startswith("adapter"):
        T, K, N, r = (case[x] for x in ("T", "K", "N", "rank"))
        two = 2 if case["kind"] == "adapter_gated" else 1
        hit = min(case["adapters"], case["requests"]) * (1 - case["without"])
        return {"bytes": 2 * T * K + two * 2 * (N * K + hit * r * (N + K)) + 2 * T * N * (2 if case["base"] else 1),
                "flops": two * 2 * T * (N * K + (1 - case["without"]) * r * (N + K))}
    T, d, F, E, k = (case[n] for n in ("T", "d", "F", "E", "k"))
    R = T * k
    if case["kind"] == "combine_backward":
        return {"bytes": 2 * T * d + 4 * R * d + 12 * R, "flops": 3 * R * d}
    p = np.arange(1, E + 1) ** -float(case["skew"])
    hit = float((1 - (1 - np.minimum(1.0, p / p.sum() * k)) ** T).sum())
    if case["kind"] == "ffn_train":
        return {"bytes": 4 * R * d + 6 * R * F + 6 * hit * d * F, "flops": 6 * R * d * F}
    return {"bytes": 6 * R * d + 4 * R * F + 6 * (hit + E) * d * F, "flops": 12 * R * d * F}


def _exact_projection(i, m):
    x = i["x"].double()
    y = x @ i["W"][m].double().t()
    for a in range(i["scale"].numel()):
        rows = (i["adapter_of"] == a).nonzero()[:, 0]
        if rows.numel():
            low = x[rows] @ i["A"][m][a].double().t()
            y[rows] += (low @ i["B"][m][a].double().t()) * i["scale"][a].double()
    return y


def exact(case, seed):
    """The definitions in float64: the block's gradients by the chain rule from SiLU's own derivative, expert by expert."""
    i = _inputs(case, seed)
    kind = case["kind"]
    if kind == "adapter_linear":
        y = _exact_projection(i, 0)
        return {"y": y if i["base"] is None else y + i["base"].double()}
    if kind == "adapter_gated":
        return {"y": torch.nn.functional.silu(_exact_projection(i, 0)) * _exact_projection(i, 1)}
    if kind == "combine_backward":
        T, k = i["topk_w"].shape
        dy, p = i["dy"].double(), i["y_perm"].double()
        token, w = torch.empty(T * k, dtype=torch.int64, device=DEV), torch.empty(T * k, dtype=torch.float64, device=DEV)
        flat = i["row_of"].reshape(-1).long()
        token[flat] = torch.arange(T * k, device=DEV) // k
        w[flat] = i["topk_w"].reshape(-1).double()
        by_row = dy[token]
        return {"dy_perm": w[:, None] * by_row, "d_topk_w": torch.linalg.vecdot(p, by_row)[flat].view(T, k)}
    R, d = i["x"].shape
    E, F, _ = i["wg"].shape

    def empty(*shape):
        return torch.zeros(shape, dtype=torch.float64, device=DEV)

    if kind == "ffn_train":
        o = {"g": empty(R, F), "u": empty(R, F), "h": empty(R, F), "y": empty(R, d)}
    else:
        o = {"dx": empty(R, d), "dwg": empty(E, F, d), "dwu": empty(E, F, d), "dwd": empty(E, d, F)}
    b = 0
    for e, n in enumerate(i["counts"]):
        a, b = b, b + n
        if n == 0:
            continue
        x, wg, wu, wd = i["x"][a:b].double(), i["wg"][e].double(), i["wu"][e].double(), i["wd"][e].double()
        if kind == "ffn_train":
            o["g"][a:b], o["u"][a:b] = x @ wg.t(), x @ wu.t()
            o["h"][a:b] = torch.nn.functional.silu(o["g"][a:b]) * o["u"][a:b]
            o["y"][a:b] = o["h"][a:b] @ wd.t()
            continue
        g, u, dy = (i[t][a:b].double() for t in ("g", "u", "dy"))
        act, sig = torch.nn.functional.silu(g), torch.sigmoid(g)
        dh = dy @ wd
        du, dg = dh * act, dh * u * (sig + act * (1 - sig))
        o["dx"][a:b] = dg @ wg + du @ wu
        o["dwg"][e], o["dwu"][e], o["dwd"][e] = dg.t() @ x, du.t() @ x, dy.t() @ (act * u)
    return o
