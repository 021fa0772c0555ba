"""The gates' gradient where one weight is next to one: dz of that expert is the little that the others leave.

dz_i = w_i (g_i - sum_j w_j g_j) = w_i ((1 - w_i) g_i - sum_{j != i} w_j g_j), so a change of every g_j by eps of itself changes dz_i by at most eps w_i S_i, S_i = (1 - w_i) |g_i| +
sum_{j != i} w_j |g_j|.  A kernel is held to that with the roundings that it makes (u = 2^-24).  Weights come rounded from fp64, u of themselves each.

For i with w_i <= 1/2 from the first form: k + 1 u in the sum (its fmas, the weights'), and one each in the difference, the product and w_i: (k + 4) u w_i (|g_i| + sum w |g|), of which
the bracket is at most 3 S_i.  For the one above 1/2 from the second: sums of the others' w and w g, k + 1 u each, a product, the difference, w_i and the product with it: (k + 5) u w_i S_i.
Both are below 3 (k + 5) u w_i S_i; the sigmoid's slope 1 / (1 + exp z) adds 6 u of dz_i (exp 4, the sum and the division).
The softmax over all experts: exp is off by 4 u, a sum over the wavefront by 10 u more (four in a lane, six exchanges), p by 4 + 14 + 1 = 19 u, sum p G by 19 + 10 + 2 = 31 u, the difference and the
product by 3 u: 53 u in place of (k + 5) u.  Logits are exact here: a token is one in one column of x.  Each dz then enters one element of dW_r (fp32), in three parts: 3 u of it."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))

from oracle import token_oracle as orc

U = 2.0 ** -24


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_23911_amd as m
    m.lib()
    return m


def case(E, k, gating, offset, twice, seed=0):
    """One token per margin between the leading logit and the rest, 0 to 25 (sigmoid: the rest down to -26), several of each."""
    rng = np.random.default_rng([E, k, gating, seed])
    margins = np.repeat([0, 1, 3, 6, 10, 14, 18, 25], 8)
    T = margins.size
    column = rng.integers(-8, 9, size=(T, E)) / 8.0
    idx = np.argsort(rng.random((T, E)), axis=1)[:, :k].astype(np.int64)
    if gating == orc.SIGMOID:
        column -= margins[:, None]
    lead = idx[np.arange(T), rng.integers(0, k, size=T)]
    column[np.arange(T), lead] = 2.0 if gating == orc.SIGMOID else 1.0 + margins
    assert np.abs(column).max() < 32                     # eight bits
    bias = (rng.integers(-2, 3, size=E) / 8).astype(np.float32)
    z = column + bias
    w = orc.gate(z, idx, gating)
    if twice and k > 1:                                  # the second slot names the first one's expert
        idx[::3, 1] = idx[::3, 0]
        w = orc.gate(z, idx, gating)
    g = (rng.normal(size=(T, k)) + offset).astype(np.float32)
    return z, column, bias, idx, w, g


def gradient(z, idx, w, g, gating):
    """dz and w S [T, E] in fp64, in differences and without one."""
    T, E = z.shape
    g = g.astype(np.float64)
    dz, size = np.zeros((T, E)), np.zeros((T, E))
    if gating == orc.SOFTMAX:
        p = np.exp(z - z.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        G, A = np.zeros((T, E)), np.zeros((T, E))
        for i in range(idx.shape[1]):
            G[np.arange(T), idx[:, i]] += g[:, i]
            A[np.arange(T), idx[:, i]] += abs(g[:, i])
        for e in range(E):
            others = np.arange(E) != e
            dz[:, e] = p[:, e] * (p[:, others] * (G[:, e, None] - G[:, others])).sum(1)
            size[:, e] = p[:, e] * (p[:, others] * (A[:, e, None] + A[:, others])).sum(1)
        return dz, size
    for t in range(T):
        for i in range(idx.shape[1]):
            others = np.arange(idx.shape[1]) != i
            slope = 1 / (1 + np.exp(z[t, idx[t, i]])) if gating == orc.SIGMOID else 1.0
            dz[t, idx[t, i]] += slope * w[t, i] * (w[t, others] * (g[t, i] - g[t, others])).sum()
            size[t, idx[t, i]] += slope * w[t, i] * (w[t, others] * (abs(g[t, i]) + abs(g[t, others]))).sum()
    return dz, size


def run(moe, column, bias, idx, w, g, gating):
    T, E = column.shape
    d = 64 * ((T + 63) // 64)
    x, wr = torch.zeros((T, d), dtype=torch.bfloat16), torch.zeros((E, d), dtype=torch.bfloat16)
    x[torch.arange(T), torch.arange(T)] = 1
    wr[:, :T] = torch.from_numpy(column.T.copy()).bfloat16()
    cfg = moe.MoEConfig.of(T, d, 64, E, idx.shape[1], gating)
    dwr, dbias = torch.full((E, d), float("nan"), device="cuda"), torch.full((E,), float("nan"), device="cuda")
    moe.moe_route_backward(cfg, x.cuda(), wr.cuda(), torch.from_numpy(bias).cuda(), torch.from_numpy(idx.astype(np.int32)).cuda(), torch.from_numpy(w.astype(np.float32)).cuda(),
                           torch.from_numpy(g).cuda(), None, dwr, dbias, torch.full((moe.route_backward_workspace_size(cfg),), 255, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    return dwr[:, :T].double().cpu().numpy().T, dbias.double().cpu().numpy()


def limit(k, gating, dz, size):
    return 3 * (53 if gating == orc.SOFTMAX else k + 5) * U * size + (6 * (gating == orc.SIGMOID) + 3) * U * np.abs(dz) * 1.01


SHAPES = [(1, 1), (2, 2), (8, 2), (20, 4), (64, 8), (70, 8), (130, 5), (256, 8), (256, 70), (128, 128), (256, 256)]


@pytest.mark.gpu
@pytest.mark.parametrize("twice", [False, True], ids=["once", "twice"])
@pytest.mark.parametrize("offset", [0.0, 30.0])
@pytest.mark.parametrize("gating", [orc.SOFTMAX, orc.RENORM, orc.SIGMOID])
@pytest.mark.parametrize("E,k", SHAPES)
def test_confident_tokens(moe, E, k, gating, offset, twice):
    z, column, bias, idx, w, g = case(E, k, gating, offset, twice)
    dz, size = gradient(z, idx, w, g, gating)
    got, dbias = run(moe, column, bias, idx, w, g, gating)
    bound = limit(k, gating, dz, size)
    off = np.abs(got - dz)
    assert (off <= bound).all(), float((off / np.maximum(bound, 1e-300)).max())
    assert (np.abs(dbias - dz.sum(0)) <= bound.sum(0) + (len(z) + 16) * U * (np.abs(dz) + bound).sum(0)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("gating", [orc.RENORM, orc.SIGMOID])
@pytest.mark.parametrize("E,k", [(8, 2), (64, 8), (256, 70)])
@pytest.mark.parametrize("form", ["half", "twice", "dropped"])
def test_weights_that_do_not_add_up_to_one(moe, E, k, gating, form):
    """The formula as it stands: dz_i = w_i (g_i - sum_j w_j g_j) over the slots whose expert there is."""
    z, column, bias, idx, w, g = case(E, k, gating, 0.0, False, seed=1)
    w = (w * {"half": 0.5, "twice": 2.0, "dropped": 1.0}[form]).astype(np.float32).astype(np.float64)
    if form == "dropped":
        idx[::2, k - 1] = E
        idx[::5, 0] = -1
    dz = orc.gate_backward(z, idx, w, g.astype(np.float64), gating)
    got, _ = run(moe, column, bias, idx, w, g, gating)
    size = np.zeros_like(dz)
    for t in range(len(z)):
        own = (idx[t] >= 0) & (idx[t] < E)
        c = (w[t] * abs(g[t]))[own].sum()
        for i in np.nonzero(own)[0]:
            size[t, idx[t, i]] += w[t, i] * (abs(g[t, i]) + c)
    off, bound = np.abs(got - dz), (k + 16) * U * size + 9 * U * np.abs(dz)
    assert (off <= bound).all(), float((off / np.maximum(bound, 1e-300)).max())


@pytest.mark.gpu
@pytest.mark.parametrize("gating", [orc.RENORM, orc.SIGMOID])
def test_a_weight_of_a_dropped_slot_is_not_lost(moe, gating):
    """What a slot without an expert takes from the sum is no rounding, however little it is: 2^-20 of the whole, where the others have that much, too."""
    T, E, k = 16, 8, 3
    column, bias = np.full((T, E), -1.0), np.zeros(E, np.float32)
    idx = np.tile(np.array([1, 4, E]), (T, 1))
    small = np.float32(2.0 ** -20)
    w = np.tile(np.array([np.float32(1) - 2 * small, small, small], np.float64), (T, 1))
    g = np.stack([np.linspace(-2, 2, T), np.linspace(1, 3, T), np.full(T, np.nan)], 1).astype(np.float32)
    got, _ = run(moe, column, bias, idx, w, g, gating)
    g = g.astype(np.float64)
    slope = 1 / (1 + np.exp(-1.0)) if gating == orc.SIGMOID else 1.0
    want = slope * w[:, 0] * ((1 - w[:, 0]) * g[:, 0] - w[:, 1] * g[:, 1])
    size = w[:, 0] * ((1 - w[:, 0]) * abs(g[:, 0]) + w[:, 1] * abs(g[:, 1]))
    assert (np.abs(got[:, 1] - want) <= (3 * (k + 5) + 9) * U * size).all()
