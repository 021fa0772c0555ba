"""How many bits of dz the router's gradient carries into its products, against oracle/token_oracle.py (u = 2^-24, W and G the sizes of a token's gate weights and of their gradients by
expert; the logits are not needed, or exact).

dz_e itself is off by off_e = (k + 16) u W_e (G_e + sum W G) in the renormalised gate: a few roundings of w_i, of d_i and of their products, and k of the sum.  Where every
other term of a sum is zero, a product with dz in all its 24 bits adds at most one rounding per part and term.  A dz held in two bf16 numbers is off by up to 2^-16 = 256 u of
itself; the bounds below are less, which the tests without a GPU make sure of with the same inputs."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))

from oracle import token_oracle as orc

U, B = 2.0 ** -24, 2.0 ** -8
PARTS = 3


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_23911_amd as m
    m.lib()
    return m


def held(v, parts):
    """v (fp32 values) as a sum of `parts` bf16 numbers, each what the ones in front leave, rounded."""
    left, out = torch.from_numpy(v.astype(np.float32)), []
    for _ in range(parts):
        out.append(left.bfloat16().float())
        left = left - out[-1]
    return sum(o.double() for o in out).numpy()


# tokens, width, experts: few tokens, the products' small tiles, two sizes of larger ones, the largest with up to 64 experts
SHAPES = [(50, 64, 40), (1500, 1536, 40), (2112, 4160, 256), (4200, 4224, 256), (4200, 8192, 64)]


def choices(T, E, k, seed):
    rng = np.random.default_rng([T, E, k, seed])
    idx = np.argsort(rng.random((T, E)), axis=1)[:, :k].astype(np.int32)
    w = rng.random((T, k)) + 0.2
    return rng, idx, (w / w.sum(1, keepdims=True)).astype(np.float32), rng.normal(size=(T, k)).astype(np.float32)


def renormalised(idx, w, g, E):
    """dz [T, E] of the renormalised gate in fp64, and how far a kernel's may be off."""
    T, k = idx.shape
    dz = orc.gate_backward(np.zeros((T, E)), idx, w.astype(np.float64), g.astype(np.float64), orc.RENORM)
    W, G = np.zeros((T, E)), np.zeros((T, E))
    np.put_along_axis(W, idx.astype(np.int64), w.astype(np.float64), 1)
    np.put_along_axis(G, idx.astype(np.int64), np.abs(g.astype(np.float64)), 1)
    return dz, (k + 16) * U * W * (G + (W * G).sum(1, keepdims=True))


K = 3
LEVEL = 128.0


def equal_weights_case(T, E):
    """Every weight of the router is LEVEL, so dx is LEVEL times the sum of a token's dz, which is next to nothing.  3 K terms, a rounding each."""
    _, idx, w, g = choices(T, E, K, 1)
    dz, off = renormalised(idx, w, g, E)
    want = LEVEL * dz.sum(1)
    return idx, w, g, dz, want, LEVEL * (off.sum(1) + PARTS * K * U * (np.abs(dz) + off).sum(1)) * (1 + B) + B * np.abs(want)


def opposite_pairs_case(T, E, d):
    """Tokens t and t + h have one element each, in the same column, and gradients that are opposite but for 2^-13 of them: a column of dW_r is the little that is left of two dz,
    and its rounding to bf16 is less than a dz's to 16 bits."""
    h = T // 2
    _, idx, w, g = choices(h, E, K, 2)
    g2 = (-g * np.float32(1 + 2.0 ** -13)).astype(np.float32)
    dz, off = renormalised(idx, w, g, E)
    dz2, off2 = renormalised(idx, w, g2, E)
    at = (np.arange(h) * 7) % d if np.gcd(7, d) == 1 else np.arange(h)
    x = torch.zeros((2 * h, d), dtype=torch.bfloat16)
    x[torch.arange(h), torch.from_numpy(at)] = 1
    x[torch.arange(h) + h, torch.from_numpy(at)] = 1
    want = dz + dz2
    bound = (off + off2 + 2 * PARTS * U * (np.abs(dz) + np.abs(dz2) + off + off2)) * (1 + B) + B * np.abs(want)
    return np.concatenate([idx, idx]), np.concatenate([w, w]), np.concatenate([g, g2]), x, at, dz, dz2, want, bound


def single_terms_case(T, d, E, gating):
    """Token t is one in column t alone (T <= d), so its logits are that column of the router's, and column t of dW_r is its dz.  The logits, and their sums with the bias, are
    exact.  The softmax over all experts: p is off by 16 u of itself (exp, the sum, the division), and the sum over p_i g_i and the difference by a few u more: 24 u of
    their sizes; the sigmoid gate as the renormalised one."""
    rng, idx, w, g = choices(T, E, K, 3)
    column = rng.integers(-16, 17, size=(T, E)) / 8.0
    bias = (rng.integers(-8, 9, size=E) / 8).astype(np.float32)
    z = column + bias
    if gating != orc.RENORM:
        w = orc.gate(z, idx.astype(np.int64), gating).astype(np.float32)
    dz = orc.gate_backward(z, idx, w.astype(np.float64), g.astype(np.float64), gating)
    if gating == orc.SOFTMAX:
        p = np.exp(z - z.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        G = np.zeros((T, E))
        np.put_along_axis(G, idx.astype(np.int64), np.abs(g.astype(np.float64)), 1)
        off = 24 * U * p * (G + 2 * (p * G).sum(1, keepdims=True))
    else:
        off = renormalised(idx, w, g, E)[1]
    x, wr = torch.zeros((T, d), dtype=torch.bfloat16), torch.zeros((E, d), dtype=torch.bfloat16)
    x[torch.arange(T), torch.arange(T)] = 1
    wr[:, :T] = torch.from_numpy(column.T.copy()).bfloat16()
    return idx, w, g, bias, x, wr, dz, off + PARTS * U * (np.abs(dz) + off)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_two_parts_would_be_seen(shape):
    """The bounds admit dz in three parts and not in two."""
    T, d, E = shape
    _, _, _, dz, want, bound = equal_weights_case(T, E)
    assert (np.abs(LEVEL * held(dz, 3).sum(1) - want) <= bound).all() and (np.abs(LEVEL * held(dz, 2).sum(1) - want) > bound).any()
    *_, dz, dz2, want, bound = opposite_pairs_case(T, E, d)
    assert (np.abs(held(dz, 3) + held(dz2, 3) - want) <= bound).all() and (np.abs(held(dz, 2) + held(dz2, 2) - want) > bound).any()
    for gating in (orc.SOFTMAX, orc.RENORM, orc.SIGMOID):
        *_, dz, bound = single_terms_case(T, d, E, gating)
        assert (np.abs(held(dz, 3) - dz) <= bound).all() and (np.abs(held(dz, 2) - dz) > bound).mean() > 0.001


def run(moe, x, wr, idx, w, g, gating, dx, dwr, bias=None):
    T, d = x.shape
    E = wr.shape[0]
    cfg = moe.MoEConfig.of(T, d, 64, E, idx.shape[1], gating)
    moe.moe_route_backward(cfg, x.cuda(), wr.cuda(), None if bias is None else torch.from_numpy(bias).cuda(), *(torch.from_numpy(v).cuda() for v in (idx, w, g)), dx, dwr, None,
                           torch.full((moe.route_backward_workspace_size(cfg),), 255, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()


def full(shape, dtype=torch.bfloat16):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("weights", [None, torch.float32, torch.bfloat16], ids=["dx alone", "fp32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_dx_has_all_bits(moe, shape, weights):
    T, d, E = shape
    idx, w, g, _, want, bound = equal_weights_case(T, E)
    dx = full((T, d))
    run(moe, torch.zeros((T, d), dtype=torch.bfloat16), torch.full((E, d), LEVEL, dtype=torch.bfloat16), idx, w, g, orc.RENORM, dx, None if weights is None else full((E, d), weights))
    off = (dx.double().cpu().numpy() - want[:, None])
    assert (np.abs(off) <= bound[:, None]).all(), float((np.abs(off) / bound[:, None]).max())


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [True, False], ids=["with dx", "alone"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_bf16_weight_gradients_have_all_bits(moe, shape, rows):
    T, d, E = shape
    idx, w, g, x, at, _, _, want, bound = opposite_pairs_case(T, E, d)
    dwr = full((E, d))
    run(moe, x, torch.zeros((E, d), dtype=torch.bfloat16), idx, w, g, orc.RENORM, full((x.shape[0], d)) if rows else None, dwr)
    got = dwr.double().cpu().numpy()
    off = np.abs(got[:, at].T - want)
    assert (off <= bound).all(), float((off / np.maximum(bound, 1e-300)).max())
    got[:, at] = 0
    assert (got == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [True, False], ids=["with dx", "alone"])
@pytest.mark.parametrize("gating", [orc.SOFTMAX, orc.RENORM, orc.SIGMOID])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_fp32_weight_gradients_have_all_bits(moe, shape, gating, rows):
    T, d, E = shape
    idx, w, g, bias, x, wr, dz, bound = single_terms_case(T, d, E, gating)
    dwr = full((E, d), torch.float32)
    run(moe, x, wr, idx, w, g, gating, full((T, d)) if rows else None, dwr, bias)
    off = np.abs(dwr[:, :T].double().cpu().numpy().T - dz)
    assert (off <= bound).all(), float((off / np.maximum(bound, 1e-300)).max())
    assert (dwr[:, T:] == 0).all()
