"""The router's gradient against oracle/token_oracle.py.

Bounds (u = 2^-24): a logit's fp32 sum over d products is off by dz_ <= d u sum |x||w| (worst case, any order), and by one rounding for the bias.  A softmax weight
is then off by eps = 2 max dz_ + 16 u of itself (the maximum's error cancels in p; exp and the division a few u), so dz_e by
p_e (eps + 8 u) (|G_e| + 2 sum p |G|); the normalised gates by (2 dz_ + (k + 16) u) w_i (|d_i| + sum w |d|) (dz_ for the sigmoid alone).  In the products dz is held
in 16 bits, 2^-16 of itself, and n fp32 sums add n u of their absolute values; dx (and dW_r in bf16) is rounded once, 2^-8.
Where x and W_r are small whole numbers (over a power of two) the logits are exact, dz_ = 0, and the bound is that of the rest."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))

from oracle import token_oracle as orc

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8
NAN = float("nan")


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_23911_amd as m
    m.lib()
    return m


def full(shape, dtype=torch.bfloat16, value=NAN):
    return torch.full(shape, value, dtype=dtype, device="cuda")


def f64(t):
    return t.detach().cpu().double().numpy()


class Case:
    def __init__(self, T, d, E, k, gating, seed=0, whole=False, bias=True):
        rng = np.random.default_rng([T, d, E, seed])
        if whole:
            x, wr = rng.integers(-2, 3, size=(T, d)), rng.integers(-4, 5, size=(E, d)) / 2.0 ** round(np.log2(4 * d ** 0.5))
        else:
            x, wr = rng.normal(size=(T, d)), rng.normal(size=(E, d)) * d ** -0.5
        self.x, self.wr = torch.from_numpy(x).to(torch.bfloat16), torch.from_numpy(wr).to(torch.bfloat16)
        self.bias = (rng.integers(-8, 9, size=E) / 8).astype(np.float32) if bias else None
        self.shape, self.gating = (T, d, E, k), gating
        self.z = f64(self.x) @ f64(self.wr).T + (self.bias if bias else 0)
        self.idx = np.argsort(-self.z, axis=1, kind="stable")[:, :k].astype(np.int32)
        self.w = orc.gate(self.z, self.idx.astype(np.int64), gating).astype(np.float32)
        self.g = rng.normal(size=(T, k)).astype(np.float32)
        self.dz_ = 0.0 if whole or gating == orc.RENORM else float((d * U * (np.abs(f64(self.x)) @ np.abs(f64(self.wr)).T)).max()) + U * np.abs(self.z).max()

    def run(self, moe, f32=True, accumulate=False, want=("dx", "dwr", "dbias"), held=None, ws=None):
        T, d, E, k = self.shape
        cfg = moe.MoEConfig.of(T, d, 64, E, k, self.gating)
        o = {"dx": full((T, d)), "dwr": full((E, d), torch.float32 if f32 else torch.bfloat16), "dbias": full((E,), torch.float32)}
        if held is not None:
            o["dwr"].copy_(held[0])
            o["dbias"].copy_(held[1])
        ws = full((moe.route_backward_workspace_size(cfg),), torch.uint8, 255) if ws is None else ws
        b = None if self.bias is None else torch.from_numpy(self.bias).cuda()
        moe.moe_route_backward(cfg, self.x.cuda(), self.wr.cuda(), b, *(torch.from_numpy(v).cuda() for v in (self.idx, self.w, self.g)),
                               *(o[n] if n in want else None for n in ("dx", "dwr", "dbias")), ws, accumulate=accumulate)
        torch.cuda.synchronize()
        return o

    def check(self, o, f32=True, held=None, want=("dx", "dwr", "dbias")):
        T, d, E, k = self.shape
        x, wr, idx, w, g = f64(self.x), f64(self.wr), self.idx.astype(np.int64), self.w.astype(np.float64), self.g.astype(np.float64)
        dz = orc.gate_backward(self.z, idx, w, g, self.gating)
        G, own = np.zeros((T, E)), (idx >= 0) & (idx < E)
        for t, i in zip(*np.nonzero(own)):
            G[t, idx[t, i]] += abs(g[t, i])
        if self.gating == orc.SOFTMAX:
            p = np.exp(self.z - self.z.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            off = p * (2 * self.dz_ + 24 * U) * (G + 2 * (p * G).sum(1, keepdims=True))
        else:
            W = np.zeros((T, E))
            for t, i in zip(*np.nonzero(own)):
                W[t, idx[t, i]] += w[t, i]
            off = (2 * self.dz_ + (k + 16) * U) * W * (G + (W * G).sum(1, keepdims=True))
        held_dz, a = off + 2.0**-16 * np.abs(dz), np.abs(dz) + off
        bounds = {"dx": (dz @ wr, held_dz @ np.abs(wr) + 2 * E * U * (a @ np.abs(wr)), B),
                  "dwr": (dz.T @ x, held_dz.T @ np.abs(x) + 2 * (T + 16) * U * (a.T @ np.abs(x)), U if f32 else B), "dbias": (dz.sum(0), off.sum(0) + (T + 16) * U * a.sum(0), U)}
        for n in want:
            ref, bound, last = bounds[n]
            if held is not None and n != "dx":
                ref = ref + f64(held[0 if n == "dwr" else 1])
            bound = bound * (1 + B) + last * np.abs(ref)
            dist = np.abs(f64(o[n]) - ref)
            assert np.isfinite(f64(o[n])).all() and (dist <= bound).all(), (n, float((dist / np.maximum(bound, 1e-300)).max()))


SHAPES = [(1, 64, 1, 1), (1, 4096, 8, 2), (3, 128, 2, 2), (17, 256, 7, 3), (64, 512, 64, 8), (65, 320, 65, 8), (130, 192, 128, 5), (257, 576, 60, 8), (100, 1024, 256, 8),
          (700, 640, 200, 12), (1999, 128, 16, 4), (515, 1216, 129, 2), (63, 64, 256, 256), (5000, 64, 33, 6), (64, 64, 40, 2), (2048, 64, 40, 3), (2049, 192, 70, 4), (4100, 320, 256, 8), (65, 192, 129, 8), (512, 448, 65, 5), (513, 448, 65, 5), (300, 704, 256, 8), (2100, 4096, 200, 8), (2600, 7168, 256, 8), (9000, 4096, 8, 2)]


@pytest.mark.parametrize("gating", [orc.SOFTMAX, orc.RENORM, orc.SIGMOID])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_values(moe, shape, gating):
    c = Case(*shape, gating, whole=True)
    c.check(c.run(moe))
    c = Case(*shape, gating, bias=False)
    c.check(c.run(moe, f32=False), f32=False)


@pytest.mark.parametrize("T,gating", [(40, orc.SOFTMAX), (150, orc.RENORM), (900, orc.SIGMOID), (2500, orc.SOFTMAX)])
def test_what_is_not_wanted_and_what_is_added_to(moe, T, gating):
    """dW_r in one piece and in several, that a last launch joins."""
    c = Case(T, 256, 20, 4, gating, whole=True)
    whole = c.run(moe)
    c.check(whole)
    for want in (("dx",), ("dwr",), ("dbias",), ("dx", "dbias"), ("dwr", "dbias")):
        o = c.run(moe, want=want)
        for n in ("dx", "dwr", "dbias"):
            assert torch.equal(o[n], whole[n]) if n in want else torch.isnan(o[n]).all(), (want, n)
    rng = np.random.default_rng(1)
    held = torch.from_numpy(rng.normal(size=(20, 256))).float(), torch.from_numpy(rng.normal(size=20)).float()
    c.check(c.run(moe, accumulate=True, held=held), held=held)
    held = held[0].to(torch.bfloat16), held[1]
    c.check(c.run(moe, f32=False, accumulate=True, held=held), f32=False, held=held)


def test_indices_outside_have_no_part(moe):
    for gating in (orc.SOFTMAX, orc.RENORM, orc.SIGMOID):
        for E in (20, 64):
            c = Case(40, 128, E, 4, gating, whole=True)
            c.idx[::3, 1], c.idx[::4, 2], c.idx[5] = -1, E, 2**31 - 1
            c.idx[6] = (-2**31, E + 1, 63 if E < 64 else 64, 300)
            c.g[5, 0], c.g[6, 2] = np.inf, NAN
            c.g[5, 1:], c.g[6, [0, 1, 3]] = 1, 1
            o = c.run(moe)
            c.g[5], c.g[6] = 0, 0
            c.check(o)


def test_masked_experts_and_infinities(moe):
    """A bias of minus infinity: an expert nobody chooses and that has no gradient.  A token with a NaN spoils its own dx and, as the sum says, dW_r."""
    c = Case(30, 192, 12, 2, orc.SOFTMAX, whole=True)
    c.bias[3] = -np.inf
    c.z[:, 3] = -np.inf
    c.idx = np.argsort(-c.z, axis=1, kind="stable")[:, :2].astype(np.int32)
    o = c.run(moe)
    assert (o["dwr"][3] == 0).all() and o["dbias"][3] == 0 and torch.isfinite(o["dx"]).all()
    c.check(o)
    c.g[4, 0] = NAN
    dx = c.run(moe)["dx"]
    assert torch.isnan(dx[4]).all() and torch.equal(dx[torch.arange(30) != 4], o["dx"][torch.arange(30) != 4])


def test_no_tokens(moe):
    z = Case(0, 64, 5, 2, orc.SOFTMAX, whole=True)
    o = z.run(moe)
    assert (o["dwr"] == 0).all() and (o["dbias"] == 0).all()
    held = full((5, 64), torch.float32, 2.0), full((5,), torch.float32, 3.0)
    o = z.run(moe, accumulate=True, held=held)
    assert torch.equal(o["dwr"], held[0]) and torch.equal(o["dbias"], held[1])


@pytest.mark.parametrize("gating", [orc.SOFTMAX, orc.RENORM, orc.SIGMOID])
def test_the_widest_rows(moe, gating):
    c = Case(3, 1 << 20, 5, 2, gating, whole=True)
    c.check(c.run(moe))


def test_nan_in_one_channel(moe):
    """Without logits in between a NaN of x reaches its column of dW_r and nothing else; neighbours of the router's rows in memory are not read."""
    c = Case(77, 192, 9, 2, orc.RENORM, whole=True)
    good = c.run(moe)
    wide = torch.full((c.wr.shape[0] + 128, 192), NAN, dtype=torch.bfloat16, device="cuda")
    wide[:9] = c.wr.cuda()
    c.x[5, 17] = NAN
    cfg = moe.MoEConfig.of(77, 192, 64, 9, 2, orc.RENORM)
    dx, dwr, dbias = full((77, 192)), full((9, 192), torch.float32), full((9,), torch.float32)
    moe.moe_route_backward(cfg, c.x.cuda(), wide[:9], None, *(torch.from_numpy(v).cuda() for v in (c.idx, c.w, c.g)), dx, dwr, dbias,
                           full((moe.route_backward_workspace_size(cfg),), torch.uint8, 255))
    assert torch.equal(dx, good["dx"]) and torch.equal(dbias, good["dbias"]) and torch.isnan(dwr[:, 17]).all()
    rest = torch.arange(192) != 17
    assert torch.equal(dwr[:, rest], good["dwr"][:, rest])


def test_the_same_every_time(moe):
    c = Case(900, 512, 96, 6, orc.SOFTMAX)
    a, b = c.run(moe), c.run(moe)
    assert all(torch.equal(a[n], b[n]) for n in a)
