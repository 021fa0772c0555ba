"""The gated block for training and the combine's gradients on the GPU, through the binding, against the fp64 oracle.

Bounds, element by element, for bf16 results of fp32 sums of n products (unit roundoffs b = 2^-8 for bf16, f = 2^-24 for fp32):
  one rounding of the result         b |y|
  the fp32 sum, in any order         n f sum |a||c|      (products of two bf16 numbers are exact in fp32)
  operands that were rounded to bf16 b sum |a||c|        (dg, du, h in the products that follow)
  sigmoid in fp32                    its exponential, sum and reciprocal: 8 f relative of s, hence 16 f (s + |act|) of the slope
A second order term is covered by (1 + 2^-6) on the whole."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))

from oracle import train_oracle as orc

pytestmark = pytest.mark.gpu

B, F32 = 2.0 ** -8, 2.0 ** -24
SLACK = 1 + 2.0 ** -6


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_23911_amd as m
    m.lib()
    return m


def _bf16(rng, shape, std=1.0):
    return torch.from_numpy(rng.normal(size=shape) * std).to(torch.bfloat16)


def _np(t):
    return t.detach().cpu().double().numpy()


def _close(got, want, bound, what):
    got = _np(got)
    off = np.abs(got - want) - bound * SLACK
    assert np.isfinite(got).all(), what
    assert (off <= 0).all(), (what, float((np.abs(got - want) / np.maximum(bound, 1e-300)).max()))


class Block:
    def __init__(self, counts, d, F, seed=0, tail=0):
        rng = np.random.default_rng(seed)
        self.E, self.d, self.F, self.n = len(counts), d, F, sum(counts)
        self.R = self.n + tail
        self.off = np.concatenate([[0], np.cumsum(counts)])
        self.host = {"x": _bf16(rng, (self.R, d)), "wg": _bf16(rng, (self.E, F, d), d ** -0.5), "wu": _bf16(rng, (self.E, F, d), d ** -0.5),
                     "wd": _bf16(rng, (self.E, d, F), F ** -0.5), "g": _bf16(rng, (self.R, F), 1.5), "u": _bf16(rng, (self.R, F)),
                     "dy": _bf16(rng, (self.R, d), 0.1)}

    def to_gpu(self, moe):
        self.dev = {n: t.cuda() for n, t in self.host.items()}
        self.offsets = torch.from_numpy(self.off.astype(np.int32)).cuda()
        self.cfg = moe.MoEConfig.of(self.R, self.d, self.F, self.E, 1)
        return self

    def forward(self, moe, fill=0.0):
        v = self.dev
        o = {n: torch.full((self.R, w), fill, dtype=torch.bfloat16, device="cuda") for n, w in (("g", self.F), ("u", self.F), ("h", self.F), ("y", self.d))}
        ws = torch.empty(moe.ffn_workspace_size(self.cfg), dtype=torch.uint8, device="cuda")
        moe.moe_grouped_ffn_train(self.cfg, v["x"], self.offsets, v["wg"], v["wu"], v["wd"], o["g"], o["u"], o["h"], o["y"], ws)
        torch.cuda.synchronize()
        return o

    def grads(self, dtype=torch.bfloat16, fill=0.0):
        return {"dx": torch.full((self.R, self.d), fill, dtype=torch.bfloat16, device="cuda"),
                **{n: torch.full(self.host[n[1:]].shape, fill, dtype=dtype, device="cuda") for n in ("dwg", "dwu", "dwd")}}

    def backward(self, moe, o, accumulate=False, ws=None):
        v = self.dev
        if ws is None:
            ws = torch.empty(moe.ffn_backward_workspace_size(self.cfg), dtype=torch.uint8, device="cuda")
        moe.moe_grouped_ffn_backward(self.cfg, v["x"], self.offsets, v["wg"], v["wu"], v["wd"], v["g"], v["u"], v["dy"], o["dx"], o["dwg"], o["dwu"],
                                     o["dwd"], ws, accumulate=accumulate)
        return o

    def oracle(self):
        """(values, bounds) of the backward pass, before the results' own rounding."""
        h = {n: _np(t) for n, t in self.host.items()}
        n = self.n
        x, g, u, dy = (h[t][:n] for t in ("x", "g", "u", "dy"))
        o = orc.block_backward(x, self.off, h["wg"], h["wu"], h["wd"], g, u, dy)
        s, act = orc.sigmoid(g), np.abs(orc.silu(g))
        e_dh = np.zeros_like(g)
        for e in range(self.E):
            r = slice(self.off[e], self.off[e + 1])
            e_dh[r] = self.d * F32 * (np.abs(dy[r]) @ np.abs(h["wd"][e]))
        e_dg = B * np.abs(o["dg"]) + np.abs(u) * (e_dh * np.abs(orc.silu_slope(g)) + 16 * F32 * np.abs(o["dh"]) * (s + act)) + 4 * F32 * np.abs(o["dg"])
        e_du = B * np.abs(o["du"]) + e_dh * act + 12 * F32 * np.abs(o["du"])
        e_h = B * np.abs(o["h"]) + 12 * F32 * np.abs(o["h"])
        b = {"dx": np.zeros_like(x), "dwg": np.zeros_like(h["wg"]), "dwu": np.zeros_like(h["wu"]), "dwd": np.zeros_like(h["wd"])}
        for e in range(self.E):
            r = slice(self.off[e], self.off[e + 1])
            k = (self.off[e + 1] - self.off[e]) * F32
            wg, wu, ax, ady = np.abs(h["wg"][e]), np.abs(h["wu"][e]), np.abs(x[r]), np.abs(dy[r])
            adg, adu, ah = np.abs(o["dg"][r]), np.abs(o["du"][r]), np.abs(o["h"][r])
            b["dx"][r] = (e_dg[r] + 2 * self.F * F32 * adg) @ wg + (e_du[r] + 2 * self.F * F32 * adu) @ wu
            b["dwg"][e] = (e_dg[r] + k * adg).T @ ax
            b["dwu"][e] = (e_du[r] + k * adu).T @ ax
            b["dwd"][e] = ady.T @ (e_h[r] + k * ah)
        return o, b


# row counts around the tiles' and steps' borders; widths that end inside a tile; empty experts at the ends and in the middle
SHAPES = [
    ([1], 64, 64), ([2, 0, 1], 128, 64), ([0, 65, 0, 63, 64], 320, 448), ([300, 1, 0, 257], 192, 640), ([128] * 4, 256, 512),
    ([700], 448, 320), ([255, 256, 513], 512, 192), ([5, 17, 0, 33, 1, 90, 2], 1088, 704),
    ([(7 * e) % 5 * (e % 3) for e in range(256)], 64, 128), ([0] * 130 + [200] + [0] * 124, 128, 64),        # as many experts as there may be, most without rows
    ([3], 128, 2112), ([40, 0, 129], 192, 1984),       # dx's sum is cut into pieces, of which the last is shorter
]


# enough results for the large tiles: of both projections, of dh (wide F) and of dx (wide d), with whole and ragged blocks and an expert without rows
LARGE = [([500, 0, 1000, 13], 512, 8192), ([700, 259, 512], 8192, 448), ([120, 0, 140, 128, 257], 1024, 1088)]


@pytest.mark.parametrize("counts,d,F", SHAPES + LARGE)
def test_forward_keeps_the_projections(moe, counts, d, F):
    print("forward", counts, d, F, flush=True)
    b = Block(counts, d, F).to_gpu(moe)
    o = b.forward(moe)
    h = {n: _np(t) for n, t in b.host.items()}
    g, u, hh, y = orc.block_forward(h["x"], b.off, h["wg"], h["wu"], h["wd"])
    eg, eu, ey = np.zeros_like(g), np.zeros_like(u), np.zeros_like(y)
    for e in range(b.E):
        r = slice(b.off[e], b.off[e + 1])
        eg[r], eu[r] = d * F32 * (np.abs(h["x"][r]) @ np.abs(h["wg"][e]).T), d * F32 * (np.abs(h["x"][r]) @ np.abs(h["wu"][e]).T)
    _close(o["g"], g, eg + B * np.abs(g), "g")
    _close(o["u"], u, eu + B * np.abs(u), "u")
    eh = np.abs(u) * (1.1 * eg + 16 * F32 * np.abs(orc.silu(g))) + np.abs(orc.silu(g)) * eu + B * np.abs(hh)     # |SiLU'| < 1.1
    _close(o["h"], hh, eh, "h")
    for e in range(b.E):
        r = slice(b.off[e], b.off[e + 1])
        ey[r] = (eh[r] + F * F32 * np.abs(hh[r])) @ np.abs(h["wd"][e]).T
    _close(o["y"], y, ey + B * np.abs(y), "y")


@pytest.mark.parametrize("counts,d,F", SHAPES + LARGE)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_backward(moe, counts, d, F, dtype):
    print("backward", counts, d, F, dtype, flush=True)
    b = Block(counts, d, F, seed=1).to_gpu(moe)
    got = b.backward(moe, b.grads(dtype, fill=float("nan")))
    torch.cuda.synchronize()
    want, bound = b.oracle()
    for n in ("dx", "dwg", "dwu", "dwd"):
        r = B if got[n].dtype == torch.bfloat16 else F32
        _close(got[n], want[n], bound[n] + r * np.abs(want[n]), n)
    for e, n in enumerate(counts):
        if n == 0:
            assert not got["dwg"][e].any() and not got["dwu"][e].any() and not got["dwd"][e].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_weight_gradients_are_added(moe, dtype):
    b = Block([70, 0, 33], 128, 192, seed=2).to_gpu(moe)
    once = b.backward(moe, b.grads(dtype))
    both = b.grads(dtype, fill=0.5)
    b.backward(moe, both, accumulate=True)
    torch.cuda.synchronize()
    want, bound = b.oracle()
    for n in ("dwg", "dwu", "dwd"):
        r = B if dtype == torch.bfloat16 else F32
        _close(both[n], want[n] + 0.5, bound[n] + r * np.abs(want[n] + 0.5) + F32 * np.abs(want[n]), n)
    assert torch.equal(both["dx"], once["dx"])
    assert (both["dwg"][1] == 0.5).all()


@pytest.mark.parametrize("counts,d,F", [([65, 3, 130], 192, 320), ([65, 3, 1430], 512, 8192), ([65, 3, 1430], 8192, 512)])
def test_rows_of_one_expert_do_not_reach_another(moe, counts, d, F):
    """Rows that hold NaN: only their own expert's results have any, although tiles and steps end inside its neighbours."""
    b = Block(counts, d, F, seed=3)
    for n in ("x", "g", "u", "dy"):
        b.host[n][65:68] = float("nan")
    b.to_gpu(moe)
    got = b.backward(moe, b.grads())
    fwd = b.forward(moe)
    torch.cuda.synchronize()
    for n in ("dwg", "dwu", "dwd"):
        assert torch.isfinite(got[n][0]).all() and torch.isfinite(got[n][2]).all() and torch.isnan(got[n][1]).all(), n
    for t in (got["dx"], fwd["g"], fwd["h"], fwd["y"]):
        assert torch.isfinite(t[:65]).all() and torch.isfinite(t[68:]).all() and torch.isnan(t[65:68]).all()


def test_gates_far_from_zero(moe):
    """SiLU and its slope where exp(-g) overflows and where it vanishes, and at zero: the formula's limits, nothing that is not finite."""
    b = Block([70, 58], 64, 64, seed=6)
    far = torch.tensor([-1e30, -1e4, -100.0, -88.5, -50.0, -0.0, 0.0, 50.0, 88.5, 100.0, 1e4, 1e30]).to(torch.bfloat16)
    b.host["g"][:] = far[torch.arange(128 * 64) % 12].view(128, 64)
    b.to_gpu(moe)
    got = b.backward(moe, b.grads(torch.float32, fill=float("nan")))
    torch.cuda.synchronize()
    want, bound = b.oracle()
    for n in ("dx", "dwg", "dwu", "dwd"):
        r = B if got[n].dtype == torch.bfloat16 else F32
        _close(got[n], want[n], bound[n] + r * np.abs(want[n]) + 1e-30, n)      # s below the smallest normal number may be zero


@pytest.mark.parametrize("F", [192, 2112])
def test_rows_behind_the_last_expert_stay(moe, F):
    b = Block([40, 25], 128, F, seed=4, tail=50)
    for n in ("x", "g", "u", "dy"):
        b.host[n][b.n:] = float("nan")
    b.to_gpu(moe)
    got = b.backward(moe, b.grads(fill=7.0))
    fwd = b.forward(moe, fill=7.0)
    torch.cuda.synchronize()
    for t in (got["dx"], fwd["g"], fwd["u"], fwd["h"], fwd["y"]):
        assert (t[b.n:] == 7.0).all() and torch.isfinite(t).all()
    assert all(torch.isfinite(got[n]).all() for n in ("dwg", "dwu", "dwd"))


def test_gradients_that_are_not_wanted(moe):
    b = Block([33, 90], 128, 256, seed=5).to_gpu(moe)
    all_of = b.backward(moe, b.grads())
    for keep in ("dx", "dwg", "dwu", "dwd"):
        o = {n: (t if n == keep else None) for n, t in b.grads().items()}
        b.backward(moe, o)
        assert torch.equal(o[keep], all_of[keep]), keep


def test_no_rows_at_all(moe):
    cfg = moe.MoEConfig.of(0, 128, 64, 3, 1)
    w = {n: torch.full(s, 3.0, dtype=torch.bfloat16, device="cuda") for n, s in (("g", (3, 64, 128)), ("u", (3, 64, 128)), ("d", (3, 128, 64)))}
    z = lambda c: torch.empty((0, c), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    ws = torch.empty(moe.ffn_backward_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    dw = {n: torch.full_like(t, 5.0) for n, t in w.items()}
    args = (cfg, z(128), off, w["g"], w["u"], w["d"], z(64), z(64), z(128), z(128), dw["g"], dw["u"], dw["d"], ws)
    moe.moe_grouped_ffn_backward(*args, accumulate=True)
    assert all((t == 5.0).all() for t in dw.values())
    moe.moe_grouped_ffn_backward(*args)
    assert not any(t.any() for t in dw.values())


@pytest.mark.parametrize("T,k,E,d", [(1, 1, 1, 64), (3, 2, 4, 192), (37, 8, 16, 2112), (5, 13, 16, 4096), (200, 4, 7, 704), (9, 7, 7, 2048)])
def test_combine_backward(moe, T, k, E, d):
    rng = np.random.default_rng(T)
    row_of = rng.permutation(T * k).reshape(T, k).astype(np.int32)
    dy, p = _bf16(rng, (T, d), 0.1), _bf16(rng, (T * k, d))
    w = torch.from_numpy(rng.random((T, k)).astype(np.float32))
    cfg = moe.MoEConfig.of(T, d, 64, E, k)
    dp = torch.full((T * k, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    dw = torch.full((T, k), float("nan"), dtype=torch.float32, device="cuda")
    pg = p.cuda()
    moe.moe_combine_backward(cfg, dy.cuda(), pg, torch.from_numpy(row_of).cuda(), w.cuda(), dp, dw)
    torch.cuda.synchronize()
    want_p, want_w = orc.combine_backward(_np(dy), _np(p), row_of, _np(w))
    _close(dp, want_p, (B + F32) * np.abs(want_p), "dp")
    flat = np.abs(_np(dy))[:, None, :] * np.abs(_np(p))[row_of]
    _close(dw, want_w, d * F32 * flat.sum(2) + F32 * np.abs(want_w), "dw")
    # in place: the rows' gradient over the rows themselves
    dw2 = torch.empty_like(dw)
    moe.moe_combine_backward(cfg, dy.cuda(), pg, torch.from_numpy(row_of).cuda(), w.cuda(), pg, dw2)
    torch.cuda.synchronize()
    assert torch.equal(pg, dp) and torch.equal(dw2, dw)
