"""Low-rank adapters beside a shared projection on the GPU, through the binding, against the fp64 oracle.

Bounds, element by element (b = 2^-8 for bf16, f = 2^-24 for fp32), on y = base + x W^T + scale B (A x):
  rounding of y                b |y|
  fp32 sum of W's part         K f |x||W|
  v = scale A x in fp32        (K + 9) f scale |A||x|  (sum, up to eight pieces, scale), then two bf16 numbers: b^2 |v|;  both times |B|
  fp32 sum with B's part       (K + 2 rank) f scale |B||v|
The gated pair: |d(silu(g) u)| <= 1.1 |u| dg + |silu(g)| du, and 16 f for the sigmoid in fp32.  Second order terms: a factor 1 + 2^-6."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))

from oracle import train_oracle as orc

pytestmark = pytest.mark.gpu

B, F32, SLACK = 2.0 ** -8, 2.0 ** -24, 1 + 2.0 ** -6


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


def _ids(kind, T, n, rng):
    if kind == "none":
        return np.full(T, -1)
    if kind == "one":
        return np.full(T, n - 1)
    if kind == "requests":          # contiguous runs, some without
        return np.repeat(rng.integers(-1, n, size=T), rng.integers(1, 60, size=T))[:T]
    if kind == "own":               # every token another request
        return rng.permutation(np.arange(T) % n)
    ids = rng.integers(-1, n, size=T)
    ids[rng.random(T) < 0.2] = rng.choice([n, n + 1, 2 ** 31 - 1, -2 ** 31, -7])      # outside: none
    return ids


class Case:
    def __init__(self, T, N, K, n, rank, kind, seed=0, two=False, base=False, scale=True):
        rng = np.random.default_rng([seed, T, N, K, n, rank])
        self.T, self.N, self.K, self.n, self.rank = T, N, K, n, rank
        m = 2 if two else 1
        self.x, self.base = _bf16(rng, (T, K)), _bf16(rng, (T, N), 2.0) if base else None
        self.w = [_bf16(rng, (N, K), K ** -0.5) for _ in range(m)]
        self.a = [_bf16(rng, (n, rank, K), K ** -0.5) for _ in range(m)]
        self.b = [_bf16(rng, (n, N, rank), rank ** -0.5) for _ in range(m)]
        self.scale = torch.from_numpy((rng.random(n) * 2 - 0.5).astype(np.float32)) if scale else None
        self.ids = _ids(kind, T, n, rng).astype(np.int32)

    def gpu(self, moe):
        self.cfg = moe.AdapterConfig.of(self.T, self.N, self.K, self.n, self.rank)
        c = lambda t: None if t is None else t.cuda()  # noqa: E731
        self.d = {"x": c(self.x), "base": c(self.base), "w": [c(t) for t in self.w], "a": [c(t) for t in self.a], "b": [c(t) for t in self.b],
                  "scale": c(self.scale), "ids": torch.from_numpy(self.ids).cuda()}
        self.ws = torch.full((moe.adapter_workspace_size(self.cfg),), 255, dtype=torch.uint8, device="cuda")       # NaN wherever it is read unwritten
        self.y = torch.full((self.T, self.N), float("nan"), dtype=torch.bfloat16, device="cuda")
        return self

    def linear(self, moe, shared=True, y=None, base="own"):
        d = self.d
        y = self.y if y is None else y
        moe.moe_adapter_linear(self.cfg, d["x"], d["w"][0] if shared else None, d["a"][0], d["b"][0], d["scale"], d["ids"], y, self.ws,
                               base=d["base"] if isinstance(base, str) else base)
        torch.cuda.synchronize()
        return y

    def gated(self, moe):
        d = self.d
        moe.moe_adapter_gated_up(self.cfg, d["x"], *d["w"], *d["a"], *d["b"], d["scale"], d["ids"], self.y, self.ws)
        torch.cuda.synchronize()
        return self.y

    def want(self, m, shared=True):
        """(y, bound before y's own rounding) of projection m, without base."""
        x, w, a, b = _np(self.x), _np(self.w[m]) * bool(shared), _np(self.a[m]), _np(self.b[m])
        s = np.ones(self.n) if self.scale is None else _np(self.scale)
        y = orc.adapter_linear(x, w, a, b, s, self.ids)
        e = self.K * F32 * (np.abs(x) @ np.abs(w).T)
        for t, i in enumerate(self.ids):
            if 0 <= i < self.n:
                v = np.abs(s[i] * (a[i] @ x[t]))
                ev = (self.K + 9) * F32 * np.abs(s[i]) * (np.abs(a[i]) @ np.abs(x[t])) + B * B * v
                e[t] += np.abs(b[i]) @ (ev + (self.K + 2 * self.rank) * F32 * v)
        return y, e


def _close(got, want, bound, what):
    got = _np(got)
    assert np.isfinite(got).all(), what
    assert (np.abs(got - want) <= bound * SLACK).all(), (what, float((np.abs(got - want) / np.maximum(bound, 1e-300)).max()))


# every token count around the kernels' blocks, ranks that end inside a fragment, widths that end inside a tile, all kinds of ids
CASES = [
    (1, 64, 64, 1, 8, "one"), (1, 448, 1024, 3, 16, "own"), (1, 128, 192, 2, 16, "none"), (15, 192, 320, 4, 24, "mixed"), (16, 320, 128, 16, 40, "own"),
    (17, 64, 2048, 5, 128, "mixed"), (33, 256, 704, 33, 64, "own"), (48, 704, 256, 64, 64, "own"), (64, 128, 4160, 7, 8, "requests"), (64, 576, 192, 64, 32, "own"),
    (65, 192, 256, 3, 16, "mixed"), (100, 320, 448, 100, 72, "own"), (130, 448, 128, 9, 128, "requests"), (257, 1088, 192, 2, 32, "requests"),
    (300, 64, 64, 40, 8, "mixed"), (513, 640, 320, 6, 56, "none"), (700, 192, 576, 1, 16, "one"),
]


@pytest.mark.parametrize("T,N,K,n,rank,kind", CASES)
@pytest.mark.parametrize("base", [False, True])
def test_linear(moe, T, N, K, n, rank, kind, base):
    print("linear", T, N, K, n, rank, kind, base, flush=True)
    c = Case(T, N, K, n, rank, kind, base=base).gpu(moe)
    y, e = c.want(0)
    if base:
        y = y + _np(c.base)
        e = e + F32 * np.abs(y)
    _close(c.linear(moe), y, e + B * np.abs(y), "y")


@pytest.mark.parametrize("T,N,K,n,rank,kind", CASES)
def test_gated(moe, T, N, K, n, rank, kind):
    print("gated", T, N, K, n, rank, kind, flush=True)
    c = Case(T, N, K, n, rank, kind, seed=1, two=True, scale=T % 2 == 0).gpu(moe)
    (g, eg), (u, eu) = c.want(0), c.want(1)
    act = orc.silu(g)
    _close(c.gated(moe), act * u, np.abs(u) * (1.1 * eg + 16 * F32 * np.abs(act)) + np.abs(act) * eu + B * np.abs(act * u), "h")


@pytest.mark.parametrize("T", [3, 50, 90, 400])
def test_wide_tiles_and_many_workgroups(moe, T):
    """Enough output for 256 workgroups of the largest tile, and a vocabulary of rows that one adapter list does not hold."""
    c = Case(T, 8192, 128, 50, 16, "mixed", two=True, seed=2).gpu(moe)
    (g, eg), (u, eu) = c.want(0), c.want(1)
    act = orc.silu(g)
    _close(c.gated(moe), act * u, np.abs(u) * (1.1 * eg + 16 * F32 * np.abs(act)) + np.abs(act) * eu + B * np.abs(act * u), "h")


@pytest.mark.parametrize("T,N,rank,kind,two", [(700, 8192, 128, "mixed", True), (700, 8192, 24, "requests", True), (1400, 8192, 72, "requests", False),
                                               (1400, 8192, 8, "own", False), (300, 8192, 104, "own", False), (200, 14336, 72, "mixed", True), (200, 28672, 16, "requests", False)])
def test_large_tiles(moe, T, N, rank, kind, two):
    """Prompts with enough tiles for one launch of the projection and its adapters, ranks of one and two pieces, blocks of one adapter and of many."""
    c = Case(T, N, 192, 9, rank, kind, two=two, seed=5).gpu(moe)
    g, eg = c.want(0)
    if not two:
        _close(c.linear(moe), g, eg + B * np.abs(g), "y")
        return
    u, eu = c.want(1)
    act = orc.silu(g)
    _close(c.gated(moe), act * u, np.abs(u) * (1.1 * eg + 16 * F32 * np.abs(act)) + np.abs(act) * eu + B * np.abs(act * u), "h")


@pytest.mark.parametrize("T,kind,N", [(5, "mixed", 320), (200, "requests", 320), (300, "mixed", 8192), (1400, "requests", 8192), (200, "mixed", 28672)])
def test_without_the_shared_projection(moe, T, kind, N):
    c = Case(T, N, 192, 6, 16, kind, base=True).gpu(moe)
    y, e = c.want(0, shared=False)
    y = y + _np(c.base)
    _close(c.linear(moe, shared=False), y, e + B * np.abs(y) + F32 * np.abs(y), "y")
    alone = c.linear(moe, shared=False, base=None)
    assert not alone[torch.from_numpy((c.ids < 0) | (c.ids >= c.n)).cuda()].any()


@pytest.mark.parametrize("T", [7, 150])
def test_base_may_be_the_result(moe, T):
    c = Case(T, 256, 128, 4, 8, "mixed", base=True).gpu(moe)
    want = c.linear(moe).clone()
    y = c.d["base"].clone()
    c.linear(moe, y=y, base=y)
    assert torch.equal(y, want)


@pytest.mark.parametrize("T,N", [(9, 192), (120, 192), (300, 192), (300, 8192), (1400, 8192), (200, 28672)])
def test_a_token_s_result_is_its_own(moe, T, N):
    """Tokens and adapters that hold NaN or infinities reach nobody else's result."""
    c = Case(T, N, 256, 5, 24, "mixed", seed=3)
    c.ids[:3] = [2, 0, 2]
    clean = Case(T, N, 256, 5, 24, "mixed", seed=3)
    clean.ids[:] = c.ids
    c.x[1] = float("nan")
    c.a[0][2] = float("inf")
    c.b[0][2, 5] = float("nan")
    got, want = c.gpu(moe).linear(moe), clean.gpu(moe).linear(moe)
    hurt = torch.from_numpy(c.ids == 2).cuda()
    hurt[1] = True
    assert torch.equal(got[~hurt], want[~hurt]) and not torch.isfinite(got[hurt][:, 5]).any()


def test_results_do_not_depend_on_the_company(moe):
    """The same token alone and in a batch of the same kernel: bit for bit, whatever adapters the others have."""
    c = Case(60, 256, 512, 30, 16, "own", seed=4).gpu(moe)
    first = c.linear(moe).clone()
    c.d["ids"][1:] = -1
    c.linear(moe)
    assert torch.equal(c.y[0], first[0])
