"""SiLU and its slope as the training operators compute them, gate by gate: x, dy and the weights are unit vectors and ones, so that every h, dg and du stands
alone in a result.

What s = rcp(1 + exp2(-g log2 e)) in fp32 may be off by (f = 2^-24): the exponent's product and its constant, f each, are 2 |g| f of the exponential, which
itself is off by 2 f (1 ulp); the sum's rounding f; the reciprocal 2 f (1 ulp); and an error of the exponential reaches s by (1 - s):
    ds = ((2 |g| + 2) (1 - s) + 3) f s + 2^-126            (s below the smallest normal number may be zero)
    h = g s u                |g| ds u + 2 f |h|
    du = dh g s              the same
    dg = dh u (s + g s (1 - s))     ds + |g| ds (1 - s) + |g| s (ds + f) + 5 f (s + |g| s (1 - s)), times |dh u|
and each is rounded to bf16 once, 2^-8 of itself.  Products of second order: a factor 1 + 2^-6."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as orc

pytestmark = pytest.mark.gpu

B, F32, TINY, SLACK = 2.0 ** -8, 2.0 ** -24, 2.0 ** -126, 1 + 2.0 ** -6
N = 64


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_23911_amd as m
    m.lib()
    return m


def _gates():
    """4096 bf16 numbers: both signs, dense to 100, about the slope's zero near -1.278, next to nothing, and zeros."""
    rng = np.random.default_rng(0)
    v = np.concatenate([np.linspace(-100, 100, 2001), rng.uniform(-8, 8, 1000), np.linspace(-1.3, -1.25, 95), 10.0 ** rng.uniform(-30, 0, 600) * rng.choice([-1, 1], 600),
                        -rng.uniform(80, 90, 300), [0.0, -0.0, -1e4, 1e4], rng.normal(size=96)])
    assert v.size == N * N
    return torch.from_numpy(v).to(torch.bfloat16).view(N, N)


def _ds(g, s):
    return ((2 * np.abs(g) + 2) * (1 - s) + 3) * F32 * s + TINY


def _check(got, want, err, what):
    got = got.detach().cpu().double().numpy()
    off = np.abs(got - want) - (err + B * np.abs(want)) * SLACK
    worst = np.unravel_index(np.argmax(off), off.shape)
    assert np.isfinite(got).all() and off[worst] <= 0, (what, float(got[worst]), float(want[worst]), float(err[worst]))


def test_gate_by_gate(moe):
    gates = _gates()
    g = gates.double().numpy()
    s, act = orc.sigmoid(g), orc.silu(g)
    bf, dev = torch.bfloat16, "cuda"
    eye, ones = torch.eye(N, dtype=bf, device=dev), torch.ones((N, N), dtype=bf, device=dev)
    off = torch.tensor([0, N], dtype=torch.int32, device=dev)
    cfg = moe.MoEConfig.of(N, N, N, 1, 1)
    buf = lambda dtype=bf: torch.full((N, N), float("nan"), dtype=dtype, device=dev)  # noqa: E731
    wg = gates.T.contiguous().cuda().view(1, N, N)
    w1 = ones.view(1, N, N)
    # forward: g[r, f] = Wg[f, r], u = 1
    kept, u, h, y = buf(), buf(), buf(), buf()
    ws = torch.empty(max(moe.ffn_workspace_size(cfg), moe.ffn_backward_workspace_size(cfg)), dtype=torch.uint8, device=dev)
    moe.moe_grouped_ffn_train(cfg, eye, off, wg, w1, w1, kept, u, h, y, ws)
    assert torch.equal(kept, gates.cuda()) and (u == 1).all()
    e_act = np.abs(g) * _ds(g, s) + 2 * F32 * np.abs(act)
    _check(h, act, e_act, "h")
    # backward: dh = 1; dWg[f, r] = dg[r, f], dWu[f, r] = du[r, f], dWd[r, f] = h[r, f]
    dw = [buf(torch.float32).view(1, N, N) for _ in range(3)]
    moe.moe_grouped_ffn_backward(cfg, eye, off, wg, w1, w1, kept, u, eye, None, *dw, ws)
    a = np.abs(g) * s
    e_slope = _ds(g, s) * (1 + np.abs(g) * (1 - s) + a) + F32 * a + 5 * F32 * (s + a * (1 - s))
    _check(dw[0][0].T, orc.silu_slope(g), e_slope, "dg")
    _check(dw[1][0].T, act, e_act, "du")
    _check(dw[2][0], act, e_act, "h again")
