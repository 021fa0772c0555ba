"""The training oracle against differences: every gradient it gives is the slope of its own forward pass.  No GPU is involved."""
import os
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from oracle import train_oracle as orc

STEP = 1e-5      # central differences: error STEP^2 * third derivative (~1e-10) and 1e-16 * value / STEP (~1e-11)


def _slope(f, a, at):
    keep = a[at]
    a[at] = keep + STEP
    up = f()
    a[at] = keep - STEP
    down = f()
    a[at] = keep
    return (up - down) / (2 * STEP)


@pytest.mark.parametrize("counts", [[3, 0, 4], [5], [0, 0, 1]])
def test_block_gradients_are_slopes(counts):
    rng = np.random.default_rng(3)
    E, R, d, F = len(counts), sum(counts), 6, 5
    off = np.concatenate([[0], np.cumsum(counts)])
    t = {"x": rng.normal(size=(R, d)), "wg": rng.normal(size=(E, F, d)), "wu": rng.normal(size=(E, F, d)), "wd": rng.normal(size=(E, d, F))}
    dy = rng.normal(size=(R, d))
    g, u, h, y = orc.block_forward(t["x"], off, t["wg"], t["wu"], t["wd"])
    o = orc.block_backward(t["x"], off, t["wg"], t["wu"], t["wd"], g, u, dy)
    assert np.allclose(o["h"], h)
    loss = lambda: float((orc.block_forward(t["x"], off, t["wg"], t["wu"], t["wd"])[3] * dy).sum())  # noqa: E731
    for name, grad in (("x", "dx"), ("wg", "dwg"), ("wu", "dwu"), ("wd", "dwd")):
        for at in list(np.ndindex(t[name].shape))[::3]:
            assert abs(_slope(loss, t[name], at) - o[grad][at]) < 1e-7 * max(1.0, abs(o[grad][at])), (name, at)
    for e, n in enumerate(counts):
        if n == 0:
            assert not o["dwg"][e].any() and not o["dwd"][e].any()


def test_combine_gradients_are_slopes():
    rng = np.random.default_rng(4)
    T, k, d = 4, 3, 5
    row_of = rng.permutation(T * k).reshape(T, k)
    p, w, dy = rng.normal(size=(T * k, d)), rng.normal(size=(T, k)), rng.normal(size=(T, d))
    dp, dw = orc.combine_backward(dy, p, row_of, w)
    loss = lambda: float((np.einsum("tk,tkd->td", w, p[row_of]) * dy).sum())  # noqa: E731
    for at in np.ndindex(p.shape):
        assert abs(_slope(loss, p, at) - dp[at]) < 1e-7
    for at in np.ndindex(w.shape):
        assert abs(_slope(loss, w, at) - dw[at]) < 1e-7


def test_adapter_is_a_sum_of_two_projections():
    rng = np.random.default_rng(5)
    x, w, a, b = rng.normal(size=(5, 4)), rng.normal(size=(3, 4)), rng.normal(size=(2, 2, 4)), rng.normal(size=(2, 3, 2))
    ids = np.array([1, -1, 0, 2, 1])
    y = orc.adapter_linear(x, w, a, b, np.array([0.5, 2.0]), ids)
    for t, m in enumerate(ids):
        full = w + (np.array([0.5, 2.0])[m] * b[m] @ a[m] if 0 <= m < 2 else 0)
        assert np.allclose(y[t], full @ x[t])
