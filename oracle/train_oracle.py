"""fp64 numpy oracle of the layer's training operators, from the definitions (test infrastructure).

Gated block (the paper's Eq. 4, Sec. 2.1) over expert-contiguous rows: h = SiLU(x Wg^T) (.) (x Wu^T), y = h Wd^T; its
gradients by the chain rule.  Weighted combine (Eq. 3): y_t = sum_i w_ti p_row(t,i), and its gradients.  Low-rank adapters beside a
projection: y_t = x_t W^T + s_a (x_t A_a^T) B_a^T.
Every function also gives, where asked, the same sums over absolute values: what a bound on rounding errors is made of.
"""
from __future__ import annotations

import numpy as np


def sigmoid(g):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-g))


def silu(g):
    return g * sigmoid(g)


def silu_slope(g):
    s = sigmoid(g)
    return s * (1.0 + g * (1.0 - s))


def block_forward(x, offsets, wg, wu, wd):
    """x [R, d], offsets [E+1], wg, wu [E, F, d], wd [E, d, F] -> g, u, h [R, F], y [R, d]."""
    R, F = x.shape[0], wg.shape[1]
    g, u = np.zeros((R, F)), np.zeros((R, F))
    y = np.zeros_like(x)
    for e in range(wg.shape[0]):
        r = slice(offsets[e], offsets[e + 1])
        g[r], u[r] = x[r] @ wg[e].T, x[r] @ wu[e].T
        y[r] = (silu(g[r]) * u[r]) @ wd[e].T
    return g, u, silu(g) * u, y


def block_backward(x, offsets, wg, wu, wd, g, u, dy):
    """Gradients at g and u: dict of dh, dg, du, h [R, F], dx [R, d], dwg, dwu [E, F, d], dwd [E, d, F]."""
    E = wg.shape[0]
    o = {"dh": np.zeros_like(g), "dx": np.zeros_like(x), "dwg": np.zeros_like(wg), "dwu": np.zeros_like(wu), "dwd": np.zeros_like(wd)}
    for e in range(E):
        r = slice(offsets[e], offsets[e + 1])
        o["dh"][r] = dy[r] @ wd[e]
    o["dg"], o["du"], o["h"] = o["dh"] * u * silu_slope(g), o["dh"] * silu(g), silu(g) * u
    for e in range(E):
        r = slice(offsets[e], offsets[e + 1])
        o["dx"][r] = o["dg"][r] @ wg[e] + o["du"][r] @ wu[e]
        o["dwg"][e], o["dwu"][e], o["dwd"][e] = o["dg"][r].T @ x[r], o["du"][r].T @ x[r], dy[r].T @ o["h"][r]
    return o


def combine_backward(dy, p, row_of, w):
    """dy [T, d], p [R, d], row_of [T, k], w [T, k] -> dp [R, d], dw [T, k]."""
    dp = np.zeros_like(p)
    dw = np.zeros_like(w)
    for t in range(w.shape[0]):
        for i in range(w.shape[1]):
            dp[row_of[t, i]] = w[t, i] * dy[t]
            dw[t, i] = dy[t] @ p[row_of[t, i]]
    return dp, dw


def adapter_linear(x, w, a, b, scale, adapter_of, base=None):
    """x [T, K], w [N, K], a [n, r, K], b [n, N, r], scale [n], adapter_of [T] (outside 0..n-1: none) -> y [T, N]."""
    y = x @ w.T
    for t in range(x.shape[0]):
        m = adapter_of[t]
        if 0 <= m < a.shape[0]:
            y[t] += scale[m] * (b[m] @ (a[m] @ x[t]))
    return y if base is None else y + base
