"""fp64 numpy oracle of the operators over slots that may have no row, of dropout, and of the router's gradient (test infrastructure).

From the definitions, slot by slot: which slots have a row (an expert that is here, with room left), the rows' values, the way back, both gradients; the
Philox4x32-10 generator on Python's integers (Salmon, Moraes, Dror and Shaw, SC 2011); the gates' gradients (the paper's Eq. 1-2 and Sec. 3.4, differentiated).
"""
from __future__ import annotations

import numpy as np

LOW = 0xFFFFFFFF


def tables(idx, E, first=0, capacity=0):
    """idx [T, k] -> counts [E], offsets [E+1], row_of [T, k] (-1: none), src_of: the slot of every row."""
    T, k = idx.shape
    chose = [[] for _ in range(E)]
    for j, e in enumerate(idx.reshape(-1).tolist()):
        if first <= e < first + E:
            chose[e - first].append(j)
    taken = [c[:capacity] if capacity else c for c in chose]
    row_of = np.full(T * k, -1, np.int64)
    src_of = np.array([j for c in taken for j in c], np.int64)
    row_of[src_of] = np.arange(src_of.size)
    return np.array([len(c) for c in chose]), np.concatenate([[0], np.cumsum([len(c) for c in taken])]), row_of.reshape(T, k), src_of


def philox(key, counter, rounds=10):
    """key: two, counter: four 32-bit words -> four words."""
    k, x = list(key), list(counter)
    for _ in range(rounds):
        a, b = 0xD2511F53 * x[0], 0xCD9E8D57 * x[2]
        x = [(b >> 32) ^ x[1] ^ k[0], b & LOW, (a >> 32) ^ x[3] ^ k[1], a & LOW]
        k = [(k[0] + 0x9E3779B9) & LOW, (k[1] + 0xBB67AE85) & LOW]
    return x


def limit(p):
    return int(np.floor(p * 65536 + 0.5))


def keep(n, p, seed, offset):
    """The mask of elements 0 .. n - 1."""
    out = np.zeros((n + 7) // 8 * 8, bool)
    for b in range((n + 7) // 8):
        words = philox((seed & LOW, seed >> 32 & LOW), (b & LOW, b >> 32, offset & LOW, offset >> 32 & LOW))
        for j in range(8):
            out[8 * b + j] = (words[j // 2] >> 16 * (j % 2) & 0xFFFF) >= limit(p)
    return out[:n]


def dropped(v, p, seed, offset):
    if limit(p) == 0:
        return v
    return np.where(keep(v.size, p, seed, offset).reshape(v.shape), v * (65536 / (65536 - limit(p))), 0.0)


def scattered(v, row_of, w, R):
    """rows [R, d] (zero where no slot points), rows[row_of[t, i]] = w[t, i] v[t]."""
    out = np.zeros((R, v.shape[1]))
    for t, i in zip(*np.nonzero(row_of >= 0)):
        out[row_of[t, i]] = w[t, i] * v[t]
    return out


def gathered(rows, row_of, w):
    """[T, d]: sum_i w[t, i] rows[row_of[t, i]]."""
    out = np.zeros((row_of.shape[0], rows.shape[1]))
    for t, i in zip(*np.nonzero(row_of >= 0)):
        out[t] += w[t, i] * rows[row_of[t, i]]
    return out


def dots(v, rows, row_of):
    out = np.zeros(row_of.shape)
    for t, i in zip(*np.nonzero(row_of >= 0)):
        out[t, i] = v[t] @ rows[row_of[t, i]]
    return out


SOFTMAX, RENORM, SIGMOID = range(3)


def gate(z, idx, gating):
    """Gate weights [T, k] of logits z [T, E] at the chosen experts."""
    top = np.take_along_axis(z, idx, 1)
    if gating == SIGMOID:
        s = 1 / (1 + np.exp(-top))
        return s / s.sum(1, keepdims=True)
    of = z if gating == SOFTMAX else top
    m = of.max(1, keepdims=True)
    return np.exp(top - m) / np.exp(of - m).sum(1, keepdims=True)


def gate_backward(z, idx, w, g, gating):
    """dz [T, E].  Slots whose expert is outside 0 .. E - 1 are left out.  w: the gate weights (of the two normalised gates)."""
    T, E = z.shape
    dz = np.zeros_like(z)
    for t in range(T):
        own = [i for i in range(idx.shape[1]) if 0 <= idx[t, i] < E]
        if gating == SOFTMAX:
            p = np.exp(z[t] - z[t].max())
            p /= p.sum()
            c = sum(p[idx[t, i]] * g[t, i] for i in own)
            dz[t] = -p * c
            for i in own:
                dz[t, idx[t, i]] += p[idx[t, i]] * g[t, i]
        else:
            c = sum(w[t, i] * g[t, i] for i in own)
            for i in own:
                slope = 1 / (1 + np.exp(z[t, idx[t, i]])) if gating == SIGMOID else 1.0
                dz[t, idx[t, i]] += w[t, i] * (g[t, i] - c) * slope
    return dz
