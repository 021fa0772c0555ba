"""Checks of oracle/token_oracle.py: the generator's published answers, gradients against differences, tables by hand.  No GPU."""
import numpy as np
import pytest

from oracle import token_oracle as orc


def test_philox_known_answers():
    """The answers that the generator's authors give for ten rounds: all zeros, all ones, and digits of pi."""
    ones = 0xFFFFFFFF
    assert orc.philox((0, 0), (0, 0, 0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert orc.philox((ones, ones), (ones,) * 4) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert orc.philox((0xA4093822, 0x299F31D0), (0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344)) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_masks():
    n = 1 << 16
    for p in (0.1, 0.5, 0.9):
        m = orc.keep(n, p, 12345, 6)
        assert abs(m.mean() - (1 - p)) < 5 * (p * (1 - p) / n) ** 0.5            # five standard deviations
        assert not np.array_equal(m, orc.keep(n, p, 12345, 7)) and not np.array_equal(m, orc.keep(n, p, 12346, 6))
        assert np.array_equal(m[:1001], orc.keep(1001, p, 12345, 6))
    assert orc.keep(100, 0.0, 1, 2).all() and orc.limit(65535 / 65536) == 65535
    v = np.ones(n)
    assert abs(orc.dropped(v, 0.25, 3, 4).mean() - 1) < 5 * (0.25 / 0.75 / n) ** 0.5


def test_tables_by_hand():
    idx = np.array([[3, 1], [1, 2], [1, 0], [2, 1]])
    counts, off, row, src = orc.tables(idx, 2, first=1)
    assert counts.tolist() == [4, 2] and off.tolist() == [0, 4, 6] and src.tolist() == [1, 2, 4, 7, 3, 6]
    assert row.tolist() == [[-1, 0], [1, 4], [2, -1], [5, 3]]
    counts, off, row, src = orc.tables(idx, 2, first=1, capacity=3)
    assert counts.tolist() == [4, 2] and off.tolist() == [0, 3, 5] and row.tolist() == [[-1, 0], [1, 3], [2, -1], [4, -1]] and src.tolist() == [1, 2, 4, 3, 6]


def test_rows_and_back_are_each_others_gradient():
    """<scatter(v, w), r> = <v, gather(r, w)> = <w, dots(v, r)>, all three linear in each argument."""
    rng = np.random.default_rng(0)
    T, k, d = 9, 3, 5
    idx = np.array([rng.permutation(6)[:k] for _ in range(T)])
    _, off, row, _ = orc.tables(idx, 4, first=1, capacity=4)
    v, r, w = rng.normal(size=(T, d)), rng.normal(size=(T * k, d)), rng.normal(size=(T, k))
    a = (orc.scattered(v, row, w, T * k) * r).sum()
    assert np.isclose(a, (v * orc.gathered(r, row, w)).sum(), rtol=1e-12) and np.isclose(a, (w * orc.dots(v, r, row)).sum(), rtol=1e-12)
    assert (orc.scattered(v, row, w, T * k)[off[-1]:] == 0).all()


@pytest.mark.parametrize("gating", [orc.SOFTMAX, orc.RENORM, orc.SIGMOID])
def test_the_gates_gradient_against_differences(gating):
    rng = np.random.default_rng(gating)
    z, g = rng.normal(size=(4, 7)), rng.normal(size=(4, 3))
    idx = np.array([rng.permutation(7)[:3] for _ in range(4)])
    dz = orc.gate_backward(z, idx, orc.gate(z, idx, gating), g, gating)
    h = 1e-5
    for t in range(4):
        for e in range(7):
            up, down = z.copy(), z.copy()
            up[t, e] += h
            down[t, e] -= h
            diff = ((orc.gate(up, idx, gating) - orc.gate(down, idx, gating)) * g).sum() / (2 * h)
            assert abs(diff - dz[t, e]) < 1e-9, (t, e)          # h^2 times third derivatives, which are below 1
