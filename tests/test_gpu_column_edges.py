"""Results whose columns end inside a large tile, on the GPU through the binding against the fp64 oracle: every tile of the training and adapter
operators, and every height of its bodies, at widths that are no multiple of it, with rows behind the result that have to stay as they were.
Each case says which tiles it is for and asks the library whether the call takes them.  Bounds: as in the two files that the oracles come from."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))

from oracle import train_oracle as orc
from test_gpu_adapter import Case
from test_gpu_adapter import _close as close_adapter
from test_gpu_ffn_train import B, F32, Block, _close, _np

pytestmark = pytest.mark.gpu

GUARD = 7.0


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_23911_amd as m
    m.lib()
    return m


# counts, d, F, {product: tiles}: F ends inside the tiles of the forward pass (but Tall's and Small's, 64 features of both projections), of dh and
# of the weight gradients, d inside those of dx
FFN = [
    ([30, 100, 150, 250], 192, 8256, {"forward": "Wide", "dh": "Deep", "dx": "Small, sum in pieces", "dw": "Pair"}),      # bodies of one to four blocks
    ([190, 256, 0, 65, 320], 192, 8256, {"forward": "Wide", "dh": "Deep", "dw": "Pair"}),
    ([30, 100, 150, 250], 8256, 192, {"dx": "Deep", "dw": "Pair"}),
    ([190, 256, 0, 65, 320], 8256, 192, {"dx": "Deep", "dw": "Pair"}),
    ([65, 3, 130], 192, 320, {"forward": "Tall", "dh": "Tall", "dx": "Tall", "dw": "Small"}),                             # 65 and 130 rows: Tall's body of one block and of two
    ([129, 140, 0, 70, 200], 320, 192, {"forward": "Tall", "dh": "Tall", "dx": "Tall", "dw": "Small"}),
    ([70, 257, 30, 129], 192, 192, {"forward": "Tall", "dh": "Tall", "dx": "Tall", "dw": "Small"}),                       # a second block behind a whole one
]


@pytest.mark.parametrize("counts,d,F,tiles", FFN)
def test_block(moe, counts, d, F, tiles):
    from paper_2605_23911_amd import binding
    print("block", counts, d, F, flush=True)
    b = Block(counts, d, F, seed=7, tail=2)
    b.to_gpu(moe)
    assert {p: binding.train_tiles(b.cfg, p) for p in tiles} == tiles
    n = b.n
    # forward
    o = b.forward(moe, fill=GUARD)
    h = {k: _np(t) for k, t in b.host.items()}
    g, u, hh, y = orc.block_forward(h["x"][:n], b.off, h["wg"], h["wu"], h["wd"])
    eg, eu, ey = np.zeros_like(g), np.zeros_like(u), np.zeros_like(y)
    for e in range(b.E):
        r = slice(b.off[e], b.off[e + 1])
        ax = np.abs(h["x"][r])
        eg[r], eu[r] = d * F32 * (ax @ np.abs(h["wg"][e]).T), d * F32 * (ax @ np.abs(h["wu"][e]).T)
    act = np.abs(orc.silu(g))
    eh = np.abs(u) * (1.1 * eg + 16 * F32 * act) + act * eu + B * np.abs(hh)
    for e in range(b.E):
        r = slice(b.off[e], b.off[e + 1])
        ey[r] = (eh[r] + F * F32 * np.abs(hh[r])) @ np.abs(h["wd"][e]).T
    for name, want, bound in (("g", g, eg), ("u", u, eu), ("h", hh, eh), ("y", y, ey)):
        _close(o[name][:n], want, bound + B * np.abs(want), name)
        assert (o[name][n:] == GUARD).all(), name
    # backward, in both types, and added
    want, bound = b.oracle()
    for dtype, rounding in ((torch.bfloat16, B), (torch.float32, F32)):
        got = b.backward(moe, b.grads(dtype, fill=GUARD))
        both = b.backward(moe, b.grads(dtype, fill=0.5), accumulate=True)
        torch.cuda.synchronize()
        assert (got["dx"][n:] == GUARD).all()
        _close(got["dx"][:n], want["dx"], bound["dx"] + B * np.abs(want["dx"]), "dx")
        assert torch.equal(both["dx"][:n], got["dx"][:n])
        for w in ("dwg", "dwu", "dwd"):
            _close(got[w], want[w], bound[w] + rounding * np.abs(want[w]), (w, dtype))
            _close(both[w], want[w] + 0.5, bound[w] + rounding * np.abs(want[w] + 0.5) + F32 * np.abs(want[w]), (w, dtype, "added"))


# T, N, rank, ids, matrices, tiles
ADAPTERS = [
    (513, 14400, 24, "requests", 1, "Wide"), (600, 14400, 72, "mixed", 1, "Wide"), (400, 8256, 24, "requests", 1, "Tall"), (430, 8256, 128, "mixed", 1, "Tall"),
    (300, 8256, 40, "mixed", 1, "Small"), (200, 14400, 8, "own", 1, "Small"), (130, 4160, 24, "own", 1, "Half"), (64, 8256, 24, "own", 1, "Flat"),
    (513, 8256, 24, "requests", 2, "Wide"), (450, 8256, 104, "mixed", 2, "Wide"), (200, 14400, 24, "mixed", 2, "Tall"), (257, 8256, 72, "mixed", 2, "Small"),
    (128, 8256, 16, "own", 2, "Half"), (33, 8256, 72, "own", 2, "Flat"),
]


@pytest.mark.parametrize("T,N,rank,ids,two,tiles", ADAPTERS)
def test_adapters(moe, T, N, rank, ids, two, tiles):
    from paper_2605_23911_amd import binding
    print("adapters", T, N, rank, ids, two, flush=True)
    c = Case(T, N, 192, 9, rank, ids, seed=8, two=two == 2, base=two == 1).gpu(moe)
    assert binding.adapter_tiles(c.cfg, two) == tiles
    room = torch.full((T + 2, N), GUARD, dtype=torch.bfloat16, device="cuda")
    c.y = room[:T]
    g, eg = c.want(0)
    if two == 1:
        y = g + _np(c.base)
        close_adapter(c.linear(moe), y, eg + (B + F32) * np.abs(y), "y")
    else:
        u, eu = c.want(1)
        act = orc.silu(g)
        close_adapter(c.gated(moe), act * u, np.abs(u) * (1.1 * eg + 16 * F32 * np.abs(act)) + np.abs(act) * eu + B * np.abs(act * u), "h")
    assert (room[T:] == GUARD).all()


@pytest.mark.parametrize("T,N,tiles", [(513, 14400, "Wide"), (400, 8256, "Tall"), (300, 8256, "Small")])
def test_adapters_without_the_shared_projection(moe, T, N, tiles):
    from paper_2605_23911_amd import binding
    c = Case(T, N, 192, 6, 40, "mixed", seed=9, base=True).gpu(moe)
    assert binding.adapter_tiles(c.cfg, 1) == tiles
    y, e = c.want(0, shared=False)
    y = y + _np(c.base)
    close_adapter(c.linear(moe, shared=False), y, e + (B + F32) * np.abs(y), "y")
