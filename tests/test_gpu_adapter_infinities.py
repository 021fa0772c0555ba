"""An infinity in one adapter's B: its tokens' results at that feature are not finite (NaN as a rule, as include/moe.h says), and no other result changes by a bit."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))

from test_gpu_adapter import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_23911_amd as m
    m.lib()
    return m


# joined sums of both kinds, and all three tiles of the single launch
@pytest.mark.parametrize("T,N,tiles", [(9, 192, "Flat"), (120, 192, "Half"), (300, 8256, "Small"), (400, 8256, "Tall"), (513, 14400, "Wide")])
def test_an_infinity_stays_where_it_is(moe, T, N, tiles):
    from paper_2605_23911_amd import binding
    c, clean = (Case(T, N, 256, 5, 24, "mixed", seed=11) for _ in range(2))
    for k in (c, clean):
        k.ids[:3] = [2, 0, -1]
    c.b[0][2, 7, 3], c.b[0][2, N - 1, 20] = float("inf"), float("-inf")
    got, want = c.gpu(moe).linear(moe), clean.gpu(moe).linear(moe)
    assert binding.adapter_tiles(c.cfg, 1) == tiles
    hurt = torch.zeros((T, N), dtype=torch.bool, device="cuda")
    mine = torch.from_numpy(c.ids == 2).cuda()
    hurt[mine, 7] = hurt[mine, N - 1] = True
    assert not torch.isfinite(got[hurt]).any() and torch.equal(got[~hurt], want[~hurt])
