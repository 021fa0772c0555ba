"""With all experts here, no limit of rows, no residual and no dropout the calls over slots that may have no row are the layer's own: the same tables, rows and tokens, bit for bit.
The weights' gradients are sums of d products in another order where a token has a wavefront of its own (d <= 1024): fp32 sums of n terms, each within n 2^-24 of their absolute values."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_23911_amd as m
    m.lib()
    return m


@pytest.mark.parametrize("T,k,d,E", [(1, 2, 4096, 8), (333, 8, 3584, 64), (1999, 3, 1024, 7), (2500, 12, 512, 60), (515, 2, 64, 5), (2300, 8, 7168, 256)])
def test_the_same_as_the_layers_own_calls(moe, T, k, d, E):
    gen = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn((T, d), generator=gen, device="cuda").bfloat16()
    idx = torch.rand((T, E), generator=gen, device="cuda").topk(k, dim=1).indices.int()
    w = torch.rand((T, k), generator=gen, device="cuda")
    c, dc = moe.MoEConfig.of(T, d, 64, E, k), moe.DispatchConfig.of(T, d, k, E)
    ws = torch.empty(max(moe.permute_workspace_size(c), moe.dispatch_workspace_size(dc)), dtype=torch.uint8, device="cuda")

    def tables():
        return [torch.full(s, -5, dtype=torch.int32, device="cuda") for s in ((E,), (E + 1,), (T, k), (T * k,))] + [torch.full((T * k, d), 7.0, dtype=torch.bfloat16, device="cuda")]

    a, b = tables(), tables()
    moe.moe_permute(c, x, idx, *a, ws)
    moe.moe_dispatch(dc, x, idx, None, *b, ws)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    row, rows = a[2], torch.randn((T * k, d), generator=gen, device="cuda").bfloat16()
    y, y2 = torch.empty_like(x), torch.empty_like(x)
    moe.moe_combine(c, rows, row, w, y)
    moe.moe_collect(dc, rows, row, w, y2)
    assert torch.equal(y, y2)
    g, g2, dw, dw2 = torch.empty_like(rows), torch.empty_like(rows), torch.empty_like(w), torch.empty_like(w)
    moe.moe_combine_backward(c, x, rows, row, w, g, dw)
    moe.moe_collect_backward(dc, x, rows, row, w, g2, d_topk_w=dw2)
    assert torch.equal(g, g2)
    if d > 1024:
        assert torch.equal(dw, dw2)
    size = (x.abs().double()[:, None] * rows[row.long()].abs().double()).sum(2)
    assert ((dw - dw2).abs() <= 2 * d * 2.0**-24 * size).all()
