"""The combine's gradients in calls whose rows pass the caches by (2^26 elements of them or more), against their definition in 64 bits by slices of tokens.

Bounds (b = 2^-8 for bf16, f = 2^-24 for fp32): a row's gradient is one product in fp32, rounded to bf16: (b + f) |w dy|; a gate weight's is an fp32 sum of d products:
d f <|dy|, |p|>."""
import pytest
import torch

pytestmark = pytest.mark.gpu

B, F32 = 2.0 ** -8, 2.0 ** -24
FEW = 1 << 26


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_23911_amd as m
    m.lib()
    return m


@pytest.mark.parametrize("k,d", [(1, 4160), (2, 4160), (3, 704), (4, 2048), (5, 4160), (6, 2112), (7, 4160), (8, 4096), (8, 7168), (13, 4160), (17, 2112)])
def test_streamed(moe, k, d):
    print("combine", k, d, flush=True)
    T = (FEW + k * d - 1) // (k * d)               # the fewest tokens whose rows are streamed
    assert T * k * d >= FEW > (T - 1) * k * d
    gen = torch.Generator(device="cuda").manual_seed(k * d)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    dy, p, w = rand(T, d).mul_(0.1).bfloat16(), rand(T * k, d).bfloat16(), rand(T, k)
    row_of = torch.randperm(T * k, generator=gen, device="cuda").to(torch.int32).view(T, k)
    cfg = moe.MoEConfig.of(T, d, 64, max(k, 8), k)
    room = torch.full((T * k + 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
    dp, dw = room[:-1], torch.full((T, k), float("nan"), dtype=torch.float32, device="cuda")
    moe.moe_combine_backward(cfg, dy, p, row_of, w, dp, dw)
    step = max(1, (1 << 22) // (k * d))
    for a in range(0, T, step):
        s = slice(a, min(a + step, T))
        rows = row_of[s].long()
        g, q = dy[s].double(), p[rows].double()
        want = w[s].double()[:, :, None] * g[:, None, :]
        assert ((dp[rows].double() - want).abs() <= (B + F32) * want.abs()).all(), a
        terms = g[:, None, :] * q
        assert ((dw[s].double() - terms.sum(2)).abs() <= d * F32 * terms.abs().sum(2)).all(), a
    assert (room[-1] == 7.0).all()
    # over the rows themselves
    dw2 = torch.empty_like(dw)
    moe.moe_combine_backward(cfg, dy, p, row_of, w, p, dw2)
    assert torch.equal(p, dp) and torch.equal(dw2, dw)
