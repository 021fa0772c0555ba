"""Operators over slots that may have no row, where offsets pass 32 bits: more than 4 GiB of rows, more than 2^32 elements; and where rows pass the caches by.  Compared on the GPU: tables and copies exactly,
sums of two or three terms and products against fp32 torch operations on the same values, whose own errors are below (k + 4) 2^-24 of the terms' sizes: with the one rounding
to bf16, 2^-8 |y| + 2^-20 A holds for both."""
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


def _rand(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda").bfloat16()


@pytest.mark.parametrize("T,d,k,capacity", [(300_000, 4104, 2, 90_000), (11_000_000, 200, 1, 0)])
def test_rows_beyond_four_gib(moe, T, d, k, capacity):
    assert T * k * d * 2 > 1 << 32
    assert _there_and_back(moe, T, d, k, capacity) * d * 2 > (1 << 32) - (1 << 30)


@pytest.mark.parametrize("T,d,k,capacity", [(2300, 4104, 4, 1000), (2050, 7176, 6, 0), (1500, 7176, 8, 0), (70_000, 520, 2, 0), (6000, 1032, 12, 8000)])
def test_rows_that_pass_the_caches_by(moe, T, d, k, capacity):
    """From 64 MiB on those that collect's gradient writes, from 128 MiB on all; every batch of slots."""
    assert T * k * d >= 1 << 25
    _there_and_back(moe, T, d, k, capacity)


def _there_and_back(moe, T, d, k, capacity):
    E, R = 8 if k < 8 else 16, T * k
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty((T, d), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    idx = torch.rand((T, E + 1), generator=gen, device="cuda").topk(k, dim=1).indices.to(torch.int32)          # the last expert is elsewhere
    w = torch.randn((T, k), generator=gen, device="cuda")
    cfg = moe.DispatchConfig.of(T, d, k, E, 0, capacity)
    i32 = {"dtype": torch.int32, "device": "cuda"}
    counts, off, row, src = torch.empty(E, **i32), torch.empty(E + 1, **i32), torch.empty((T, k), **i32), torch.full((R,), -7, **i32)
    rows = torch.full((R, d), 7.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_dispatch(cfg, x, idx, None, counts, off, row, src, rows, torch.empty(moe.dispatch_workspace_size(cfg), dtype=torch.uint8, device="cuda"))
    # tables: a stable sort by expert
    e = idx.view(-1).long()
    order = torch.sort(e, stable=True).indices
    n = torch.bincount(e, minlength=E + 1)
    rank = torch.empty_like(e)
    rank[order] = torch.arange(R, device="cuda") - (n.cumsum(0) - n)[e[order]]
    kept = n[:E].clamp(max=capacity) if capacity else n[:E]
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), kept.cumsum(0)])
    have = (e < E) & ((rank < capacity) if capacity else torch.ones_like(e, dtype=torch.bool))
    want = torch.where(have, start[e.clamp(max=E - 1)] + rank, -1)
    N = int(start[-1])
    assert torch.equal(counts, n[:E].int()) and torch.equal(off, start.int()) and torch.equal(row.view(-1), want.int())
    assert (src[N:] == -7).all() and torch.equal(want[src[:N].long()], torch.arange(N, device="cuda"))
    for a in range(0, R, 1 << 17):
        b = min(a + (1 << 17), R)
        got = rows[a:b]
        if a < N:
            m = min(b, N)
            assert torch.equal(got[:m - a].view(torch.int16), x[src[a:m].long() // k].view(torch.int16)), a
        if b > N:
            assert (got[max(N - a, 0):] == 7.0).all(), a
    # the way back, with residual and dropout, and the gradients, in the same buffers
    state = torch.tensor([17, 1 << 33], dtype=torch.int64, device="cuda")
    y, mask = torch.empty_like(x), torch.empty_like(x)
    moe.moe_collect(cfg, rows, row, w, y, residual=x, p=0.25, rng=state)
    moe.moe_dropout(torch.ones_like(x), mask, 0.25, state)              # 4/3 where an element is kept
    moe.moe_collect_backward(cfg, x, rows, row, w, rows, d_topk_w=(dw := torch.empty((T, k), device="cuda")), p=0.25, rng=state)
    dx = torch.empty_like(x)
    moe.moe_dispatch_backward(cfg, rows, row, None, dx, base=x)
    has = row >= 0
    ws = torch.where(has, w, 0.0)
    for a in range(0, T, 1 << 16):
        b = min(a + (1 << 16), T)
        xx, s = x[a:b].float(), torch.where(mask[a:b] != 0, 4.0 / 3.0, 0.0)
        # every row is a copy of its token
        total, size = ws[a:b].sum(1, keepdim=True) * xx * s + xx, ws[a:b].abs().sum(1, keepdim=True) * xx.abs() * s + xx.abs()
        assert ((y[a:b].float() - total).abs() <= 2.0**-8 * total.abs() + 2.0**-20 * size).all(), a
        dots = (s.double() * xx.double() ** 2).sum(1, keepdim=True) * has[a:b]
        assert ((dw[a:b] - dots).abs() <= 2 * (d / 64 + 24) * 2.0**-24 * dots).all(), a
        # rows now hold w v, each rounded once
        v = s * xx
        total, size = xx + ws[a:b].sum(1, keepdim=True) * v, xx.abs() + ws[a:b].abs().sum(1, keepdim=True) * v.abs()
        assert ((dx[a:b].float() - total).abs() <= 2.0**-8 * total.abs() + 2.0**-8 * 1.01 * size).all(), a
    return N


def test_dropout_beyond_32_bits(moe):
    """More than 2^32 elements: kept and dropped as the tensor's own halves say, and the mask does not repeat."""
    n = (1 << 32) + 12_345
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(x)
    state = torch.tensor([3, 4], dtype=torch.int64, device="cuda")
    moe.moe_dropout(x, y, 0.5, state)
    tail, head = y[-12_345:], y[:12_345]
    for part in (tail, head):
        assert ((part == 0) | (part == 2)).all() and abs(float((part != 0).float().mean()) - 0.5) < 5 * (0.25 / 12_345) ** 0.5
    assert float(((tail != 0) == (head != 0)).float().mean()) < 0.6
    from oracle import token_oracle as orc
    block = (1 << 32) // 8
    words = orc.philox((3, 0), (block & 0xFFFFFFFF, block >> 32, 4, 0))
    want = [2.0 if (words[j // 2] >> 16 * (j % 2) & 0xFFFF) >= 32768 else 0.0 for j in range(8)]
    assert y[1 << 32:(1 << 32) + 8].tolist() == want
    block = n // 8                                                       # the last, partial block
    words = orc.philox((3, 0), (block & 0xFFFFFFFF, block >> 32, 4, 0))
    assert y[block * 8:].tolist() == [2.0 if (words[j // 2] >> 16 * (j % 2) & 0xFFFF) >= 32768 else 0.0 for j in range(n % 8)]


def test_router_of_many_tokens(moe):
    """dz of more than 4 GiB.  x and W_r are whole numbers over powers of two, so logits are exact; dW_r is a sum of a hundred and more pieces of up to 2^15 tokens each: off by
    at most (2^15 + 2^8) 2^-24 of the sum of absolute values."""
    T, d, E, k = 3_000_000, 64, 256, 2
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randint(-2, 3, (T, d), generator=gen, device="cuda").bfloat16()
    wr = (torch.randint(-4, 5, (E, d), generator=gen, device="cuda") / 32).bfloat16()
    g = torch.randn((T, k), generator=gen, device="cuda")
    cfg = moe.MoEConfig.of(T, d, 64, E, k)
    idx, w = torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda")
    for a in range(0, T, 1 << 18):
        b = min(a + (1 << 18), T)
        top = torch.topk(torch.softmax(x[a:b].double() @ wr.double().T, 1), k, dim=1)
        idx[a:b], w[a:b] = top.indices.int(), top.values.float()
    size = moe.route_backward_workspace_size(cfg)
    assert T * 3 * E * 2 > 1 << 32 and size > T * 3 * E * 2
    dx, dwr, dbias = torch.empty_like(x), torch.empty((E, d), device="cuda"), torch.empty(E, device="cuda")
    moe.moe_route_backward(cfg, x, wr, None, idx, w, g, dx, dwr, dbias, torch.empty(size, dtype=torch.uint8, device="cuda"))
    want_w, size_w = torch.zeros((E, d), dtype=torch.float64, device="cuda"), torch.zeros((E, d), dtype=torch.float64, device="cuda")
    want_b, size_b = torch.zeros(E, dtype=torch.float64, device="cuda"), torch.zeros(E, dtype=torch.float64, device="cuda")
    for a in range(0, T, 1 << 18):
        b = min(a + (1 << 18), T)
        xx, p = x[a:b].double(), torch.softmax(x[a:b].double() @ wr.double().T, 1)
        G = torch.zeros_like(p).scatter_add_(1, idx[a:b].long(), g[a:b].double())
        dz = p * (G - (p * G).sum(1, keepdim=True))
        off = p * (24 * 2.0**-24) * (G.abs() + 2 * (p * G.abs()).sum(1, keepdim=True))
        ref = dz @ wr.double()
        bound = (off + 2.0**-16 * dz.abs() + 2 * E * 2.0**-24 * dz.abs()) @ wr.double().abs() + 2.0**-8 * ref.abs()
        assert ((dx[a:b].double() - ref).abs() <= bound * (1 + 2.0**-8)).all(), a
        want_w += dz.T @ xx
        size_w += (dz.abs() * (2**15 + 2**8) * 2.0**-24 + off).T @ xx.abs()
        want_b += dz.sum(0)
        size_b += (dz.abs() * (2**13) * 2.0**-24 + off).sum(0)           # 4096 wavefronts' sums of 733 tokens, then their sum
    assert ((dwr.double() - want_w).abs() <= size_w).all() and ((dbias.double() - want_b).abs() <= size_b).all()


def test_in_place_over_several_launches(moe):
    """More tokens than a launch takes, at the width whose workgroups hold a number of tokens that does not divide it (84 at 24 elements): in place each is added to once.  All values are
    exact."""
    T, d = (1 << 29) + 60, 24
    cfg = moe.DispatchConfig.of(T, d, 1, 1)
    row = torch.arange(T, dtype=torch.int32, device="cuda").view(T, 1)
    rows, y = (torch.full((T, d), v, dtype=torch.bfloat16, device="cuda") for v in (0.5, 0.25))

    def check(t, value):
        for a in range(0, T, 1 << 26):
            assert bool((t[a:a + (1 << 26)] == value).all()), a

    moe.moe_collect(cfg, rows, row, None, y, residual=y)
    check(y, 0.75)
    moe.moe_dispatch_backward(cfg, rows, row, None, y, base=y)
    check(y, 1.25)
    dw = torch.empty((T, 1), device="cuda")
    moe.moe_collect_backward(cfg, y, rows, row, None, rows, d_topk_w=dw)
    check(rows, 1.25)
    check(dw, 24 * 0.5 * 1.25)
