"""Training and adapter operators where offsets pass 32 bits: weights and their gradients of more than 2^31 elements, adapters' matrices of as many, and rows
close below the 4 GiB that the activation buffers may hold.  Compared on the GPU in 64 bits where something was put, and with zero elsewhere.

Bounds (b = 2^-8 for bf16, f = 2^-24 for fp32) are norms here, an output at a time: n roundings to bf16 whose errors are independent and at most b of the rounded
value each add at most b of the result's norm each; an fp32 sum of m products adds at most m f sqrt(m) of it, which is below b / 8 for m <= 2^10 (and for
longer sums of independent terms, whose error grows with sqrt(m) f, far below)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

B = 2.0 ** -8


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_23911_amd as m
    m.lib()
    return m


def _near(got, want, roundings, what):
    got, want = got.double(), want.double()
    off = float((got - want).norm() / want.norm())
    assert off <= (roundings + 0.125) * B, (what, off / B)


def _rand(gen, *shape, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).bfloat16()


def _buf(*shape, dtype=torch.bfloat16, fill=float("nan")):
    return torch.full(shape, fill, dtype=dtype, device="cuda")


def _block(x, g, u, dy, wg, wu, wd):
    """dx, dWg, dWu, dWd and, from x, the forward's g, u, y of one expert, in 64 bits."""
    x, g, u, dy, wg, wu, wd = (t.double() for t in (x, g, u, dy, wg, wu, wd))
    s = torch.sigmoid(g)
    dh = dy @ wd
    dg, du = dh * u * s * (1 + g * (1 - s)), dh * g * s
    fg, fu = x @ wg.T, x @ wu.T
    return dg @ wg + du @ wu, dg.T @ x, du.T @ x, dy.T @ (g * s * u), fg, fu, (fg * torch.sigmoid(fg) * fu) @ wd.T


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_wide_experts(moe, dtype):
    E, d, F = 256, 7168, 2048
    assert E * d * F > 1 << 31
    counts = [0] * E
    counts[0], counts[150], counts[E - 1] = 5, 33, 90
    n = sum(counts)
    gen = torch.Generator(device="cuda").manual_seed(1)
    w = {k: torch.zeros(s, dtype=torch.bfloat16, device="cuda") for k, s in (("g", (E, F, d)), ("u", (E, F, d)), ("d", (E, d, F)))}
    for e in (0, 150, E - 1):
        w["g"][e], w["u"][e], w["d"][e] = _rand(gen, F, d, std=d ** -0.5), _rand(gen, F, d, std=d ** -0.5), _rand(gen, d, F, std=F ** -0.5)
    x, g, u, dy = _rand(gen, n, d), _rand(gen, n, F), _rand(gen, n, F), _rand(gen, n, d, std=0.1)
    off = torch.cat([torch.zeros(1, dtype=torch.int64), torch.tensor(counts).cumsum(0)]).to(torch.int32).cuda()
    cfg = moe.MoEConfig.of(n, d, F, E, 1)
    ws = torch.empty(max(moe.ffn_workspace_size(cfg), moe.ffn_backward_workspace_size(cfg)), dtype=torch.uint8, device="cuda")
    fg, fu, fh, fy = _buf(n, F), _buf(n, F), _buf(n, F), _buf(n, d)
    moe.moe_grouped_ffn_train(cfg, x, off, w["g"], w["u"], w["d"], fg, fu, fh, fy, ws)
    dx, dw = _buf(n, d), [_buf(*w[k].shape, dtype=dtype) for k in "gud"]
    moe.moe_grouped_ffn_backward(cfg, x, off, w["g"], w["u"], w["d"], g, u, dy, dx, *dw, ws)
    torch.cuda.synchronize()
    a = 0
    for e, m in enumerate(counts):
        r = slice(a, a + m)
        a += m
        if m == 0:
            assert not any(t[e].any() for t in dw), e
            continue
        want = _block(x[r], g[r], u[r], dy[r], w["g"][e], w["u"][e], w["d"][e])
        _near(dx[r], want[0], 2, "dx")             # dg and du, dx
        for t, v, name in zip(dw, want[1:4], ("dwg", "dwu", "dwd")):
            _near(t[e], v, 2, name)                # the operand, the result
        _near(fg[r], want[4], 1, "g")
        _near(fu[r], want[5], 1, "u")
        _near(fy[r], want[6], 2, "y")              # h, y


def test_rows_up_to_the_limit(moe):
    d, F = 64, 16320
    R = ((1 << 32) - 1) // (2 * F)                 # one more is refused
    assert moe.ffn_workspace_size(moe.MoEConfig.of(R + 1, d, F, 2, 1)) == 0
    gen = torch.Generator(device="cuda").manual_seed(2)
    cut = R - 1000
    off = torch.tensor([0, cut, R], dtype=torch.int32, device="cuda")
    wg, wu, wd = _rand(gen, 2, F, d, std=d ** -0.5), _rand(gen, 2, F, d, std=d ** -0.5), _rand(gen, 2, d, F, std=F ** -0.5)
    x, dy = _rand(gen, R, d), _rand(gen, R, d, std=0.1)
    cfg = moe.MoEConfig.of(R, d, F, 2, 1)
    ws = torch.empty(max(moe.ffn_workspace_size(cfg), moe.ffn_backward_workspace_size(cfg)), dtype=torch.uint8, device="cuda")
    g, u, h, y = _buf(R, F), _buf(R, F), _buf(R, F), _buf(R, d)
    moe.moe_grouped_ffn_train(cfg, x, off, wg, wu, wd, g, u, h, y, ws)
    dx, dw = _buf(R, d), [_buf(2, F, d, dtype=torch.float32), _buf(2, F, d, dtype=torch.float32), _buf(2, d, F, dtype=torch.float32)]
    moe.moe_grouped_ffn_backward(cfg, x, off, wg, wu, wd, g, u, dy, dx, *dw, ws)
    torch.cuda.synchronize()
    for e, a, b in ((0, 0, 700), (0, cut - 700, cut), (1, cut, R)):
        r = slice(a, b)
        want = _block(x[r], g[r], u[r], dy[r], wg[e], wu[e], wd[e])
        for got, v, n, name in ((g, want[4], 1, "g"), (u, want[5], 1, "u"), (y, want[6], 2, "y"), (dx, want[0], 2, "dx")):
            _near(got[r], v, n, (name, e, a))
        if e == 1:
            for t, v, name in zip(dw, want[1:4], ("dwg", "dwu", "dwd")):
                _near(t[1], v, 1, name)
    # the first expert's weight gradients are sums over nearly all rows
    sums = [torch.zeros(t.shape[1:], dtype=torch.float64, device="cuda") for t in dw]
    for a in range(0, cut, 8192):
        r = slice(a, min(a + 8192, cut))
        for t, v in zip(sums, _block(x[r], g[r], u[r], dy[r], wg[0], wu[0], wd[0])[1:4]):
            t += v
    for t, v, name in zip(dw, sums, ("dwg", "dwu", "dwd")):
        _near(t[0], v, 1, name)


def test_adapters_of_many_elements(moe):
    N, K, rank, n = 14336, 14336, 128, 1200
    assert n * rank * N > 1 << 31 and n * rank * K > 1 << 31
    gen = torch.Generator(device="cuda").manual_seed(3)
    A = [torch.zeros((n, rank, K), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    Bm = [torch.zeros((n, N, rank), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for a in (0, 600, n - 1):
        for m in range(2):
            A[m][a], Bm[m][a] = _rand(gen, rank, K, std=K ** -0.5), _rand(gen, N, rank, std=rank ** -0.5)
    W = [_rand(gen, N, K, std=K ** -0.5) for _ in range(2)]
    scale = torch.rand(n, generator=gen, device="cuda") + 0.5
    for T in (40, 300):
        x = _rand(gen, T, K)
        ids = torch.tensor([0, 600, n - 1, -1], dtype=torch.int32, device="cuda").repeat(T // 4)
        cfg = moe.AdapterConfig.of(T, N, K, n, rank)
        ws = torch.empty(moe.adapter_workspace_size(cfg), dtype=torch.uint8, device="cuda")
        y, h = _buf(T, N), _buf(T, N)
        moe.moe_adapter_linear(cfg, x, W[0], A[0], Bm[0], scale, ids, y, ws)
        moe.moe_adapter_gated_up(cfg, x, *W, *A, *Bm, scale, ids, h, ws)
        want = [x.double() @ W[m].double().T for m in range(2)]
        for a in (0, 600, n - 1):
            r = ids == a
            for m in range(2):
                want[m][r] += scale[a].double() * ((x[r].double() @ A[m][a].double().T) @ Bm[m][a].double().T)
        _near(y, want[0], 1, "y")
        _near(h, want[0] * torch.sigmoid(want[0]) * want[1], 1, "h")


def test_adapter_tokens_up_to_the_limit(moe):
    N, K, rank, n = 16320, 64, 16, 3
    T = ((1 << 32) - 1) // (2 * N)
    assert moe.adapter_workspace_size(moe.AdapterConfig.of(T + 1, N, K, n, rank)) == 0
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, base = _rand(gen, T, K), _rand(gen, T, N)
    W, A, Bm = _rand(gen, N, K, std=K ** -0.5), _rand(gen, n, rank, K, std=K ** -0.5), _rand(gen, n, N, rank, std=rank ** -0.5)
    ids = (torch.arange(T, device="cuda") // 1000 % (n + 1)).to(torch.int32)       # n: without
    cfg = moe.AdapterConfig.of(T, N, K, n, rank)
    ws = torch.empty(moe.adapter_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    y = _buf(T, N)
    moe.moe_adapter_linear(cfg, x, W, A, Bm, None, ids, y, ws, base=base)
    for a in (0, T // 2, T - 3000):
        r = slice(a, a + 3000)
        xd = x[r].double()
        want = xd @ W.double().T + base[r].double()
        for i in range(n):
            m = ids[r] == i
            want[m] += (xd[m] @ A[i].double().T) @ Bm[i].double().T
        _near(y[r], want, 1, ("y", a))
