"""The training operators together as a layer's step uses them, the adapters together as a shared expert uses them, and the ways in which calls meet:
captured and replayed, two at once on two streams, with tensors that were misplaced.

End to end: a result went through n roundings to bf16 whose errors are independent and at most 2^-8 of the rounded value each, so that each adds at most 2^-8 of
the result's norm (a sum's errors add in squares, as its terms do); SiLU' passes a rounding of g on by |g SiLU''(g) / SiLU'(g)|, which is
counted as two.  n is given with each check."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))

import moe_inputs as mi
from oracle import train_oracle as orc

pytestmark = pytest.mark.gpu

B = 2.0 ** -8


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_23911_amd as m
    m.lib()
    return m


def _gpu(shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _near(got, want, roundings, what):
    got, want = got.detach().cpu().double(), want.detach().double()
    off = float((got - want).norm() / want.norm())
    assert off <= roundings * B, (what, off, roundings * B)


class Step:
    """One training step of a layer: everything that moe.h names for it, in its order."""

    def __init__(self, moe, s, seed=0):
        self.moe, self.s = moe, s
        self.cfg = moe.MoEConfig.of(s.T, s.d, s.F, s.E, s.k, s.gating)
        self.x, self.wr = mi.make_x(s, seed).cuda(), mi.make_router(s, seed).cuda()
        self.w = [t.cuda() for t in mi.make_all_experts(s, seed)]
        self.dy = (mi.make_x(s, seed + 1).float() * 0.1).to(torch.bfloat16).cuda()
        T, k, R, d, F, E = s.T, s.k, s.R, s.d, s.F, s.E
        i32, f32, u8 = torch.int32, torch.float32, torch.uint8
        self.idx, self.tw, self.counts, self.off = _gpu((T, k), i32), _gpu((T, k), f32), _gpu(E, i32), _gpu(E + 1, i32)
        self.row, self.src, self.xp = _gpu(R, i32), _gpu(R, i32), _gpu((R, d))
        self.g, self.u, self.h, self.yp, self.y = _gpu((R, F)), _gpu((R, F)), _gpu((R, F)), _gpu((R, d)), _gpu((T, d))
        self.dyp, self.dtw, self.dxp, self.dx = _gpu((R, d)), _gpu((T, k), f32), _gpu((R, d)), _gpu((T, d))
        self.dw = [torch.empty_like(t) for t in self.w]
        self.ones = torch.ones((T, k), dtype=f32, device="cuda")
        self.ws = _gpu(max(moe.route_workspace_size(self.cfg), moe.permute_workspace_size(self.cfg), moe.ffn_workspace_size(self.cfg),
                           moe.ffn_backward_workspace_size(self.cfg)), u8)

    def run(self):
        m, c = self.moe, self.cfg
        m.moe_route(c, self.x, self.wr, None, self.idx, self.tw, self.ws)
        m.moe_permute(c, self.x, self.idx, self.counts, self.off, self.row, self.src, self.xp, self.ws)
        m.moe_grouped_ffn_train(c, self.xp, self.off, *self.w, self.g, self.u, self.h, self.yp, self.ws)
        m.moe_combine(c, self.yp, self.row, self.tw, self.y)
        m.moe_combine_backward(c, self.dy, self.yp, self.row, self.tw, self.dyp, self.dtw)
        m.moe_grouped_ffn_backward(c, self.xp, self.off, *self.w, self.g, self.u, self.dyp, self.dxp, *self.dw, self.ws)
        m.moe_combine(c, self.dxp, self.row, self.ones, self.dx)

    def results(self):
        return {"y": self.y, "dx": self.dx, "dtw": self.dtw, "dwg": self.dw[0], "dwu": self.dw[1], "dwd": self.dw[2]}

    def clear(self):
        for t in self.results().values():
            t.fill_(float("nan"))


SHAPES = [mi.MoEShape("few", 5, 128, 192, 4, 2), mi.MoEShape("step", 301, 320, 448, 7, 3, mi.GATE_SOFTMAX_RENORM), mi.MoEShape("dense", 130, 256, 512, 1, 1, mi.GATE_SIGMOID_NORM)]


@pytest.mark.parametrize("s", SHAPES, ids=lambda s: s.name)
def test_a_step_has_the_gradients_of_the_layer(moe, s):
    """Against torch's own differentiation of the layer's formula in 64 bits, for the routing that the router chose."""
    step = Step(moe, s)
    step.run()
    torch.cuda.synchronize()
    leaf = lambda t: t.detach().cpu().double().requires_grad_()  # noqa: E731
    x, w, (wg, wu, wd) = leaf(step.x), leaf(step.tw), [leaf(t) for t in step.w]
    idx = step.idx.cpu().long()
    y = torch.zeros_like(x)
    for e in range(s.E):
        t, i = torch.nonzero(idx == e, as_tuple=True)
        h = torch.nn.functional.silu(x[t] @ wg[e].T) * (x[t] @ wu[e].T)
        y = y.index_add(0, t, w[t, i][:, None] * (h @ wd[e].T))
    y.backward(step.dy.cpu().double())
    _near(step.y, y, 3, "y")                       # h, y_perm, y
    _near(step.dtw, w.grad, 2, "dtw")              # h, y_perm
    _near(step.dx, x.grad, 7, "dx")                # dy_perm, g (two), u, dg and du, dx_perm, dx
    _near(step.dw[0], wg.grad, 6, "dwg")           # dy_perm, g (two), u, dg, dwg
    _near(step.dw[1], wu.grad, 5, "dwu")           # dy_perm, g (two), du, dwu
    _near(step.dw[2], wd.grad, 6, "dwd")           # dy_perm, g (two), u, h, dwd


def test_a_step_is_the_same_every_time_and_in_a_graph(moe):
    """Bit for bit: again, captured, and replayed with other work and other inputs in between."""
    step = Step(moe, SHAPES[1])
    step.run()
    first = {n: t.clone() for n, t in step.results().items()}
    step.clear()
    step.run()
    torch.cuda.synchronize()
    assert all(torch.equal(t, first[n]) for n, t in step.results().items())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.run()
    other = (step.dy.float() * -0.5).to(torch.bfloat16)
    kept = step.dy.clone()
    for i in range(4):
        step.clear()
        step.dy.copy_(other if i == 2 else kept)
        torch.mm(torch.ones(64, 64, device="cuda"), torch.ones(64, 64, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        if i == 2:
            assert not torch.equal(step.dx, first["dx"]) and torch.equal(step.y, first["y"])
        else:
            assert all(torch.equal(t, first[n]) for n, t in step.results().items()), i


def test_two_steps_at_once(moe):
    """Two streams, each with its own workspace and results."""
    a, b = Step(moe, SHAPES[1], seed=3), Step(moe, SHAPES[2], seed=4)
    for st in (a, b):
        st.run()
    torch.cuda.synchronize()
    want = [{n: t.clone() for n, t in st.results().items()} for st in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for st in (a, b):
        st.clear()
    torch.cuda.synchronize()
    for _ in range(5):
        for st, stream in zip((a, b), streams):
            with torch.cuda.stream(stream):
                st.run()
    torch.cuda.synchronize()
    for st, w in zip((a, b), want):
        assert all(torch.equal(t, w[n]) for n, t in st.results().items())


class Shared:
    """A shared expert with per-request adapters behind the routed experts: h = gated, y = routed + down."""

    def __init__(self, moe, T, d, F, n, rank, seed=0):
        rng = np.random.default_rng(seed)
        b = lambda shape, std: torch.from_numpy(rng.normal(size=shape) * std).to(torch.bfloat16)  # noqa: E731
        self.moe, self.n = moe, n
        self.host = {"x": b((T, d), 1), "wg": b((F, d), d ** -0.5), "wu": b((F, d), d ** -0.5), "wd": b((d, F), F ** -0.5), "routed": b((T, d), 1),
                     "ag": b((n, rank, d), d ** -0.5), "au": b((n, rank, d), d ** -0.5), "ad": b((n, rank, F), F ** -0.5),
                     "bg": b((n, F, rank), rank ** -0.5), "bu": b((n, F, rank), rank ** -0.5), "bd": b((n, d, rank), rank ** -0.5)}
        self.ids, self.scale = rng.integers(-1, n, size=T).astype(np.int32), rng.random(n).astype(np.float32) + 0.5
        self.d = {k: t.cuda() for k, t in self.host.items()}
        self.dids, self.dscale = torch.from_numpy(self.ids).cuda(), torch.from_numpy(self.scale).cuda()
        self.up, self.down = moe.AdapterConfig.of(T, F, d, n, rank), moe.AdapterConfig.of(T, d, F, n, rank)
        self.h, self.y = _gpu((T, F)), _gpu((T, d))
        self.ws = _gpu(max(moe.adapter_workspace_size(self.up), moe.adapter_workspace_size(self.down)), torch.uint8)

    def run(self, stream=None):
        d = self.d
        self.moe.moe_adapter_gated_up(self.up, d["x"], d["wg"], d["wu"], d["ag"], d["au"], d["bg"], d["bu"], self.dscale, self.dids, self.h, self.ws, stream=stream)
        self.moe.moe_adapter_linear(self.down, self.h, d["wd"], d["ad"], d["bd"], self.dscale, self.dids, self.y, self.ws, base=d["routed"], stream=stream)


@pytest.mark.parametrize("T,d,F,n,rank", [(1, 256, 512, 3, 16), (37, 320, 576, 20, 8), (140, 512, 256, 9, 72), (600, 192, 1024, 2, 32)])
def test_a_shared_expert_with_adapters(moe, T, d, F, n, rank):
    s = Shared(moe, T, d, F, n, rank)
    s.run()
    torch.cuda.synchronize()
    f = {k: t.double().numpy() for k, t in s.host.items()}
    g = orc.adapter_linear(f["x"], f["wg"], f["ag"], f["bg"], s.scale.astype(np.float64), s.ids)
    u = orc.adapter_linear(f["x"], f["wu"], f["au"], f["bu"], s.scale.astype(np.float64), s.ids)
    y = orc.adapter_linear(orc.silu(g) * u, f["wd"], f["ad"], f["bd"], s.scale.astype(np.float64), s.ids, base=f["routed"])
    _near(s.h, torch.from_numpy(orc.silu(g) * u), 1, "h")
    _near(s.y, torch.from_numpy(y), 2, "y")        # h, y


@pytest.mark.parametrize("T", [3, 100, 400])
def test_adapters_in_a_graph_and_on_another_stream(moe, T):
    s = Shared(moe, T, 256, 512, 6, 16, seed=T)
    s.run()
    torch.cuda.synchronize()
    want = s.y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for i in range(3):
        s.y.fill_(float("nan"))
        s.ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(s.y, want), i
    side = torch.cuda.Stream()
    s.y.fill_(float("nan"))
    side.wait_stream(torch.cuda.current_stream())
    s.run(stream=side)
    side.synchronize()
    assert torch.equal(s.y, want)


def test_calls_that_are_refused_leave_their_results_alone(moe):
    s = Shared(moe, 20, 256, 512, 6, 16)
    s.y.fill_(3.0)
    with pytest.raises(ValueError):
        moe.moe_adapter_linear(s.down, s.h, s.d["wd"].T, s.d["ad"], s.d["bd"], s.dscale, s.dids, s.y, s.ws)                   # strides
    with pytest.raises(ValueError):
        moe.moe_adapter_linear(s.down, s.h, s.d["wd"], s.d["ad"].cpu(), s.d["bd"], s.dscale, s.dids, s.y, s.ws)              # another device
    with pytest.raises(ValueError):
        moe.moe_adapter_linear(s.down, s.h[:19], s.d["wd"], s.d["ad"], s.d["bd"], s.dscale, s.dids, s.y, s.ws)
    with pytest.raises(moe.MoEError) as e:
        moe.moe_adapter_linear(s.down, s.h, s.d["wd"], s.d["ad"], s.d["bd"], s.dscale, s.dids, s.y, s.ws[:16])
    assert e.value.status == -4
    flat = torch.empty(20 * 512 + 4, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(moe.MoEError) as e:
        moe.moe_adapter_linear(s.down, flat[4:].view(20, 512), s.d["wd"], s.d["ad"], s.d["bd"], s.dscale, s.dids, s.y, s.ws)  # 8 bytes off
    assert e.value.status == -3
    torch.cuda.synchronize()
    assert (s.y == 3.0).all()
