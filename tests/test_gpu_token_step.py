"""A whole training step with slots that have no row, residual, dropout and the router's gradient, as a program uses the operators together; and the ways in which the calls
meet: captured and replayed with other masks, two at once on two streams, shared workspaces, misplaced tensors.

End to end: a result went through n roundings to bf16 whose errors are independent and at most 2^-8 of the rounded value each, so that each adds at most 2^-8 of the
result's norm; SiLU' passes a rounding of g on by |g SiLU''(g) / SiLU'(g)|, which is counted as two.  n is given with each check."""
import os
import sys
import threading

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))

import moe_inputs as mi
from oracle import token_oracle as orc

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
    """Forward and backward of y = x + dropout(sum_i w_i FFN_i(x)) on the GPU that holds experts first .. first + E - 1 of s.E; `inside`: the weights are applied to the
    experts' inputs instead."""

    def __init__(self, moe, s, E, first=0, capacity=0, p=0.0, inside=False, seed=0):
        self.moe, self.s, self.E, self.first, self.capacity, self.p, self.inside = moe, s, E, first, capacity, p, inside
        T, k, R, d, F = s.T, s.k, s.R, s.d, s.F
        self.route = moe.MoEConfig.of(T, d, F, s.E, k, s.gating)
        self.disp = moe.DispatchConfig.of(T, d, k, E, first, capacity)
        self.ffn = moe.MoEConfig.of(R, d, F, E, 1)              # the rows as tokens of one slot: k may be more than the experts that are here
        self.x, self.wr = mi.make_x(s, seed).cuda(), mi.make_router(s, seed).cuda()
        self.w = [t[first:first + E].contiguous().cuda() for t in mi.make_all_experts(s, seed)]
        self.dy = (mi.make_x(s, seed + 1).float() * 0.1).to(torch.bfloat16).cuda()
        self.bias = torch.linspace(-0.5, 0.5, s.E, device="cuda")
        self.rng = torch.tensor([seed + 11, 1000], dtype=torch.int64, device="cuda")
        i32, f32, u8 = torch.int32, torch.float32, torch.uint8
        self.idx, self.tw, self.counts, self.off = _gpu((T, k), i32), _gpu((T, k), f32), _gpu(E, i32), _gpu(E + 1, i32)
        self.row, self.src, self.xp = _gpu((T, k), i32), _gpu(R, i32), _gpu((R, d))
        self.g, self.u, self.h, self.yp, self.y = _gpu((R, F)), _gpu((R, F)), _gpu((R, F)), _gpu((R, d)), _gpu((T, d))
        self.dyp, self.dtw, self.dxp, self.dxr, self.dx = _gpu((R, d)), _gpu((T, k), f32), _gpu((R, d)), _gpu((T, d)), _gpu((T, d))
        self.dw = [torch.empty_like(t) for t in self.w]
        self.dwr, self.dbias = _gpu((s.E, d), f32), _gpu(s.E, f32)
        self.ws = _gpu(max(moe.route_workspace_size(self.route), moe.dispatch_workspace_size(self.disp), moe.ffn_workspace_size(self.ffn),
                           moe.ffn_backward_workspace_size(self.ffn), moe.route_backward_workspace_size(self.route)), u8)

    def run(self, stream=None):
        m = self.moe
        st = {"stream": stream}
        outer = None if self.inside else self.tw
        m.moe_route(self.route, self.x, self.wr, self.bias, self.idx, self.tw, self.ws, **st)
        m.moe_dispatch(self.disp, self.x, self.idx, self.tw if self.inside else None, self.counts, self.off, self.row, self.src, self.xp, self.ws, **st)
        m.moe_grouped_ffn_train(self.ffn, self.xp, self.off, *self.w, self.g, self.u, self.h, self.yp, self.ws, **st)
        m.moe_collect(self.disp, self.yp, self.row, outer, self.y, residual=self.x, p=self.p, rng=self.rng, **st)
        m.moe_collect_backward(self.disp, self.dy, self.yp, self.row, outer, self.dyp, d_topk_w=None if self.inside else self.dtw, p=self.p, rng=self.rng, **st)
        m.moe_grouped_ffn_backward(self.ffn, self.xp, self.off, *self.w, self.g, self.u, self.dyp, self.dxp, *self.dw, self.ws, **st)
        if self.inside:         # the weights' gradient comes from the rows' inputs; the residual's gradient is dy
            m.moe_dispatch_backward(self.disp, self.dxp, self.row, self.tw, self.dx, x=self.x, d_topk_w=self.dtw, base=self.dy, **st)
            m.moe_route_backward(self.route, self.x, self.wr, self.bias, self.idx, self.tw, self.dtw, self.dxr, self.dwr, self.dbias, self.ws, **st)
        else:
            m.moe_route_backward(self.route, self.x, self.wr, self.bias, self.idx, self.tw, self.dtw, self.dxr, self.dwr, self.dbias, self.ws, **st)
            m.moe_dispatch_backward(self.disp, self.dxp, self.row, None, self.dx, base=self.dxr, **st)

    def results(self):
        return {"y": self.y, "dx": self.dx, "dxr": self.dxr, "dtw": self.dtw, "dwg": self.dw[0], "dwu": self.dw[1], "dwd": self.dw[2], "dwr": self.dwr, "dbias": self.dbias}

    def clear(self):
        for t in self.results().values():
            t.fill_(float("nan"))


STEPS = [(mi.MoEShape("few", 5, 128, 192, 4, 2), 4, 0, 0, 0.0, False), (mi.MoEShape("limit", 301, 320, 448, 7, 3, mi.GATE_SOFTMAX_RENORM), 7, 0, 100, 0.1, False),
         (mi.MoEShape("share", 257, 192, 320, 12, 4, mi.GATE_SIGMOID_NORM), 3, 5, 0, 0.25, False), (mi.MoEShape("inside", 130, 256, 512, 6, 2), 4, 1, 50, 0.2, True)]


@pytest.mark.parametrize("step", STEPS, ids=lambda s: s[0].name)
def test_a_step_has_the_gradients_of_the_layer(moe, step):
    """Against torch's own differentiation in 64 bits of the layer's formula, from the input to the router's weights, for the slots that got a row."""
    s, E, first, capacity, p, inside = step
    st = Step(moe, *step)
    st.run()
    torch.cuda.synchronize()
    leaf = lambda t: t.detach().cpu().double().requires_grad_()  # noqa: E731
    x, wr, bias, (wg, wu, wd) = leaf(st.x), leaf(st.wr), leaf(st.bias), [leaf(t) for t in st.w]
    idx = st.idx.cpu().long()
    z = x @ wr.T + bias
    top = torch.gather(z, 1, idx)
    w = torch.gather(torch.softmax(z, 1), 1, idx) if s.gating == mi.GATE_SOFTMAX else torch.softmax(top, 1) if s.gating == mi.GATE_SOFTMAX_RENORM else \
        torch.sigmoid(top) / torch.sigmoid(top).sum(1, keepdim=True)
    counts, off, row, _ = orc.tables(idx.numpy(), E, first, capacity)
    assert np.array_equal(st.row.cpu(), row) and np.array_equal(st.off.cpu(), off) and (row < 0).any() == bool(capacity or E < s.E)
    total = torch.zeros_like(x)
    for e in range(E):
        t, i = np.nonzero((idx.numpy() == first + e) & (row >= 0))
        t, i = torch.from_numpy(t), torch.from_numpy(i)
        a = x[t] * w[t, i][:, None] if inside else x[t]
        f = (torch.nn.functional.silu(a @ wg[e].T) * (a @ wu[e].T)) @ wd[e].T
        total = total.index_add(0, t, f if inside else w[t, i][:, None] * f)
    if p:
        keep = torch.from_numpy(orc.keep(s.T * s.d, p, 11, 1000).reshape(s.T, s.d))
        total = torch.where(keep, total * (65536 / (65536 - orc.limit(p))), 0.0)
    y = x + total
    y.backward(st.dy.cpu().double())
    # the residual path adds its gradient to x as it is; `inside` takes it in, the other order leaves it to the caller
    dx = x.grad if inside else x.grad - st.dy.cpu().double()
    more = inside                               # one rounding more: the weighted rows that everything reads
    _near(st.y, y, 4 + more, "y")
    got = st.dx.cpu().double() + (st.dxr.cpu().double() if inside else 0)
    _near(got, dx, 9 + more, "dx")              # dy_perm, g (two), u, dg and du, dx_perm, dxr, dx
    for n, got, want, r in (("dwg", st.dw[0], wg, 6), ("dwu", st.dw[1], wu, 5), ("dwd", st.dw[2], wd, 6)):
        _near(got, want.grad, r + more, n)
    # h, y_perm (inside: g, u, dyp, dg, du, dxp); the gates' differences of weights' gradients can cancel: their own size counts
    n = 7 if inside else 2
    scale = float((torch.linalg.norm(wr.grad)))
    off = float((st.dwr.cpu().double() - wr.grad).norm())
    dtw = st.dtw.cpu().double()
    spread = float(torch.linalg.norm(_route(x, w, idx, dtw, z, s.gating).abs().T @ x.abs().detach()))
    assert off <= n * B * max(scale, spread), ("dwr", off, scale, spread)
    assert float((st.dbias.cpu().double() - bias.grad).norm()) <= n * B * max(float(bias.grad.norm()), float(torch.linalg.norm(_route(x, w, idx, dtw, z, s.gating).abs().sum(0))))


def _route(x, w, idx, dtw, z, gating):
    """The gates' gradient with every difference taken as a sum: what its terms add up to."""
    z, w = z.detach(), w.detach()
    out = torch.zeros_like(z)
    c = (w * dtw.abs()).sum(1, keepdim=True)
    if gating == mi.GATE_SOFTMAX:
        out += torch.softmax(z, 1) * c
    return out.scatter_add(1, idx, w * (dtw.abs() + c))


def test_the_same_every_time_and_in_a_graph_with_other_masks(moe):
    """Bit for bit: again, captured, and replayed with the generator's offset moved on the device between the replays and other work in between."""
    st = Step(moe, *STEPS[1])
    want = {}
    for offset in (1000, 1001):
        st.rng[1] = offset
        st.clear()
        st.run()
        want[offset] = {n: t.clone() for n, t in st.results().items()}
    assert not torch.equal(want[1000]["y"], want[1001]["y"]) and not torch.equal(want[1000]["dwr"], want[1001]["dwr"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.run()
    for i in range(5):
        offset = 1000 + i % 2
        st.rng[1] = offset
        st.clear()
        st.ws.fill_(255)
        torch.mm(torch.ones(64, 64, device="cuda"), torch.ones(64, 64, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, want[offset][n]) for n, t in st.results().items()), i


def test_two_graphs_that_share_a_workspace_one_after_the_other(moe):
    a, b = Step(moe, *STEPS[1]), Step(moe, *STEPS[2])
    a.ws = b.ws = max((a.ws, b.ws), key=lambda t: t.numel())
    graphs, want = [], []
    for st in (a, b):
        st.run()
        torch.cuda.synchronize()
        want.append({n: t.clone() for n, t in st.results().items()})
    for st in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            st.run()
        graphs.append(g)
    for _ in range(3):
        for st in (a, b):
            st.clear()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for st, w in zip((a, b), want):
            assert all(torch.equal(t, w[n]) for n, t in st.results().items())


def test_two_steps_at_once(moe):
    """Two streams, handed over as arguments, each with its own workspace and results."""
    a, b = Step(moe, *STEPS[2], seed=3), Step(moe, *STEPS[3], seed=4)
    want = []
    for st in (a, b):
        st.run()
        torch.cuda.synchronize()
        want.append({n: t.clone() for n, t in st.results().items()})
        st.clear()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, stream in zip((a, b), streams):
            st.run(stream=stream)
    torch.cuda.synchronize()
    for st, w in zip((a, b), want):
        assert all(torch.equal(t, w[n]) for n, t in st.results().items())


def test_two_host_threads(moe):
    """Each with a stream, a workspace and tensors of its own."""
    steps = [Step(moe, *STEPS[i], seed=5 + i) for i in (1, 3)]
    want = []
    for st in steps:
        st.run()
        torch.cuda.synchronize()
        want.append({n: t.clone() for n, t in st.results().items()})
        st.clear()
    torch.cuda.synchronize()
    failed = []

    def work(st):
        try:
            stream = torch.cuda.Stream()
            for _ in range(20):
                st.run(stream=stream)
            stream.synchronize()
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work, args=(st,)) for st in steps]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    for st, w in zip(steps, want):
        assert all(torch.equal(t, w[n]) for n, t in st.results().items())


def test_a_share_of_every_gpu_adds_up_to_the_whole(moe):
    """Three GPUs' shares of the experts, one after the other here: with the residual handed on, the tokens' sums are those of all experts (three roundings more)."""
    s = mi.MoEShape("whole", 200, 256, 320, 9, 4)
    whole = Step(moe, s, 9)
    whole.run()
    x, total = whole.x, None
    for first in (0, 3, 6):
        st = Step(moe, s, 3, first)
        st.run()
        part = _gpu((s.T, s.d))
        st.moe.moe_collect(st.disp, st.yp, st.row, st.tw, part, residual=x if total is None else total)
        total = part
    torch.cuda.synchronize()
    # y and the three partial sums are rounded once each
    size = float(whole.y.double().norm())
    assert float((total.double() - whole.y.double()).norm()) <= 4 * B * size


@pytest.mark.parametrize("T", [1, 24, 300])
@pytest.mark.parametrize("packed", [True, False])
def test_serving_a_share_of_the_experts(moe, T, packed):
    """The inference block over the rows that a share of the experts has (fewer than T k, for some tokens none), and the way back onto the residual stream: for each token the
    paper's sum over the experts that are here (h, y_perm and y are rounded once each)."""
    s = mi.MoEShape("serve", T, 256, 320, 8, 3)
    E, first = 3, 4
    x, wr = mi.make_x(s).cuda(), mi.make_router(s).cuda()
    w = [t[first:first + E].contiguous().cuda() for t in mi.make_all_experts(s)]
    route, disp, ffn = moe.MoEConfig.of(T, s.d, s.F, s.E, s.k), moe.DispatchConfig.of(T, s.d, s.k, E, first), moe.MoEConfig.of(T * s.k, s.d, s.F, E, 1)
    i32, f32 = torch.int32, torch.float32
    idx, tw, counts, off, row, src = _gpu((T, s.k), i32), _gpu((T, s.k), f32), _gpu(E, i32), _gpu(E + 1, i32), _gpu((T, s.k), i32), _gpu(T * s.k, i32)
    rows, h, yp, y = _gpu((T * s.k, s.d)), _gpu((T * s.k, s.F)), _gpu((T * s.k, s.d)).fill_(float("nan")), _gpu((T, s.d))
    ws = _gpu(max(moe.route_workspace_size(route), moe.dispatch_workspace_size(disp), moe.ffn_workspace_size(ffn)), torch.uint8)
    W = None
    if packed:
        W = _gpu(moe.packed_weights_size(ffn), torch.uint8)
        moe.moe_pack_weights(ffn, *w, W)
    moe.moe_route(route, x, wr, None, idx, tw, ws)
    moe.moe_dispatch(disp, x, idx, None, counts, off, row, src, rows, ws)
    moe.moe_grouped_ffn(ffn, rows, off, *((None,) * 3 if packed else w), h, yp, ws, W_packed=W)
    moe.moe_collect(disp, yp, row, tw, y, residual=x)
    torch.cuda.synchronize()
    xx, ii, want = x.cpu().double(), idx.cpu(), x.cpu().double()
    for e in range(E):
        t, i = torch.nonzero(ii == first + e, as_tuple=True)
        g, u, d = (m[e].cpu().double() for m in w)
        f = (torch.nn.functional.silu(xx[t] @ g.T) * (xx[t] @ u.T)) @ d.T
        want = want.index_add(0, t, tw.cpu().double()[t, i][:, None] * f)
    _near(y, want, 3, "y")
    none = ~((ii >= first) & (ii < first + E)).any(1)
    assert torch.equal(y.cpu()[none], x.cpu()[none])


def test_calls_that_are_refused_leave_their_results_alone(moe):
    st = Step(moe, *STEPS[1])
    st.run()
    st.y.fill_(3.0)
    st.dx.fill_(3.0)
    c = st.disp
    with pytest.raises(ValueError):
        moe.moe_collect(c, st.yp, st.row, st.tw.cpu(), st.y)
    with pytest.raises(ValueError):
        moe.moe_collect(c, st.yp.T, st.row, st.tw, st.y)
    with pytest.raises(ValueError):
        moe.moe_collect(c, st.yp, st.row.T.contiguous().T, st.tw, st.y)
    with pytest.raises(ValueError, match="rng"):
        moe.moe_collect(c, st.yp, st.row, st.tw, st.y, p=0.1)
    with pytest.raises(moe.MoEError):
        moe.moe_collect(c, st.yp, st.row, st.tw, st.y, p=1.0, rng=st.rng)
    with pytest.raises(ValueError, match="x is required"):
        moe.moe_dispatch_backward(c, st.dxp, st.row, st.tw, st.dx, d_topk_w=st.dtw)
    with pytest.raises(moe.MoEError) as e:
        moe.moe_route_backward(st.route, st.x, st.wr, st.bias, st.idx, st.tw, st.dtw, st.dx, st.dwr, st.dbias, st.ws[:256])
    assert e.value.status == -4
    flat = torch.empty(st.s.T * st.s.d + 4, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(moe.MoEError) as e:
        moe.moe_dropout(flat[4:].view(st.s.T, st.s.d), st.y, 0.5, st.rng)
    assert e.value.status == -3
    torch.cuda.synchronize()
    assert (st.y == 3.0).all() and (st.dx == 3.0).all()
