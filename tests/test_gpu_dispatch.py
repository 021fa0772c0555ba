"""Rows of slots that may have none, their way back, both gradients, and dropout, against oracle/token_oracle.py.

Bounds, from the arithmetic of each call (u = 2^-24, a rounding to fp32; 2^-8 a rounding to bf16, relative to the rounded value):
  tables, masks        exact
  scattered rows       v = dy scale (u), w v (u), bf16: (2^-8 + 4 u) |row|
  gathered rows        k products and sums in fp32, scale, residual: 2^-8 |y| + 2 (k + 4) u A, A the same sum over absolute values (the second 2 is for the 2^-8 of it)
  dots                 a thread adds up at most d / 64 + 8 products in a row, then ten sums join the threads: 2 (d / 64 + 24) u A
"""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))

from oracle import token_oracle as orc

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8
NAN = float("nan")


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_23911_amd as m
    m.lib()
    return m


def bf(rng, *shape, std=1.0):
    return torch.from_numpy(rng.normal(size=shape) * std).to(torch.bfloat16)


def full(shape, dtype=torch.bfloat16, value=NAN):
    return torch.full(shape, value, dtype=dtype, device="cuda")


def f64(t):
    return t.detach().cpu().double().numpy()


def within(got, want, bound, what):
    off = np.abs(f64(got) - want)
    assert np.isfinite(f64(got)).all() and (off <= bound).all(), (what, float((off / np.maximum(bound, 1e-300)).max()))


def choices(rng, T, k, experts, skew=0.0):
    p = np.arange(1, experts + 1) ** -float(skew)
    return np.stack([rng.choice(experts, k, replace=k > experts, p=p / p.sum()) for _ in range(T)]).astype(np.int32).reshape(T, k)


class Plan:
    def __init__(self, moe, T, d, k, experts, E=None, first=0, capacity=0, skew=0.0, seed=0, idx=None):
        rng = self.rng = np.random.default_rng(seed)
        self.moe, self.T, self.d, self.k, self.R = moe, T, d, k, T * k
        self.cfg = moe.DispatchConfig.of(T, d, k, E or experts, first, capacity)
        self.idx = choices(rng, T, k, experts, skew) if idx is None else idx
        self.counts, self.off, self.row, self.src = orc.tables(self.idx, E or experts, first, capacity)
        self.N = int(self.off[-1])
        self.w = rng.normal(size=(T, k)).astype(np.float32)
        self.x, self.rows = bf(rng, T, d), bf(rng, T * k, d)
        self.rows[self.N:] = NAN                     # nothing may come from rows that no slot has
        self.add = bf(rng, T, d)
        self.mask_key = ((seed * 0x123456789ABCDEF + 77) % (1 << 63), (1 << 40) + seed)
        self.drng = torch.tensor(self.mask_key, dtype=torch.int64, device="cuda")
        self.d_row = torch.from_numpy(self.row.astype(np.int32)).cuda()
        self.d_w = torch.from_numpy(self.w).cuda()

    def dispatch(self, weighted, move=True, stream=None):
        i32 = torch.int32
        E = self.cfg.E
        o = {"counts": full((E,), i32, -7), "offsets": full((E + 1,), i32, -7), "row_of": full((self.T, self.k), i32, -7), "src_of": full((self.R,), i32, -7),
             "rows": full((self.R, self.d), value=7.0) if move else None}
        ws = full((self.moe.dispatch_workspace_size(self.cfg),), torch.uint8, 255)
        self.moe.moe_dispatch(self.cfg, self.x.cuda() if move else None, torch.from_numpy(self.idx).cuda(), self.d_w if weighted else None, o["counts"], o["offsets"], o["row_of"],
                              o["src_of"], o["rows"], ws, stream=stream)
        torch.cuda.synchronize()
        return o

    def check_tables(self, o):
        assert np.array_equal(o["counts"].cpu(), self.counts) and np.array_equal(o["offsets"].cpu(), self.off) and np.array_equal(o["row_of"].cpu(), self.row)
        src = o["src_of"].cpu().numpy()
        assert np.array_equal(src[:self.N], self.src) and (src[self.N:] == -7).all()

    def check_dispatch(self, weighted):
        o = self.dispatch(weighted)
        self.check_tables(o)
        assert (o["rows"][self.N:] == 7.0).all()
        if not weighted:
            assert torch.equal(o["rows"][:self.N].cpu().view(torch.int16), self.x[self.src // self.k].view(torch.int16))
            return
        want = orc.scattered(f64(self.x), self.row, self.w.astype(np.float64), self.R)[:self.N]
        within(o["rows"][:self.N], want, (B + 4 * U) * np.abs(want), "rows")

    def check_collect(self, weighted, add, p, call="collect"):
        w = self.w.astype(np.float64) if weighted else np.ones((self.T, self.k))
        rows = f64(self.rows)
        total, size = orc.gathered(rows, self.row, w), orc.gathered(np.abs(rows), self.row, np.abs(w))
        if p:
            total, size = (orc.dropped(v, p, *self.mask_key) for v in (total, size))
        if add:
            total, size = total + f64(self.add), size + np.abs(f64(self.add))
        y = full((self.T, self.d))
        more = self.add.cuda() if add else None
        if call == "collect":
            self.moe.moe_collect(self.cfg, self.rows.cuda(), self.d_row, self.d_w if weighted else None, y, residual=more, p=p, rng=self.drng if p else None)
        else:
            dw = full((self.T, self.k), torch.float32)
            self.moe.moe_dispatch_backward(self.cfg, self.rows.cuda(), self.d_row, self.d_w if weighted else None, y, x=self.x.cuda(), d_topk_w=dw, base=more)
            self.check_dots(dw, f64(self.x))
            alone = full((self.T, self.d))
            self.moe.moe_dispatch_backward(self.cfg, self.rows.cuda(), self.d_row, self.d_w if weighted else None, alone, base=more)
            assert torch.equal(alone, y)
        within(y, total, B * np.abs(total) + 2 * (self.k + 4) * U * size, "y")

    def check_dots(self, dw, v):
        rows = f64(self.rows)
        within(dw, orc.dots(v, rows, self.row), 2 * (self.d / 64 + 24) * U * orc.dots(np.abs(v), np.abs(rows), self.row), "dw")

    def check_collect_backward(self, weighted, p, dots=True, in_place=False):
        dy = bf(self.rng, self.T, self.d, std=0.1)
        v = orc.dropped(f64(dy), p, *self.mask_key)
        rows = self.rows.cuda()
        drows, dw = rows if in_place else full((self.R, self.d), value=7.0), full((self.T, self.k), torch.float32) if dots else None
        kept = drows[self.N:].clone()
        self.moe.moe_collect_backward(self.cfg, dy.cuda(), rows if dots else None, self.d_row, self.d_w if weighted else None, drows, d_topk_w=dw, p=p, rng=self.drng)
        want = orc.scattered(v, self.row, self.w.astype(np.float64) if weighted else np.ones((self.T, self.k)), self.R)[:self.N]
        within(drows[:self.N], want, (B + 4 * U) * np.abs(want), "drows")
        assert torch.equal(drows[self.N:].view(torch.int16), kept.view(torch.int16))
        if dots:
            self.check_dots(dw, v)


# tokens, width, slots, experts in all, then experts here, the first of them, capacity, skew
PLANS = [(1, 8, 1, 1), (1, 4096, 2, 8), (3, 256, 2, 8, 4, 2), (5, 1032, 3, 7, 7, 0, 2), (64, 1024, 4, 16, 5, 9, 3, 1.0), (65, 1040, 8, 64), (257, 72, 8, 60, 60, 0, 20, 1.5),
         (130, 2048, 5, 9, 3, 6), (301, 320, 12, 32, 20, 4, 50), (40, 2056, 11, 256, 256, 0, 1), (33, 128, 64, 200, 100, 50), (2, 64, 256, 256), (7, 16, 9, 3),
         (700, 64, 12, 40, 40, 0, 100), (1025, 8, 8, 8, 8, 0, 0, 2.0), (9000, 16, 1, 17), (9001, 8, 8, 8, 3, 1, 2000), (5, 48, 2, 100, 2, 90),
         (6, 520, 9, 20), (5, 2064, 13, 40, 30, 5), (5, 264, 15, 30), (6, 1104, 16, 30, 20), (5, 1032, 17, 40, 30), (4, 264, 64, 100, 50, 20), (3, 2056, 256, 256, 200, 9)]


@pytest.mark.parametrize("plan", PLANS, ids=lambda p: "-".join(map(str, p)))
def test_dispatch(moe, plan):
    p = Plan(moe, *plan, seed=len(plan))
    p.check_dispatch(True)
    p.check_dispatch(False)
    p.check_tables(p.dispatch(True, move=False))


@pytest.mark.parametrize("plan", PLANS, ids=lambda p: "-".join(map(str, p)))
def test_dispatch_backward(moe, plan):
    p = Plan(moe, *plan, seed=len(plan))
    for weighted, add in ((True, False), (False, True), (True, True)):
        p.check_collect(weighted, add, 0.0, "dispatch_backward")


@pytest.mark.parametrize("plan", [p for p in PLANS if p[0] * p[1] <= 150_000], ids=lambda p: "-".join(map(str, p)))
def test_collect(moe, plan):
    p = Plan(moe, *plan, seed=len(plan))
    for weighted, add, drop in ((True, False, 0.0), (False, True, 0.0), (True, True, 0.1), (True, False, 0.97), (False, False, 0.5)):
        p.check_collect(weighted, add, drop)


@pytest.mark.parametrize("plan", [p for p in PLANS if p[0] * p[1] <= 150_000], ids=lambda p: "-".join(map(str, p)))
def test_collect_backward(moe, plan):
    p = Plan(moe, *plan, seed=len(plan))
    p.check_collect_backward(True, 0.0)
    p.check_collect_backward(True, 0.1)
    p.check_collect_backward(False, 0.3)
    p.check_collect_backward(True, 0.5, dots=False)
    p.check_collect_backward(False, 0.0, dots=False)
    p.check_collect_backward(True, 0.2, in_place=True)


@pytest.mark.parametrize("plan", [(1, 16), (700, 16), (90_000, 8)], ids=str)
def test_ids_of_no_expert_here(moe, plan):
    """Ids below, above and far outside: no slot has a row, nothing is written but the tables, and tokens come back as their residual (or zero)."""
    T, d = plan
    idx = np.resize(np.array([-1, 3, 8, 2**31 - 1, -2**31, 12, -2**31 + 5], np.int32), (T, 2))
    p = Plan(moe, T, d, 2, 16, E=4, first=4, idx=np.ascontiguousarray(idx))
    o = p.dispatch(True)
    assert p.N == 0
    p.check_tables(o)
    assert (o["rows"] == 7.0).all()
    y = full((T, d))
    moe.moe_collect(p.cfg, p.rows.cuda(), o["row_of"], p.d_w, y, residual=p.add.cuda(), p=0.5, rng=p.drng)
    assert torch.equal(y.cpu(), p.add)
    moe.moe_collect(p.cfg, p.rows.cuda(), o["row_of"], None, y)
    assert (y == 0).all()
    drows, dw = full((p.R, d), value=7.0), full((T, 2), torch.float32)
    inf = torch.full((T, d), float("inf"), dtype=torch.bfloat16, device="cuda")
    moe.moe_collect_backward(p.cfg, inf, p.rows.cuda(), o["row_of"], p.d_w, drows, d_topk_w=dw)
    assert (drows == 7.0).all() and (dw == 0).all()
    moe.moe_dispatch_backward(p.cfg, p.rows.cuda(), o["row_of"], p.d_w, y, x=inf, d_topk_w=dw.fill_(NAN))
    assert (y == 0).all() and (dw == 0).all()


def test_no_tokens(moe):
    p = Plan(moe, 0, 64, 2, 8, idx=np.zeros((0, 2), np.int32))
    o = p.dispatch(True)
    assert (o["counts"] == 0).all() and (o["offsets"] == 0).all()
    o = p.dispatch(False, move=False)
    assert (o["counts"] == 0).all() and (o["offsets"] == 0).all()


def test_one_expert_chosen_by_every_slot(moe):
    """All slots in one counter, one expert twice per token, and a limit that ends inside a workgroup's slots."""
    for T, k, cap in ((600, 4, 0), (600, 4, 1001), (9000, 2, 0), (9000, 2, 17001), (70_000, 1, 66_001)):
        p = Plan(moe, T, 8, k, 256, E=256, capacity=cap, idx=np.full((T, k), 131, np.int32))
        p.check_dispatch(True)


@pytest.mark.parametrize("T,k,experts,cap", [(8192, 1, 8, 0), (8193, 1, 8, 0), (32768, 1, 64, 600), (32769, 1, 64, 600), (4097, 2, 256, 20), (8200, 8, 256, 0), (65536, 1, 60, 0), (65537, 1, 60, 900), (40_000, 12, 33, 0),
                                             (300_000, 4, 256, 4000)])
def test_tables_of_many_slots(moe, T, k, experts, cap):
    """Both sides of the lines between one, two and three launches; against a stable sort."""
    rng = np.random.default_rng(T)
    idx = np.minimum(rng.integers(0, experts, size=(T, k)), rng.integers(0, experts, size=(T, k))).astype(np.int32)
    e = idx.reshape(-1)
    order = np.argsort(e, kind="stable")
    counts = np.bincount(e, minlength=experts)
    rank = np.empty(e.size, np.int64)
    rank[order] = np.arange(e.size) - (np.cumsum(counts) - counts)[e[order]]
    off = np.concatenate([[0], np.cumsum(np.minimum(counts, cap or 1 << 30))])
    row = np.where(rank < (cap or 1 << 30), off[e] + rank, -1)
    d = 8
    cfg = moe.DispatchConfig.of(T, d, k, experts, 0, cap)
    x = (torch.arange(T, device="cuda") % 251).to(torch.bfloat16)[:, None].repeat(1, d).contiguous()
    i32 = torch.int32
    o = [full((experts,), i32, -7), full((experts + 1,), i32, -7), full((T, k), i32, -7), full((T * k,), i32, -7)]
    ws = full((moe.dispatch_workspace_size(cfg),), torch.uint8, 255)
    for move in (True, False):
        rows = full((T * k, d), value=7.0) if move else None
        for t in o:
            t.fill_(-7)
        moe.moe_dispatch(cfg, x if move else None, torch.from_numpy(idx).cuda(), None, *o, rows, ws)
        assert np.array_equal(o[0].cpu(), counts) and np.array_equal(o[1].cpu(), off) and np.array_equal(o[2].cpu().view(-1), row)
        src = np.full(T * k, -7)
        src[row[row >= 0]] = np.nonzero(row >= 0)[0]
        assert np.array_equal(o[3].cpu(), src)
        if move:
            want = torch.from_numpy(np.where(src >= 0, src // k % 251, 7)).to(torch.bfloat16)
            assert torch.equal(rows.cpu(), want[:, None].repeat(1, d))


@pytest.mark.parametrize("k", [1, 2, 3, 5, 8, 12])
@pytest.mark.parametrize("d", [1000, 1024, 1032, 2048, 2056, 4104])
def test_widths(moe, k, d):
    """Around the widths at which a token goes from a wavefront to a workgroup, and rows that end inside a workgroup's stride."""
    p = Plan(moe, 9, d, k, 16, 10, 3, seed=d + k)
    p.check_dispatch(True)
    p.check_collect(True, True, 0.0, "dispatch_backward")
    p.check_collect(True, True, 0.1)
    p.check_collect_backward(True, 0.1)


def test_the_widest_rows(moe):
    p = Plan(moe, 3, 1 << 20, 2, 4, 3, 1)
    p.check_dispatch(True)
    p.check_collect(True, True, 0.0, "dispatch_backward")
    p.check_collect(True, True, 0.0)
    p.check_collect_backward(True, 0.0)


def test_in_place_on_the_residual_and_the_base(moe):
    p = Plan(moe, 33, 264, 3, 8, 6, 1)
    for call in ("collect", "backward"):
        want, got = full((p.T, p.d)), p.add.cuda()
        for out, more in ((want, p.add.cuda()), (got, got)):
            if call == "collect":
                moe.moe_collect(p.cfg, p.rows.cuda(), p.d_row, p.d_w, out, residual=more, p=0.3, rng=p.drng)
            else:
                moe.moe_dispatch_backward(p.cfg, p.rows.cuda(), p.d_row, p.d_w, out, base=more)
        assert torch.equal(want, got)


@pytest.mark.parametrize("k,d", [(1, 8), (3, 64), (12, 136), (3, 264), (11, 1032), (17, 2048)])
def test_gradients_of_rows_in_place_of_the_rows(moe, k, d):
    p = Plan(moe, 41, d, k, 8, 6, 1)
    for weights in (p.d_w, None):
        for drop in (0.0, 0.3):
            rows, dw = p.rows.cuda(), full((p.T, p.k), torch.float32)
            want, want_dw = p.rows.cuda(), full((p.T, p.k), torch.float32)
            moe.moe_collect_backward(p.cfg, p.add.cuda(), p.rows.cuda(), p.d_row, weights, want, d_topk_w=want_dw, p=drop, rng=p.drng)
            moe.moe_collect_backward(p.cfg, p.add.cuda(), rows, p.d_row, weights, rows, d_topk_w=dw, p=drop, rng=p.drng)
            assert torch.equal(rows.view(torch.int16), want.view(torch.int16)) and torch.equal(dw, want_dw)         # bits: rows of no slot hold NaN


def test_infinities_stay_where_they_belong(moe):
    """NaN and infinities of a row reach its token alone; what dropout takes out is zero, whatever it was; a weight of a slot without a row is not used."""
    p = Plan(moe, 50, 136, 3, 8, 5, 1, capacity=12, seed=5)
    rows, w = p.rows.clone(), p.w.copy()
    hit = int(p.row[p.row >= 0][7])
    t_hit = int(p.src[hit] // p.k)
    rows[hit] = float("inf")
    w[p.row < 0] = NAN
    y = full((p.T, p.d))
    moe.moe_collect(p.cfg, rows.cuda(), p.d_row, torch.from_numpy(w).cuda(), y, p=0.5, rng=p.drng)
    keep = torch.from_numpy(orc.keep(p.T * p.d, 0.5, *p.mask_key).reshape(p.T, p.d))
    got = y.cpu()
    assert torch.isinf(got[t_hit][keep[t_hit]]).all() and (got[~keep] == 0).all()
    assert torch.isfinite(got[torch.arange(p.T) != t_hit]).all()
    dy = p.add.clone()
    dy[t_hit] = NAN
    drows, dw = full((p.R, p.d), value=7.0), full((p.T, p.k), torch.float32, 3.0)
    moe.moe_collect_backward(p.cfg, dy.cuda(), p.rows.cuda(), p.d_row, torch.from_numpy(w).cuda(), drows, d_topk_w=dw, p=0.5, rng=p.drng)
    drows, dw = drows.cpu(), dw.cpu()
    of_hit = torch.from_numpy(p.src // p.k == t_hit)
    assert torch.isfinite(drows[:p.N][~of_hit]).all() and (drows[:p.N][of_hit][:, ~keep[t_hit]] == 0).all() and torch.isnan(drows[:p.N][of_hit][:, keep[t_hit]]).all()
    assert (dw[torch.from_numpy(p.row < 0)] == 0).all() and torch.isfinite(dw[torch.arange(p.T) != t_hit]).all()


def test_row_numbers_outside_the_buffer_are_slots_without_a_row(moe):
    p = Plan(moe, 20, 64, 2, 8)
    row = p.row.copy()
    row[3, 1], row[7, 0], row[11] = p.R, 2**31 - 1, -5
    p.row = np.where((row < 0) | (row >= p.R), -1, row)
    p.d_row = torch.from_numpy(row.astype(np.int32)).cuda()
    p.check_collect(True, False, 0.0)
    p.check_collect(True, False, 0.0, "dispatch_backward")
    want = orc.scattered(f64(p.x), p.row, p.w.astype(np.float64), p.R)
    drows = full((p.R, p.d), value=0.0)
    moe.moe_collect_backward(p.cfg, p.x.cuda(), None, p.d_row, p.d_w, drows)
    within(drows, want, (B + 4 * U) * np.abs(want), "drows")


# ---- dropout alone -------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("n", [1, 7, 8, 9, 2047, 2048, 2049, 65_543])
@pytest.mark.parametrize("p", [0.0, 2.0**-16, 0.1, 0.5, 65535 / 65536])
def test_dropout(moe, n, p):
    rng = np.random.default_rng(n)
    x, add = bf(rng, n), bf(rng, n)
    key = (0xFEDCBA9876543210 - (1 << 64), -3)           # negative as int64: the bits count
    state = torch.tensor(key, dtype=torch.int64, device="cuda")
    y = full((n,))
    moe.moe_dropout(x.cuda(), y, p, state)
    want = orc.dropped(f64(x), p, key[0] & (1 << 64) - 1, key[1] & (1 << 64) - 1)
    within(y, want, (B + 2 * U) * np.abs(want), "y")
    assert np.array_equal(f64(y) == 0, want == 0)
    moe.moe_dropout(x.cuda(), y, p, state, residual=add.cuda())
    want = want + f64(add)
    within(y, want, B * np.abs(want) + 2 * U * (np.abs(want) + 2 * np.abs(f64(add))), "y with residual")
    for inout in (x, add):                               # in place
        z, other = inout.cuda(), (add if inout is x else x).cuda()
        moe.moe_dropout(z if inout is x else other, z, p, state, residual=other if inout is x else z)
        assert torch.equal(z, y)


def test_dropout_of_a_long_tensor(moe):
    """More than the launch's threads take at once, against the collected form of the same elements (one row per token, no weights): one mask."""
    T, d = 20_000, 1024
    x = torch.randn((T, d), device="cuda").to(torch.bfloat16)
    state = torch.tensor([5, 9], dtype=torch.int64, device="cuda")
    y, z = full((T, d)), full((T, d))
    moe.moe_dropout(x, y, 0.3, state)
    row = torch.arange(T, dtype=torch.int32, device="cuda").view(T, 1)
    moe.moe_collect(moe.DispatchConfig.of(T, d, 1, 1), x, row, None, z, p=0.3, rng=state)
    assert torch.equal(y, z)
    kept = float((y != 0).float().mean())
    assert abs(kept - 0.7) < 5 * (0.21 / (T * d)) ** 0.5 + 2.0**-16
    flat = (y.view(-1)[:4000] != 0).cpu().numpy()
    assert np.array_equal(flat, orc.keep(4000, 0.3, 5, 9) & (f64(x.view(-1)[:4000]) != 0))
