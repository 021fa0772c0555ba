"""Calls that take the large tiles, or the sum of dx in pieces, captured and replayed with other work in between, and two at once on two streams with a workspace
each: bit for bit what the calls give alone."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(__file__))

from test_gpu_adapter import Case
from test_gpu_ffn_train import Block

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_23911_amd as m
    m.lib()
    return m


class Adapters:
    def __init__(self, moe, T, N, matrices, seed):
        self.moe, self.two = moe, matrices == 2
        self.c = Case(T, N, 192, 9, 24, "mixed", seed=seed, two=self.two).gpu(moe)

    def run(self):
        c, d = self.c, self.c.d
        if self.two:
            self.moe.moe_adapter_gated_up(c.cfg, d["x"], *d["w"], *d["a"], *d["b"], d["scale"], d["ids"], c.y, c.ws)
        else:
            self.moe.moe_adapter_linear(c.cfg, d["x"], d["w"][0], d["a"][0], d["b"][0], d["scale"], d["ids"], c.y, c.ws)

    def results(self):
        return [self.c.y]

    def scratch(self):
        return self.c.ws


class Training:
    def __init__(self, moe, counts, d, F, seed):
        self.moe = moe
        self.b = Block(counts, d, F, seed=seed).to_gpu(moe)
        b, bf = self.b, torch.bfloat16
        self.g, self.u, self.h = (torch.empty((b.R, F), dtype=bf, device="cuda") for _ in range(3))
        self.y, self.o = torch.empty((b.R, d), dtype=bf, device="cuda"), b.grads()
        self.ws = torch.empty(max(moe.ffn_workspace_size(b.cfg), moe.ffn_backward_workspace_size(b.cfg)), dtype=torch.uint8, device="cuda")

    def run(self):
        b, v = self.b, self.b.dev
        self.moe.moe_grouped_ffn_train(b.cfg, v["x"], b.offsets, v["wg"], v["wu"], v["wd"], self.g, self.u, self.h, self.y, self.ws)
        b.backward(self.moe, self.o, ws=self.ws)

    def results(self):
        return [self.g, self.u, self.h, self.y, *self.o.values()]

    def scratch(self):
        return self.ws


# what is run, and the tiles that it is for
KINDS = {
    "adapters Wide": lambda m, s: (Adapters(m, 513, 14400, 1, s), "Wide"), "adapters Tall": lambda m, s: (Adapters(m, 200, 14400, 2, s), "Tall"),
    "adapters Small": lambda m, s: (Adapters(m, 300, 8256, 1, s), "Small"),
    "block, wide F": lambda m, s: (Training(m, [30, 100, 150, 250], 192, 8256, s), ("Wide", "Deep", "Small, sum in pieces", "Pair")),
    "block, wide d": lambda m, s: (Training(m, [190, 256, 0, 65, 320], 8256, 192, s), ("Small", "Small", "Deep", "Pair")),
    "block, Tall": lambda m, s: (Training(m, [129, 140, 0, 70, 200], 320, 192, s), ("Tall", "Tall", "Tall", "Small")),
}


def _make(moe, kind, seed):
    from paper_2605_23911_amd import binding
    call, tiles = KINDS[kind](moe, seed)
    if isinstance(call, Adapters):
        assert binding.adapter_tiles(call.c.cfg, 2 if call.two else 1) == tiles
    else:
        assert tuple(binding.train_tiles(call.b.cfg, p) for p in ("forward", "dh", "dx", "dw")) == tiles
    call.run()
    torch.cuda.synchronize()
    return call, [t.clone() for t in call.results()]


def _clear(call):
    for t in call.results():
        t.fill_(float("nan"))
    call.scratch().fill_(255)              # NaN wherever it is read unwritten


def _same(call, want):
    return all(torch.equal(t, w) for t, w in zip(call.results(), want))


@pytest.mark.parametrize("kind", KINDS)
def test_captured(moe, kind):
    print(kind, flush=True)
    call, want = _make(moe, kind, 20)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call.run()
    for i in range(4):
        _clear(call)
        torch.mm(torch.ones(64, 64, device="cuda"), torch.ones(64, 64, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert _same(call, want), i


@pytest.mark.parametrize("one,other", [("adapters Wide", "adapters Tall"), ("block, wide F", "block, wide d"), ("block, Tall", "adapters Small")])
def test_two_at_once(moe, one, other):
    print(one, other, flush=True)
    calls = [_make(moe, one, 21), _make(moe, other, 22)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for call, _ in calls:
        _clear(call)
    torch.cuda.synchronize()
    for _ in range(6):
        for (call, _), stream in zip(calls, streams):
            with torch.cuda.stream(stream):
                call.run()
    torch.cuda.synchronize()
    assert all(_same(call, want) for call, want in calls)
