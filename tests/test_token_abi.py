"""Host-side checks of the operators over slots that may have no row, of dropout and of the router's gradient: sizes, refusals, what is allowed to be missing, and what
the Python entry points say of a missing argument.  No GPU is involved: every call has to fail, or to have nothing to do, on the host."""
import ctypes as C
import math
import re

import pytest
import torch

import paper_2605_23911_amd as moe
from test_train_binding import Tensor

P = 4096            # an address that no call below may touch
I32, F32, BF16 = torch.int32, torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def L():
    return moe.lib()


def _ref(c):
    return C.byref(c) if c is not None else None


def _dispatch(L, c, size=1 << 40, **bad):
    a = dict(x=P, idx=P, w=P, counts=P, off=P, row=P, src=P, rows=P, ws=P)
    a.update(bad)
    return L.moe_dispatch(_ref(c), a["x"], a["idx"], a["w"], a["counts"], a["off"], a["row"], a["src"], a["rows"], a["ws"], size, None)


def _dispatch_backward(L, c, **bad):
    a = dict(x=P, drows=P, row=P, w=P, base=P, dx=P, dw=P)
    a.update(bad)
    return L.moe_dispatch_backward(_ref(c), a["x"], a["drows"], a["row"], a["w"], a["base"], a["dx"], a["dw"], None)


def _collect(L, c, p=0.1, **bad):
    a = dict(rows=P, row=P, w=P, res=P, rng=P, y=P)
    a.update(bad)
    return L.moe_collect(_ref(c), a["rows"], a["row"], a["w"], a["res"], p, a["rng"], a["y"], None)


def _collect_backward(L, c, p=0.1, **bad):
    a = dict(dy=P, rows=P, row=P, w=P, rng=P, drows=P, dw=P)
    a.update(bad)
    return L.moe_collect_backward(_ref(c), a["dy"], a["rows"], a["row"], a["w"], p, a["rng"], a["drows"], a["dw"], None)


def _dropout(L, n=64, p=0.1, **bad):
    a = dict(x=P, res=P, rng=P, y=P)
    a.update(bad)
    return L.moe_dropout(n, a["x"], a["res"], p, a["rng"], a["y"], None)


def _route(L, c, flags=0, size=1 << 40, **bad):
    a = dict(x=P, wr=P, bias=P, idx=P, w=P, g=P, dx=P, dwr=P, dbias=P, ws=P)
    a.update(bad)
    return L.moe_route_backward(_ref(c), a["x"], a["wr"], a["bias"], a["idx"], a["w"], a["g"], a["dx"], a["dwr"], a["dbias"], flags, a["ws"], size, None)


ALL = (_dispatch, _dispatch_backward, _collect, _collect_backward)
D = moe.DispatchConfig.of


@pytest.mark.parametrize("call,names", [(_dispatch, "x idx counts off row src rows ws"), (_dispatch_backward, "x drows row dx"), (_collect, "rows row rng y"),
                                        (_collect_backward, "dy rows row rng drows")], ids=lambda v: getattr(v, "__name__", ""))
def test_missing_pointers(L, call, names):
    c = D(64, 256, 2, 8)
    assert call(L, None) == -1
    for n in names.split():
        assert call(L, c, **{n: None}) == -1, n


def test_alignment(L):
    c = D(64, 256, 2, 8)
    for call, names in ((_dispatch, "x rows ws"), (_dispatch_backward, "x drows base dx"), (_collect, "rows res y"), (_collect_backward, "dy rows drows")):
        for n in names.split():
            assert call(L, c, **{n: P + 8}) == -3, (call.__name__, n)
    for call in (_collect, _collect_backward):
        assert call(L, c, rng=P + 4) == -3
    for n in ("x", "res", "y"):
        assert _dropout(L, **{n: P + 8}) == -3, n
    assert _dropout(L, rng=P + 4) == -3
    r = moe.MoEConfig.of(64, 256, 64, 8, 2)
    for n in ("x", "wr", "dx", "dwr"):
        assert _route(L, r, **{n: P + 8}) == -3, n
    assert _route(L, r, ws=P + 16) == -3


def test_shapes(L):
    for bad, status in ((D(-1, 64, 2, 8), -2), (D(4, 0, 2, 8), -2), (D(4, 64, 0, 8), -2), (D(4, 64, 2, 0), -2), (D(4, 64, 2, 8, -1), -2), (D(4, 64, 2, 8, 0, -1), -2),
                        (D(4, 64, 2, 8, 2**31 - 8), -2), (D(4, 60, 2, 8), -5), (D(4, (1 << 20) + 8, 2, 8), -5), (D(4, 64, 257, 8), -5), (D(4, 64, 2, 257), -5),
                        (D((1 << 29) + 1, 64, 2, 8), -5)):
        for call in ALL:
            assert call(L, bad) == status, (call.__name__, [getattr(bad, f) for f, _ in bad._fields_])
        assert moe.dispatch_workspace_size(bad) == 0
    assert moe.dispatch_workspace_size(D(1 << 20, 64, 256, 256, 2**31 - 1 - 256)) > 0
    assert _dispatch(L, D(64, 256, 2, 8), size=0) == -4
    big = D(1 << 20, 64, 8, 64)
    assert _dispatch(L, big, size=moe.dispatch_workspace_size(big) - 1) == -4
    assert moe.dispatch_workspace_size(big) >= (1 << 23) // 1024 * 64 * 4


def test_dropout_refuses(L):
    for p in (-0.1, 1.0, 1.5, math.nan, math.inf, -math.inf, 1 - 2.0**-18):
        assert _dropout(L, p=p) == -2 and _collect(L, D(64, 256, 2, 8), p) == -2 and _collect_backward(L, D(64, 256, 2, 8), p) == -2, p
    assert _dropout(L, n=-1) == -2 and _dropout(L, n=(1 << 40) + 1) == -5
    for n in ("x", "y", "rng"):
        assert _dropout(L, **{n: None}) == -1, n
    assert _dropout(L, n=0, x=None, y=None) == 0 and _dropout(L, n=0, p=0.0, rng=None) == 0


def test_nothing_to_do(L):
    z = D(0, 256, 2, 8)
    assert _dispatch_backward(L, z, x=None, drows=None, row=None, w=None, base=None, dx=None, dw=None) == 0
    assert _collect(L, z, rows=None, row=None, w=None, res=None, y=None) == 0
    assert _collect_backward(L, z, dy=None, rows=None, row=None, w=None, drows=None, dw=None) == 0
    assert _collect(L, z, 0.0, rng=None) == 0
    m = moe.MoEConfig.of
    assert _route(L, m(0, 256, 64, 8, 2), x=None, idx=None, w=None, g=None, dx=None, dwr=None, dbias=None) == 0
    assert _route(L, m(0, 256, 64, 8, 2), 2) == 0                      # added to, by no token
    assert _route(L, m(64, 256, 64, 8, 2), dx=None, dwr=None, dbias=None) == 0


def test_route_backward_refuses(L):
    m = moe.MoEConfig.of
    c = m(64, 256, 64, 8, 2)
    assert _route(L, None) == -1
    for n in ("x", "wr", "idx", "w", "g", "ws"):
        assert _route(L, c, **{n: None}) == -1, n
    assert _route(L, c, 4) == -2 and _route(L, c, -1) == -2
    assert _route(L, c, size=moe.route_backward_workspace_size(c) - 1) == -4
    for bad, status in ((m(-1, 256, 64, 8, 2), -2), (m(4, 250, 64, 8, 2), -5), (m(4, 256, 64, 257, 2), -5), (m(4, 256, 64, 8, 9), -2), (m(1, (1 << 20) + 64, 64, 8, 2), -5),
                        (m(4, 256, 64, 8, 2, 3), -2)):
        assert _route(L, bad) == status and moe.route_backward_workspace_size(bad) == 0


@pytest.mark.parametrize("d,E,k", [(7168, 256, 8), (4096, 8, 2), (3584, 64, 8), (2048, 128, 8), (64, 40, 3), (64, 65, 1)])
def test_a_workspace_for_the_most_tokens_does_for_fewer(d, E, k):
    sizes = {}
    for T in [*range(1200), *range(1200, 9000, 7), *range(9000, 37000, 61)]:
        for gating in (0, 1, 2):
            sizes.setdefault(gating, []).append(moe.route_backward_workspace_size(moe.MoEConfig.of(T, d, 64, E, k, gating)))
        sizes.setdefault("dispatch", []).append(moe.dispatch_workspace_size(moe.DispatchConfig.of(T, d, k, E)))
    for of, s in sizes.items():
        assert s[0] > 0 and all(a <= b for a, b in zip(s, s[1:])), of


T, W, K, E = 4, 64, 2, 2


def _py_dispatch(missing):
    a = dict(x=Tensor(T, W), topk_idx=Tensor(T, K, dtype=I32), topk_w=Tensor(T, K, dtype=F32), counts=Tensor(E, dtype=I32), offsets=Tensor(E + 1, dtype=I32),
             row_of=Tensor(T, K, dtype=I32), src_of=Tensor(T * K, dtype=I32), rows=Tensor(T * K, W), workspace=Tensor(1 << 20, dtype=torch.uint8))
    moe.moe_dispatch(D(T, W, K, E), **{**a, missing: None})


def _py_dispatch_backward(missing):
    a = dict(drows=Tensor(T * K, W), row_of=Tensor(T, K, dtype=I32), topk_w=None, dx=Tensor(T, W), x=Tensor(T, W), d_topk_w=Tensor(T, K, dtype=F32))
    moe.moe_dispatch_backward(D(T, W, K, E), **{**a, missing: None})


def _py_collect(missing):
    a = dict(rows=Tensor(T * K, W), row_of=Tensor(T, K, dtype=I32), topk_w=None, y=Tensor(T, W), p=0.5, rng=Tensor(2, dtype=torch.int64))
    moe.moe_collect(D(T, W, K, E), **{**a, missing: None})


def _py_collect_backward(missing):
    a = dict(dy=Tensor(T, W), rows=Tensor(T * K, W), row_of=Tensor(T, K, dtype=I32), topk_w=None, drows=Tensor(T * K, W), d_topk_w=Tensor(T, K, dtype=F32), p=0.5,
             rng=Tensor(2, dtype=torch.int64))
    moe.moe_collect_backward(D(T, W, K, E), **{**a, missing: None})


def _py_dropout(missing):
    moe.moe_dropout(**{**dict(x=Tensor(T, W), y=Tensor(T, W), p=0.5, rng=Tensor(2, dtype=torch.int64)), missing: None})


def _py_route_backward(missing):
    a = dict(x=Tensor(T, W), W_r=Tensor(E, W), bias=None, topk_idx=Tensor(T, K, dtype=I32), topk_w=Tensor(T, K, dtype=F32), d_topk_w=Tensor(T, K, dtype=F32), dx=None,
             dW_r=None, dbias=None, workspace=Tensor(1 << 20, dtype=torch.uint8))
    moe.moe_route_backward(moe.MoEConfig.of(T, W, 64, E, K), **{**a, missing: None})


@pytest.mark.parametrize("call,names", [
    (_py_dispatch, "x topk_idx counts offsets row_of src_of rows workspace"), (_py_dispatch_backward, "drows row_of dx x"), (_py_collect, "rows row_of y rng"),
    (_py_collect_backward, "dy rows row_of drows rng"), (_py_dropout, "x y rng"), (_py_route_backward, "x W_r topk_idx topk_w d_topk_w workspace")],
    ids=lambda v: v.__name__ if callable(v) else "")
def test_a_missing_argument_is_named(call, names):
    for name in names.split():
        with pytest.raises(ValueError, match=rf"^{name} is required"):
            call(name)


def test_sizes_and_types_are_checked():
    t = lambda *s, d=BF16: torch.zeros(s, dtype=d)  # noqa: E731
    with pytest.raises(ValueError, match="GPU"):
        moe.moe_dropout(t(4, 64), t(4, 64), 0.0, None)
    with pytest.raises(ValueError, match="rng"):
        moe.moe_collect(D(T, W, K, E), Tensor(T * K, W), Tensor(T, K, dtype=I32), None, Tensor(T, W), p=0.1, rng=Tensor(1, dtype=torch.int64))
    with pytest.raises(ValueError, match="row_of"):
        moe.moe_collect(D(T, W, K, E), Tensor(T * K, W), Tensor(T * K, dtype=I32), None, Tensor(T, W))
    with pytest.raises(ValueError, match="residual"):
        moe.moe_dropout(Tensor(T, W), Tensor(T, W), 0.5, Tensor(2, dtype=torch.int64), residual=Tensor(T, W + 8))
    with pytest.raises(ValueError, match="dW_r"):
        moe.moe_route_backward(moe.MoEConfig.of(T, W, 64, E, K), Tensor(T, W), Tensor(E, W), None, Tensor(T, K, dtype=I32), Tensor(T, K, dtype=F32), Tensor(T, K, dtype=F32),
                               None, Tensor(E, W, dtype=torch.float16), None, Tensor(1 << 20, dtype=torch.uint8))


def test_no_scratch_memory():
    blob = open(moe.library_path(), "rb").read()
    key = b"\\xbb.private_segment_fixed_size".decode("unicode_escape").encode("latin-1")
    scratch = {}
    for m in re.finditer(rb"\xa5\.name(?:\xd9.|\xda..|[\xa0-\xbf])(_Z\w+?)" + re.escape(key) + rb"([\x00-\x7f]|\xcc.|\xcd..)", blob, re.S):
        n = m[2]
        scratch[m[1].decode()] = n[0] if len(n) == 1 else int.from_bytes(n[1:], "big")
    mine = {k: v for k, v in scratch.items() if re.search(r"dispatch_kernel|gather_kernel|scatter_kernel|dropout_kernel|count_chunks|sum_chunks|route_(logits|dz|dx|dw|join)", k)}
    assert len(mine) >= 20 and not any(mine.values()), {k: v for k, v in mine.items() if v} or sorted(mine)


KERNELS = ("count_chunks_kernel", "sum_chunks_kernel", "tables_kernel", "dispatch_kernel", "gather_kernel", "scatter_kernel", "narrow_gather_kernel", "narrow_scatter_kernel", "dropout_kernel",
           "route_logits_kernel", "route_dz_kernel", "route_products_kernel", "route_join_kernel", "route_bias_kernel")


def _kernels_scratch():
    """Mangled name and scratch bytes of every kernel in the library, from the notes that the compiler wrote beside its code."""
    blob = open(moe.library_path(), "rb").read()
    number = {0xCC: 1, 0xCD: 2, 0xCE: 4}
    for m in re.finditer(rb"\xa5\.name(?:\xd9.|\xda..|[\xa0-\xbf])(_Z\w+?)\xbb\.private_segment_fixed_size(.....)", blob, re.S):
        n = m[2]
        yield m[1].decode(), n[0] if n[0] < 0x80 else int.from_bytes(n[1:1 + number[n[0]]], "big")


def test_no_kernel_of_these_operators_has_scratch_memory():
    """All of them, by their names: each is in the library, and none of its instances spills."""
    scratch = list(_kernels_scratch())
    for name in KERNELS:
        mine = {k: v for k, v in scratch if f"{len(name)}{name}" in k}      # the length in front: a whole name
        assert mine, name
        assert not any(mine.values()), {k: v for k, v in mine.items() if v}
