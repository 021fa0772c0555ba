"""Host-side checks of the training and adapter entry points: sizes, refusals, and the wait states of their loads into LDS.  No GPU is involved."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

import paper_2605_23911_amd as moe
from paper_2605_23911_amd import build
from test_lds_dma_hazards import hazards

P = 4096            # an address that no call below may touch: each has to fail on the host


@pytest.fixture(scope="module")
def L():
    return moe.lib()


def _train(L, c, size=1 << 40, **bad):
    a = dict(x=P, off=P, wg=P, wu=P, wd=P, g=P, u=P, h=P, y=P, ws=P)
    a.update(bad)
    return L.moe_grouped_ffn_train(C.byref(c) if c else None, a["x"], a["off"], a["wg"], a["wu"], a["wd"], a["g"], a["u"], a["h"], a["y"], a["ws"], size, None)


def _back(L, c, flags=0, size=1 << 40, **bad):
    a = dict(x=P, off=P, wg=P, wu=P, wd=P, g=P, u=P, dy=P, dx=P, dwg=P, dwu=P, dwd=P, ws=P)
    a.update(bad)
    return L.moe_grouped_ffn_backward(C.byref(c) if c else None, a["x"], a["off"], a["wg"], a["wu"], a["wd"], a["g"], a["u"], a["dy"], a["dx"], a["dwg"],
                                      a["dwu"], a["dwd"], flags, a["ws"], size, None)


def test_train_and_backward_refuse(L):
    c = moe.MoEConfig.of(64, 256, 512, 8, 2)
    assert _train(L, None) == -1 and _back(L, None) == -1
    for n in ("x", "off", "wg", "wu", "wd", "g", "u", "ws"):
        assert _train(L, c, **{n: None}) == -1, n
        assert _back(L, c, **{n: None}) == -1, n
    assert _train(L, c, h=None) == -1 and _train(L, c, y=None) == -1 and _back(L, c, dy=None) == -1
    for n in ("x", "wg", "wu", "wd", "g", "u"):
        assert _train(L, c, **{n: P + 8}) == -3, n
        assert _back(L, c, **{n: P + 8}) == -3, n
    for n in ("dy", "dx", "dwg", "dwu", "dwd"):
        assert _back(L, c, **{n: P + 2}) == -3, n
    assert _back(L, c, size=8) == -4 and _back(L, c, size=3 * 128 * 512 * 2 - 1) == -4
    assert _back(L, c, ws=P + 16) == -3
    assert _train(L, c, size=8) == -4
    assert _back(L, c, flags=4) == -2 and _back(L, c, flags=-1) == -2
    assert moe.ffn_backward_workspace_size(c) >= 3 * 128 * 512 * 2
    assert moe.ffn_backward_workspace_size(moe.MoEConfig.of(8192, 4096, 512, 1, 1)) == 3 * 8192 * 512 * 2
    for bad, status in ((moe.MoEConfig.of(-1, 256, 512, 8, 2), -2), (moe.MoEConfig.of(4, 250, 512, 8, 2), -5), (moe.MoEConfig.of(4, 256, 512, 257, 2), -5),
                        (moe.MoEConfig.of(1, (1 << 20) + 64, 512, 8, 2), -5), (moe.MoEConfig.of(1, 64, (1 << 20) + 64, 8, 2), -5),
                        (moe.MoEConfig.of(1, 1 << 19, 1 << 19, 8, 2), -5), (moe.MoEConfig.of(1 << 20, 4096, 64, 8, 2), -5)):
        assert _train(L, bad) == status and _back(L, bad) == status and moe.ffn_backward_workspace_size(bad) == 0
    # no rows: the rows' tensors may be missing, a forward pass has nothing to do
    z = moe.MoEConfig.of(0, 256, 512, 8, 2)
    assert _train(L, z, x=None, g=None, u=None, h=None, y=None) == 0
    assert _back(L, z, x=None, g=None, u=None, dy=None, dx=None, dwg=None, dwu=None, dwd=None) == 0


def test_combine_backward_refuses(L):
    c = moe.MoEConfig.of(64, 256, 512, 8, 2)

    def call(cfg=c, **bad):
        a = dict(dy=P, p=P, row=P, w=P, dp=P, dw=P)
        a.update(bad)
        return L.moe_combine_backward(C.byref(cfg), a["dy"], a["p"], a["row"], a["w"], a["dp"], a["dw"], None)

    for n in ("dy", "p", "row", "w", "dp", "dw"):
        assert call(**{n: None}) == -1, n
    for n in ("dy", "p", "dp"):
        assert call(**{n: P + 4}) == -3, n
    assert call(moe.MoEConfig.of(64, 256, 512, 8, 9)) == -2
    assert call(moe.MoEConfig.of(0, 256, 512, 8, 2), dy=None, p=None, row=None, w=None, dp=None, dw=None) == 0


def test_adapter_refuses(L):
    ok = moe.AdapterConfig.of(48, 512, 256, 4, 16)

    def linear(cfg=ok, size=1 << 40, **bad):
        a = dict(x=P, W=P, A=P, B=P, s=P, of=P, base=P, y=P, ws=P)
        a.update(bad)
        return L.moe_adapter_linear(C.byref(cfg) if cfg else None, a["x"], a["W"], a["A"], a["B"], a["s"], a["of"], a["base"], a["y"], a["ws"], size, None)

    def gated(cfg=ok, size=1 << 40, **bad):
        a = dict(x=P, W=P, V=P, A=P, C=P, B=P, D=P, s=P, of=P, h=P, ws=P)
        a.update(bad)
        return L.moe_adapter_gated_up(C.byref(cfg) if cfg else None, a["x"], a["W"], a["V"], a["A"], a["C"], a["B"], a["D"], a["s"], a["of"], a["h"], a["ws"], size, None)

    assert linear(None) == -1 and gated(None) == -1
    for n in ("x", "A", "B", "of", "y", "ws"):
        assert linear(**{n: None}) == -1, n
    for n in ("x", "W", "V", "A", "C", "B", "D", "of", "h", "ws"):
        assert gated(**{n: None}) == -1, n
    for n in ("x", "W", "A", "B", "base", "y", "ws"):
        assert linear(**{n: P + 8}) == -3, n
    for n in ("x", "W", "V", "A", "C", "B", "D", "h", "ws"):
        assert gated(**{n: P + 8}) == -3, n
    assert linear(size=16) == -4 and gated(size=16) == -4
    A = moe.AdapterConfig.of
    for bad, status in ((A(-1, 512, 256, 4, 16), -2), (A(4, 0, 256, 4, 16), -2), (A(4, 512, 0, 4, 16), -2), (A(4, 512, 256, 0, 16), -2), (A(4, 512, 256, 4, 0), -2),
                        (A(4, 500, 256, 4, 16), -5), (A(4, 512, 250, 4, 16), -5), (A(4, 512, 256, 4, 12), -5), (A(4, 512, 256, 4, 136), -5),
                        (A(4, 512, 256, 65537, 16), -5), (A(4, (1 << 20) + 64, 256, 4, 16), -5), (A(1 << 22, 512, 256, 4, 16), -5)):
        assert linear(bad) == status and gated(bad) == status and moe.adapter_workspace_size(bad) == 0, (bad.T, bad.N, bad.K, bad.adapters, bad.rank)
    assert linear(A(0, 512, 256, 4, 16), x=None, of=None, y=None) == 0 and gated(A(0, 512, 256, 4, 16), x=None, of=None, h=None) == 0


@pytest.mark.parametrize("T", [1, 17, 64, 65, 128, 129, 1000, 4096])
def test_adapter_workspace_holds_v_and_the_partial_sums(L, T):
    """Room for v of both projections at least, and no more than eight pieces of everything."""
    for N, K, r in ((64, 64, 8), (4096, 14336, 16), (14336, 4096, 128)):
        n = moe.adapter_workspace_size(moe.AdapterConfig.of(T, N, K, 64, r))
        assert 2 * T * r * 4 <= n <= 8 * 2 * T * (r + N) * 4 + 1024


def test_the_binding_checks_sizes_types_and_places():
    b, f = torch.bfloat16, torch.float32
    c = moe.MoEConfig.of(4, 64, 128, 2, 1)
    t = lambda s, d=b: torch.zeros(s, dtype=d)  # noqa: E731
    good = [t((4, 64)), t(3, torch.int32), t((2, 128, 64)), t((2, 128, 64)), t((2, 64, 128)), t((4, 128)), t((4, 128)), t((4, 128)), t((4, 64)), t(4096, torch.uint8)]
    with pytest.raises(ValueError, match="GPU"):
        moe.moe_grouped_ffn_train(c, *good)
    for i, wrong in ((0, t((4, 65))), (0, t((4, 64), f)), (0, None), (1, t(2, torch.int32))):
        args = list(good)
        args[i] = wrong
        with pytest.raises(ValueError, match="x_perm" if i == 0 else "GPU"):        # arguments are looked at in order
            moe.moe_grouped_ffn_train(c, *args)
    a = moe.AdapterConfig.of(4, 64, 64, 2, 8)
    with pytest.raises(ValueError):
        moe.moe_adapter_linear(a, t((4, 64)), t((64, 64)), t((2, 8, 64)), t((2, 64, 8)), None, t(4, torch.int64), t((4, 64)), t(4096, torch.uint8))
    with pytest.raises(ValueError):
        moe.moe_combine_backward(c, t((4, 64)), t((4, 64)), t((4, 1), torch.int32), t((4, 1)), t((4, 64)), t((4, 1), f))


def test_no_hazard_in_loads_from_a_descriptor(tmp_path):
    """As tests/test_lds_dma_hazards.py, for the load whose descriptor the compiler may have put together in vector registers."""
    src = tmp_path / "probe.hip"
    src.write_text("""
#include "lds_dma.hpp"
extern __shared__ char lds[];
__global__ void probe(const moe::i32x4* descs, uint32_t* out) {
    const moe::i32x4 d = descs[threadIdx.x];      // differs by lane as far as the compiler can tell
    const moe::i32x4 u = {__builtin_amdgcn_readfirstlane(d[0]), __builtin_amdgcn_readfirstlane(d[1]), __builtin_amdgcn_readfirstlane(d[2]),
                          __builtin_amdgcn_readfirstlane(d[3])};
    moe::buffer_dma(threadIdx.x * 16, u, (uint32_t)(uintptr_t)lds);
    moe::wait_vmcnt<0>();
    __syncthreads();
    out[threadIdx.x] = lds[threadIdx.x];
}
""")
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-Wall")]
    res = subprocess.run([build.hipcc(), *flags, "-I", build.CSRC, "-I", os.path.join(build.ROOT, "include"), "--offload-device-only", "-S",
                          str(src), "-o", str(tmp_path / "probe.s")], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr
    asm = (tmp_path / "probe.s").read_text()
    assert re.search(r"buffer_load_dwordx4 v\d+, s\[\d+:\d+\], 0 offen lds", asm)
    found, loads = hazards(asm.replace("buffer_load_dwordx4", "buffer_load_lds_dwordx4"))
    assert loads == 1 and not found, found
    # the checker sees the fault where the waits are taken out
    bad, _ = hazards(re.sub(r"s_nop 4\n", "", asm).replace("buffer_load_dwordx4", "buffer_load_lds_dwordx4"))
    assert bad


def test_no_scratch_in_the_tiles():
    blob = open(moe.library_path(), "rb").read()
    key = b"\\xbb.private_segment_fixed_size".decode("unicode_escape").encode("latin-1")
    scratch = {}
    for m in re.finditer(rb"\xa5\.name(?:\xd9.|\xda..|[\xa0-\xbf])(_Z\w+?)" + re.escape(key) + rb"([\x00-\x7f]|\xcc.|\xcd..)", blob, re.S):
        n = m[2]
        scratch[m[1].decode()] = n[0] if len(n) == 1 else int.from_bytes(n[1:], "big")
    mine = {k: v for k, v in scratch.items() if re.search(r"gated_keep|gated_grad|rows_grad|weights_grad|adapter_|low_rank|combine_backward", k)}
    assert len(mine) >= 30 and not any(mine.values()), {k: v for k, v in mine.items() if v} or sorted(mine)
