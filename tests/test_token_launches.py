"""The launches over tokens of collect, dispatch's gradient and collect's gradient, without a GPU: together they take every token once, whatever the width, also where
there are several.  A kernel knows the first token of its launch and the last one of the call, so a launch in front of another has to end with a whole workgroup."""
import ctypes as C

import pytest

import paper_2605_23911_amd as moe

MOST = 1 << 30          # T * k <= 2^30


def tokens_of_a_workgroup(d):
    if d <= 256:
        return 4 * (64 // (d // 8))
    return 4 if d <= 1024 else 1


@pytest.mark.parametrize("T", [1, 4095, (1 << 23) + 1, (1 << 25) + 3, (1 << 29) - 1, 1 << 29, (1 << 29) + 1, (1 << 29) + 52, MOST - 1, MOST])
def test_every_token_once(T):
    f = moe.lib().moe_test_token_launches
    f.argtypes, f.restype = [C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_int32)], C.c_int32
    out = (C.c_int32 * 512)()
    for d in [*range(8, 520, 8), 1016, 1024, 1032, 2048, 8192, 1 << 20]:
        each, upto = tokens_of_a_workgroup(d), 0
        n = f(T, d, 256, out)
        assert n >= 1
        for i in range(n):
            t0, groups = out[2 * i], out[2 * i + 1]
            assert t0 == upto and groups * 256 <= 1 << 31, (d, i)
            upto = t0 + groups * each
            assert upto <= T or (i == n - 1 and upto - T < each), (d, i)
        assert upto >= T
