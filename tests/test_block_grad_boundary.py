"""Argument checks of AdamW and of the linear layer's and the attention's gradient, on the host: nothing below touches a device."""
import ctypes

import pytest

import paper_2507_03211_amd as zo_amd
from paper_2507_03211_amd import ZO_BF16, ZO_FP16, ZO_FP32

INF, NAN = float("inf"), float("nan")
A = [(i + 1) << 20 for i in range(12)]                          # buffers that lie apart


def refused(f, *args):
    with pytest.raises(zo_amd.ZoError) as e:
        f(*args)
    assert e.value.status == zo_amd.ZO_EINVAL
    return str(e.value)


def changed(args, at, value):
    return args[:at] + [value] + args[at + 1:]


def test_adamw():
    #       0 param        1 grad         2 state        3 numel  4 n 5 dtype  6 bits 7 lr  8 b1  9 b2  10 eps 11 wd 12 step 13 norm 14 max 15 rounding 16 seed
    good = [[A[0], A[1]], [A[2], A[3]], [A[4], A[5]], [4, 300], 2, ZO_BF16, 32, 1e-3, 0.9, 0.99, 1e-8, 0.1, 1, A[6], 1.0, 0, 7]
    f = zo_amd.zo_kernel_adamw
    for at in range(3):
        assert "NULL" in refused(f, *changed(good, at, [A[0], None]))
        assert "aligned" in refused(f, *changed(good, at, [good[at][0] + 8, good[at][1]]))
        assert "address" in refused(f, *changed(good, at, [1 << 50, good[at][1]]))
    for at, value in ((3, [4, 1 << 50]), (4, -1), (5, 3), (5, -1), (6, 16), (6, 0), (7, -1.0), (7, NAN), (7, INF), (8, 1.0), (8, -0.1), (8, NAN), (9, 1.0), (9, 1 - 1e-9),
                      (9, NAN), (10, 0.0), (10, -1e-8), (10, 1e-60), (10, NAN), (10, INF), (11, -0.1), (11, NAN), (11, INF), (12, 0), (13, A[6] + 4), (14, 0.0), (14, NAN),
                      (14, -1.0), (15, 2)):
        refused(f, *changed(good, at, value))
    assert "stochastic" in refused(f, *changed(changed(good, 5, ZO_FP32), 15, 1))
    L = zo_amd.lib()
    assert L.zo_kernel_adamw(None, None, None, None, 1, ZO_BF16, 8, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1, None, 1.0, 0, 0, None) == zo_amd.ZO_EINVAL
    with pytest.raises(ValueError):
        f(*changed(good, 4, 3))
    with pytest.raises(TypeError):
        f(*changed(good, 0, (ctypes.c_uint64 * 2)(*A[:2])))


def test_adamw_tensors_lie_apart():
    good = [[A[0], A[1]], [A[2], A[3]], [A[4], A[5]], [4, 300], 2, ZO_FP16, 32, 1e-3, 0.9, 0.99, 1e-8, 0.1, 1, None, INF, 0, 7]
    f = zo_amd.zo_kernel_adamw
    for at, value in ((0, [A[0], A[0]]), (0, [A[1] + 592, A[1]]), (0, [A[2], A[1]]), (0, [A[3] + 592, A[1]]), (0, [A[4], A[1]]), (0, [A[0], A[5] + 4080]), (2, [A[4], A[4] + 2032]),
                      (2, [A[4], A[4] - 16]), (2, [A[3], A[5]]), (1, [A[0], A[3]]), (1, [A[2], A[5] + 4080])):
        assert "overlaps" in refused(f, *changed(good, at, value)), (at, value)
    assert "norm overlaps" in refused(f, *changed(good, 13, A[5] + 8))
    many = 300
    p, s = ([base + 4096 * i for i in range(many, 0, -1)] for base in (1 << 30, 1 << 40))
    assert "overlaps" in refused(f, p, p[1:] + [1 << 35], s, [32] * many, many, *good[5:])
    assert "overlaps" in refused(f, p, [1 << 35] * many, s[:-1] + [s[3] + 16], [32] * many, many, *good[5:])


def test_adamw_state_bytes():
    f = zo_amd.zo_kernel_adamw_state_bytes
    assert [f(n, 32) for n in (0, 1, 256, 257)] == [0, 2048, 2048, 4096] and [f(n, 8) for n in (0, 1, 256, 257)] == [0, 520, 520, 1040]
    assert f(10, 16) == 0 and f(1 << 44, 8) == 0 and f((1 << 44) - 1, 32) == 1 << 47
