"""Argument checks of AdamW and of the linear layer's and the attention's gradient, on the host: nothing below touches a device."""
import ctypes

import pytest
import torch

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
    # a block of an 8-bit state is 520 bytes: states side by side lie on 8
    assert "aligned" in refused(f, *changed(changed(good, 6, 8), 2, [A[4] + 4, A[5]]))
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


def test_linear_grad():
    #       0 x   1 w   2 y   3 dy  4 dx  5 dw  6 db  7 scratch 8 dtype 9 rows 10 n 11 k 12 epilogue 13 relu_x
    good = A[:8] + [ZO_BF16, 4, 64, 128, 1, False]
    f = zo_amd.zo_kernel_linear_grad
    for at in (0, 1, 2, 3, 7):
        assert "NULL" in refused(f, *changed(good, at, None))
    assert "no output" in refused(f, *(good[:4] + [None] * 3 + good[7:]))
    assert "NULL" in refused(f, None, *good[1:5], None, None, *good[7:13], True)       # relu_x asks for x, dw or not
    assert "no bias" in refused(f, *changed(good, 12, 3))
    for at, value in ((8, 3), (8, -1), (9, 0), (9, -4), (10, 0), (11, 0), (10, 60), (11, 60), (12, 4), (12, -1), (0, A[0] + 2), (1, A[1] + 8), (2, A[2] + 2), (3, A[3] + 2),
                      (4, A[4] + 8), (5, A[5] + 2), (6, A[6] + 2), (7, A[7] + 128), (9, 1 << 21), (10, 1 << 23), (11, 1 << 23)):
        refused(f, *changed(good, at, value))
        if 8 <= at <= 12:
            assert zo_amd.zo_kernel_linear_grad_scratch_bytes(*changed(good, at, value)[8:13]) == 0
    assert zo_amd.zo_kernel_linear_grad_scratch_bytes(ZO_FP32, 1, 1, 1, 0) > 0


@pytest.mark.parametrize("dtype,wide,narrow,weight", [(ZO_FP32, 8, 8, 4), (ZO_BF16, 4, 2, 2), (ZO_FP16, 4, 2, 2)])
def test_linear_gradients_lie_apart(dtype, wide, narrow, weight):
    f = zo_amd.zo_kernel_linear_grad
    x, w, y, dy, dx, dw, db = A[:7]
    for epilogue, each in ((0, narrow), (1, narrow), (2, wide)):
        args = A[:8] + [dtype, 4, 64, 128, epilogue, True]
        moves = [(4, x, "dx overlaps x"), (4, x + 512 * narrow - 16, "dx overlaps x"), (4, w, "dx overlaps w"), (4, dy, "dx overlaps dy"), (4, dy + 256 * each - 16, "dx overlaps dy"),
                 (5, dx + 16, "dx overlaps dw"), (5, w, "dw overlaps w"), (5, x - 64 * 128 * weight + 16, "dw overlaps x"), (6, dw + 64 * 128 * weight - 16, "dw overlaps db"),
                 (6, dy, "db overlaps dy"), (6, w, "db overlaps w")]
        if epilogue == 1:
            moves += [(4, y, "dx overlaps y"), (5, y + 16, "dw overlaps y")]
        for at, address, words in moves:
            assert words in refused(f, *changed(args, at, address))


def test_linear_grad_plan():
    p = zo_amd.zo_kernel_linear_grad_plan(8192, 20480, 5120, 0)
    assert p["dx"] == p["dw"] == (256, 256) and p["copy_columns"] == 0
    assert zo_amd.zo_kernel_linear_grad_plan(8192, 768, 768, 2)["dw_shares"] > 1
    assert zo_amd.zo_kernel_linear_grad_plan(20, 8192, 2048, 1)["dx_shares"] > 1
    for n, epilogue in ((72, 0), (64, 1), (64, 2)):
        assert zo_amd.zo_kernel_linear_grad_plan(100, n, 64, epilogue)["copy_columns"] >= n
    for bad in ((0, 64, 64, 0), (4, 60, 64, 0), (4, 64, 60, 0), (4, 64, 64, 4)):
        refused(zo_amd.zo_kernel_linear_grad_plan, *bad)
    assert zo_amd.lib().zo_kernel_linear_grad_plan(4, 64, 64, 0, None) == zo_amd.ZO_EINVAL


@pytest.mark.parametrize("rows,n,k", [(1048, 5000, 4096), (2050, 13000, 1288), (700, 13000, 3000), (8192, 20480, 5120), (300, 512, 512), (8192, 768, 768)])
def test_linear_grad_plan_of_the_rows_behind_whole_rounds(rows, n, k):
    """dw's launch is whole rounds of tiles over the compute units (256 where there is no device) or has all rows."""
    p = zo_amd.zo_kernel_linear_grad_plan(rows, n, k, 0)
    tall, wide = p["dw"]
    assert 0 < p["dw_rows"] <= n and (p["dw_rows"] == n or p["dw_rows"] % tall == 0)
    assert (p["dw_rows"] < n) == (n >= 5000)
    if p["dw_rows"] < n:
        assert p["dw_shares"] == 1
    if p["dw_rows"] < n and not torch.cuda.is_available():
        tiles = (p["dw_rows"] // tall) * ((k + wide - 1) // wide)
        assert -tiles % 256 < (k + wide - 1) // wide         # (what a last row of tiles would pass the rounds by)


@pytest.mark.parametrize("dtype,rows,n,k", [(ZO_BF16, 64, 1 << 22, 1 << 18), (ZO_FP16, 1 << 20, 64, 1 << 22), (ZO_FP32, 1 << 20, 64, 1 << 17)])
def test_linear_grad_of_more_tiles_than_a_launch_holds(dtype, rows, n, k):
    assert zo_amd.zo_kernel_linear_grad_scratch_bytes(dtype, rows, n, k, 0) == 0
    assert "tiles" in refused(zo_amd.zo_kernel_linear_grad, *[(i + 1) << 44 for i in range(8)], dtype, rows, n, k, 0, False)
    assert zo_amd.zo_kernel_linear_grad_scratch_bytes(dtype, rows >> 4, max(n >> 4, 8), k >> 4, 0) > 0


def test_attention_grad():
    #       0 qkv 1 out 2 dout 3 dqkv 4 scratch 5 dtype 6 n_seq 7 seq 8 heads 9 d_head
    good = A[:5] + [ZO_BF16, 2, 5, 3, 64]
    f = zo_amd.zo_kernel_attention_grad
    for at in range(5):
        assert "NULL" in refused(f, *changed(good, at, None))
    for at, value in ((5, 3), (5, -1), (6, 0), (7, 0), (8, 0), (9, 0), (9, 136), (9, 60), (7, 1 << 21), (8, 1 << 15), (0, A[0] + 2), (1, A[1] + 8), (2, A[2] + 2), (3, A[3] + 8),
                      (4, A[4] + 128), (6, 1 << 29)):
        refused(f, *changed(good, at, value))
        if at >= 5:
            assert zo_amd.zo_kernel_attention_grad_scratch_bytes(*changed(good, at, value)[5:]) == 0
    assert zo_amd.zo_kernel_attention_grad_scratch_bytes(ZO_FP32, 1, 1, 1, 1) > 0
    for shape in ((ZO_BF16, 1 << 22, 64, 8, 64), (ZO_FP32, 1 << 25, 1, 1, 16), (ZO_FP16, 1 << 21, 16, 2, 40), (ZO_FP32, 1, 1, 1 << 16, 4)):
        assert zo_amd.zo_kernel_attention_grad_scratch_bytes(*shape) == 0
        assert "launch" in refused(f, *[(i + 1) << 44 for i in range(5)], *shape)
    assert zo_amd.zo_kernel_attention_grad_scratch_bytes(ZO_BF16, (1 << 21) - 8, 64, 8, 64) > 0


@pytest.mark.parametrize("dtype,each", [(ZO_FP32, 8), (ZO_BF16, 2), (ZO_FP16, 2)])
def test_attention_gradients_lie_apart(dtype, each):
    qkv, out, dout, dqkv = A[:4]
    n = 10 * 3 * 64 * each
    for address, words in ((qkv, "qkv"), (qkv + 3 * n - 16, "qkv"), (qkv - 3 * n + 16, "qkv"), (out, "out"), (out + n - 16, "out"), (dout - 3 * n + 16, "dout"), (dout + n - 16, "dout")):
        assert "dqkv overlaps " + words in refused(zo_amd.zo_kernel_attention_grad, qkv, out, dout, address, A[4], dtype, 2, 5, 3, 64)
