"""The gradient calls' argument checks, on the host: nothing below touches a device."""
import ctypes

import pytest

import paper_2507_03211_amd as zo_amd
from paper_2507_03211_amd import ZO_BF16, ZO_FP16, ZO_FP32

P = 4096            # an address that is aligned and never followed
INF, NAN = float("inf"), float("nan")


def refused(f, *args):
    with pytest.raises(zo_amd.ZoError) as e:
        f(*args)
    assert e.value.status == zo_amd.ZO_EINVAL
    return str(e.value)


def test_layernorm():
    good = [P, P, P, P, P, P, ZO_BF16, 4, 64, 1e-5]
    for i in range(6):
        assert "NULL" in refused(zo_amd.zo_kernel_layernorm, *(good[:i] + [None] + good[i + 1:]))
    for at, value in ((6, 3), (6, -1), (7, 0), (7, -5), (8, 0), (9, 0.0), (9, -1.0), (9, NAN), (7, 1 << 24), (8, 1 << 23)):
        refused(zo_amd.zo_kernel_layernorm, *(good[:at] + [value] + good[at + 1:]))


def test_layernorm_grad():
    #       dy resid gain mean rstd dresid dgain dbias scratch dtype rows d accumulate
    good = [P, P, P, P, P, P, P, P, P, ZO_FP16, 4, 64, False]
    f = zo_amd.zo_kernel_layernorm_grad
    for i in (0, 1, 2, 3, 4, 8):
        assert "NULL" in refused(f, *(good[:i] + [None] + good[i + 1:]))
    assert "go together" in refused(f, *(good[:6] + [None] + good[7:]))
    assert "go together" in refused(f, *(good[:7] + [None] + good[8:]))
    assert "no output" in refused(f, P, P, P, P, P, None, None, None, P, ZO_FP16, 4, 64, False)
    assert "aligned" in refused(f, *(good[:8] + [P + 16] + good[9:]))
    for at, value in ((9, 5), (10, 0), (11, 0), (11, -64), (10, 1 << 24), (11, 1 << 23)):
        refused(f, *(good[:at] + [value] + good[at + 1:]))
    assert zo_amd.zo_kernel_layernorm_grad_scratch_bytes(ZO_BF16, 1, 1) > 0
    for bad in ((3, 4, 64), (-1, 4, 64), (ZO_BF16, 0, 64), (ZO_BF16, 4, 0)):
        assert zo_amd.zo_kernel_layernorm_grad_scratch_bytes(*bad) == 0


def test_lmhead_grad():
    #       x e target row_loss dx de scratch dtype rows d vocab scale
    good = [P, P, P, P, P, P, P, ZO_BF16, 4, 64, 512, 1.0]
    f = zo_amd.zo_kernel_lmhead_grad
    for i in range(7):
        assert "NULL" in refused(f, *(good[:i] + [None] + good[i + 1:]))
    for at, value in ((7, 3), (8, 0), (9, 0), (10, 1), (9, 60), (10, 500), (11, INF), (11, NAN), (0, P + 2), (1, P + 8), (4, P + 2), (5, P + 8),
                      (6, P + 128)):
        refused(f, *(good[:at] + [value] + good[at + 1:]))
    assert zo_amd.zo_kernel_lmhead_grad_scratch_bytes(ZO_FP32, 1, 1, 2) > 0
    for bad in ((3, 4, 64, 512), (ZO_BF16, 0, 64, 512), (ZO_BF16, 4, 0, 512), (ZO_BF16, 4, 64, 1)):
        assert zo_amd.zo_kernel_lmhead_grad_scratch_bytes(*bad) == 0
    for at, value in ((8, 1 << 21), (9, 1 << 23), (10, 1 << 23)):                  # beyond the sizes the header names
        refused(f, *(good[:at] + [value] + good[at + 1:]))
        assert zo_amd.zo_kernel_lmhead_grad_scratch_bytes(ZO_BF16, *(good[8:at] + [value] + good[at + 1:11])) == 0


def test_lmhead_grad_plan():
    p = zo_amd.zo_kernel_lmhead_grad_plan(8192, 5120, 50272)
    assert p == dict(logits=(256, 256), de=(256, 256), dx=(256, 256), shares=2, pieces=1, de_words=49152, de_rest=(192, 128))
    assert zo_amd.zo_kernel_lmhead_grad_plan(65536, 5120, 50272)["pieces"] > 1
    assert zo_amd.zo_kernel_lmhead_grad_plan(20, 768, 50272)["shares"] > 1
    # a workspace for more rows grows by the rows' own buffers once G fills its room
    sizes = [zo_amd.zo_kernel_lmhead_grad_scratch_bytes(ZO_BF16, r, 768, 50272) for r in (1024, 8192, 32768, 65536)]
    assert sizes == sorted(sizes) and sizes[3] < (1 << 30) + 65536 * (768 * 16 + 8192)
    for bad in ((0, 64, 512), (4, 60, 512), (4, 64, 500), (4, 64, 1)):
        refused(zo_amd.zo_kernel_lmhead_grad_plan, *bad)
    assert zo_amd.lib().zo_kernel_lmhead_grad_plan(4, 64, 512, None) == zo_amd.ZO_EINVAL


def test_grad_clip():
    #       src dst numel n dtype max_norm norm scratch
    good = [[P, P + 64], [P, P + 64], [4, 4], 2, ZO_BF16, 1.0, P, P]
    f = zo_amd.zo_kernel_grad_clip
    for at, value in ((0, [P, None]), (1, [None, P]), (0, [P + 8, P]), (1, [P, P + 2]), (2, [4, 1 << 60]), (3, -1), (4, 3), (5, 0.0), (5, -1.0),
                      (5, NAN), (6, None), (7, None), (6, P + 4), (7, P + 16)):
        refused(f, *(good[:at] + [value] + good[at + 1:]))
    # a tensor listed twice, one that ends in the next, a dst where another's src or its own lies, in order and not, more than a few
    for src, dst, n in (([P, P], [P, P], [4, 4]), ([P, P + 64], [P, P + 64], [33, 4]), ([P, P + 64], [P + 64, P], [4, 4]), ([P], [P + 16], [9]),
                        ([P + 144, P], [P + 512, P + 128], [8, 9]),
                        ([P + 64 * i for i in range(300, 0, -1)] + [P + 64 * 7 + 16], [P + 64 * i for i in range(300, 0, -1)] + [P + 64 * 400], [32] * 301)):
        with pytest.raises(zo_amd.ZoError, match="overlaps"):
            f(src, dst, n, len(src), ZO_BF16, 1.0, P, P)
    L = zo_amd.lib()
    for tables in ((None, None, None), (None, (ctypes.c_void_p * 1)(P), (ctypes.c_uint64 * 1)(4))):
        assert L.zo_kernel_grad_clip(*tables, 1, ZO_BF16, 1.0, P, P, None) == zo_amd.ZO_EINVAL
    with pytest.raises(ValueError):
        f([P], [P, P], [4, 4], 2, ZO_BF16, 1.0, P, P)                       # a table shorter than n_tensors
    with pytest.raises(TypeError):
        f((ctypes.c_uint64 * 1)(P), [P], [4], 1, ZO_BF16, 1.0, P, P)         # an array of another type


def overlaps(f, args, moves):
    """`moves`: (argument, address, words of the refusal)."""
    for at, address, words in moves:
        assert words in refused(f, *(args[:at] + [address] + args[at + 1:]))


A = [(i + 1) << 20 for i in range(9)]                           # buffers that lie apart


def test_layernorm_outputs_lie_apart():
    for dtype, wide, narrow, weight in ((ZO_FP32, 8, 8, 4), (ZO_BF16, 4, 2, 2), (ZO_FP16, 4, 2, 2)):
        args = A[:6] + [dtype, 4, 64, 1e-5]                     # resid gain bias y mean rstd
        resid, gain, bias, y, mean, rstd = A[:6]
        moves = [(3, resid + 256 * wide - narrow, "y overlaps resid"), (3, resid - 256 * narrow + 1, "y overlaps resid"), (3, gain, "y overlaps gain"),
                 (3, bias + 64 * weight - 2, "y overlaps bias"), (4, y + 255 * narrow, "y overlaps mean"), (5, mean, "mean overlaps rstd"), (5, mean + 3 * wide, "mean overlaps rstd"),
                 (5, resid, "rstd overlaps resid"), (4, gain, "mean overlaps gain")]
        if dtype != ZO_FP32:
            moves.append((3, resid, "y overlaps resid"))
        overlaps(zo_amd.zo_kernel_layernorm, args, moves)


def test_layernorm_gradients_lie_apart():
    for dtype, wide, narrow, weight in ((ZO_FP32, 8, 8, 4), (ZO_BF16, 4, 2, 2), (ZO_FP16, 4, 2, 2)):
        for rows in (4, 1000):
            #       dy resid gain mean rstd dresid dgain dbias scratch
            args = A[:9] + [dtype, rows, 64, False]
            dy, resid, gain, mean, rstd, dresid, dgain, dbias = A[:8]
            overlaps(zo_amd.zo_kernel_layernorm_grad, args, [
                (5, resid, "dresid overlaps resid"), (5, dy, "dresid overlaps dy"), (5, dy + 64 * rows * narrow - 1, "dresid overlaps dy"), (6, gain, "dgain overlaps gain"),
                (7, gain, "dbias overlaps gain"), (6, dbias, "dgain overlaps dbias"), (7, dgain + 64 * weight - 1, "dgain overlaps dbias"),
                (6, dy + 2, "dgain overlaps dy"), (7, mean, "dbias overlaps mean"), (6, rstd + rows * wide - 2, "dgain overlaps rstd"),
                (6, dresid + 64 * (rows - 1) * wide, "dresid overlaps dgain")])


@pytest.mark.parametrize("dtype,rows,d,vocab", [
    (ZO_BF16, 1 << 20, 64, 1 << 17), (ZO_FP16, 1 << 20, 128, 1 << 22), (ZO_BF16, 1 << 18, 8, 1 << 18), (ZO_FP16, 100, 1 << 14, 1 << 22), (ZO_BF16, 128, 1 << 15, 1 << 21),
    (ZO_FP32, 1, 1 << 12, 1 << 22), (ZO_FP32, 1 << 20, 1 << 14, 64)])
def test_lmhead_grad_of_more_tiles_than_a_launch_holds(dtype, rows, d, vocab):
    """Grids count threads by 32 bits: 2^24 workgroups of 256, refused before anything is launched.  A quarter of each such size is taken."""
    assert zo_amd.zo_kernel_lmhead_grad_scratch_bytes(dtype, rows, d, vocab) == 0
    assert "tiles" in refused(zo_amd.zo_kernel_lmhead_grad, *[(i + 1) << 44 for i in range(7)], dtype, rows, d, vocab, 1.0)
    quarter = (rows >> 2, d, vocab) if rows > 1 << 10 else (rows, d >> 2, vocab)
    if rows * vocab < 1 << 40:
        assert zo_amd.zo_kernel_lmhead_grad_scratch_bytes(dtype, *quarter) > 0
    if dtype != ZO_FP32:
        assert "tiles" in refused(zo_amd.zo_kernel_lmhead_grad_plan, rows, d, vocab)
        # with more to do for each tile the products have larger ones, which do not count
        assert zo_amd.zo_kernel_lmhead_grad_scratch_bytes(dtype, max(rows, 256), max(d, 256), vocab) > 0


def test_lmhead_gradients_lie_apart():
    for dtype, wide, narrow, weight in ((ZO_FP32, 8, 8, 4), (ZO_BF16, 4, 2, 2), (ZO_FP16, 4, 2, 2)):
        args = A[:7] + [dtype, 4, 64, 512, 1.0]                  # x e target row_loss dx de scratch
        x, e, target, row_loss, dx, de = A[:6]
        overlaps(zo_amd.zo_kernel_lmhead_grad, args, [
            (4, x, "dx overlaps x"), (4, x + 256 * narrow - 16, "dx overlaps x"), (5, e, "de overlaps e"), (5, e - 16, "de overlaps e"), (5, x - 512 * 64 * weight + 16, "de overlaps x"),
            (4, de + 16, "dx overlaps de"), (3, target, "row_loss overlaps target"), (3, dx + 256 * narrow - wide, "row_loss overlaps dx"), (4, target, "dx overlaps target")])
