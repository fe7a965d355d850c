"""Global norm and clipping against 64 bits.

The norm: squares are exact in fp64 or rounded by 2^-53, and any order of n additions of magnitudes keeps within n 2^-53 of the sum;
with at most 2^11 in a chain here, 2^-41 covers norm and coefficient.  A clipped element is c g, c rounded to fp32 (16-bit
types; the product too: 2^-23 together), then rounded to its type.
"""
import ctypes

import pytest
import torch

import paper_2507_03211_amd as zo_amd
import zo_inputs as zi
from gpu_util import DEV
from grad_util import Out, generator, half, least, normal, param_dtype

pytestmark = pytest.mark.gpu
DTYPES = [zi.FP32, zi.BF16, zi.FP16]
LISTS = [[1], [7, 1], [16384], [16383, 16385, 3], [5, 0, 100001, 8, 64], [300000] + [768] * 300, [40] * 125, [1 << 22, 9], [17] * 700,
         [17] * 40, [17] * 41]


def scratch():
    return torch.full((zo_amd.zo_kernel_grad_clip_scratch_bytes(),), 0xFF, dtype=torch.uint8, device=DEV)


def clip(dtype, src, max_norm, in_place=False, ws=None):
    outs = [Out(tuple(t.shape), t.dtype) for t in src]
    if in_place:
        for o, t in zip(outs, src):
            o.t.copy_(t)
        src = [o.t for o in outs]
    norm = Out((2,), torch.float64)
    zo_amd.zo_kernel_grad_clip(src, [o.t for o in outs], [t.numel() for t in src], len(src), dtype, max_norm, norm.t, scratch() if ws is None else ws)
    torch.cuda.synchronize()
    assert all(o.whole() for o in outs) and norm.whole()
    return [o.t for o in outs], norm.t.tolist()


def tensors(dtype, numels, std=0.01, seed=0):
    g = generator(seed + sum(numels))
    return [normal((n,), param_dtype(dtype), g, std) for n in numels]


def check(dtype, src, max_norm, got):
    outs, (norm, coef) = got
    want = float(torch.sqrt(sum((t.double().square().sum() for t in src), torch.zeros((), dtype=torch.float64, device=DEV))))
    assert abs(norm - want) <= 2.0**-41 * want
    c = max_norm / want if want > max_norm else 1.0
    assert abs(coef - c) <= 2.0**-41 * c
    for t, o in zip(src, outs):
        if c == 1.0:
            assert torch.equal(t, o)
            continue
        w = c * t.double()
        rounding = half(t.dtype) * (1 + 2.0**-20) + (2.0**-22 if dtype != zi.FP32 else 2.0**-40)
        tiny = 2.0**-150 if dtype == zi.FP32 else least(t.dtype)
        assert ((o.double() - w).abs() <= rounding * w.abs() + tiny).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("numels", LISTS, ids=lambda v: "%dx%d" % (len(v), max(v)))
@pytest.mark.parametrize("in_place", [False, True])
def test_clips(dtype, numels, in_place):
    src = tensors(dtype, numels)
    norm = float(torch.sqrt(sum(t.double().square().sum() for t in src)))
    for max_norm in (norm / 3, 1e-4, 2 * norm + 1, float("inf")):
        max_norm = float(torch.tensor(max_norm, dtype=torch.float32))        # as the call gets it
        check(dtype, src, max_norm, clip(dtype, src, max_norm, in_place))


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_tensors(dtype):
    assert clip(dtype, [], 1.0)[1] == [0.0, 1.0]
    outs, norm = clip(dtype, tensors(dtype, [0, 0]), 1.0)
    assert norm == [0.0, 1.0]
    zeros = [torch.zeros(100, dtype=param_dtype(dtype), device=DEV)]
    outs, norm = clip(dtype, zeros, 1.0)
    assert norm == [0.0, 1.0] and (outs[0] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("in_place", [False, True])
def test_a_norm_that_is_not_finite_clears_all(dtype, bad, in_place):
    src = tensors(dtype, [1000, 3, 40000])
    src[2][39999] = bad
    for max_norm in (0.5, float("inf")):
        outs, (norm, coef) = clip(dtype, src, max_norm, in_place)
        assert not norm - norm == 0.0 and coef == 0.0
        assert all((o == 0).all() for o in outs)


def test_squares_beyond_fp32():
    for v in (1e30, 1e-30, 3e38):
        src = [torch.full((5000,), v, device=DEV), torch.full((33,), -v, device=DEV)]
        check(zi.FP32, src, 1.0, clip(zi.FP32, src, 1.0))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("count", [9, 300])
@pytest.mark.parametrize("shift", [0, 1])
def test_neighbours_in_one_buffer(dtype, count, shift):
    """Tensors that adjoin, listed from the last one to the first: clipped in place, or into the next one's place, where nothing else lies."""
    n = 64
    base = normal((2 * count * n,), param_dtype(dtype), generator(5), 0.01)
    buf = base.clone()
    parts = [buf[2 * n * i:2 * n * i + n] for i in range(count)][::-1]
    to = [buf[2 * n * i + n * shift:2 * n * i + n * (1 + shift)] for i in range(count)][::-1]
    norm = torch.empty(2, dtype=torch.float64, device=DEV)
    zo_amd.zo_kernel_grad_clip(parts, to, [n] * count, count, dtype, 0.01, norm, scratch())
    src = [base[2 * n * i:2 * n * i + n] for i in range(count)][::-1]
    check(dtype, src, float(torch.tensor(0.01, dtype=torch.float32)), (to, norm.tolist()))
    other = base.view(count, 2, n)[:, 1 - shift]
    assert torch.equal(buf.view(count, 2, n)[:, 1 - shift], other)


@pytest.mark.parametrize("dtype", DTYPES)
def test_same_bits_every_time_and_tables_kept(dtype):
    src = tensors(dtype, [70000, 5, 123456, 768, 31])
    first = clip(dtype, src, 0.5)
    ws = scratch()
    src_t = (ctypes.c_void_p * 5)(*[t.data_ptr() for t in src])
    n = (ctypes.c_uint64 * 5)(*[t.numel() for t in src])
    for s in [torch.cuda.Stream(device=DEV) for _ in range(2)]:
        outs = [torch.empty_like(t) for t in src]
        dst_t = (ctypes.c_void_p * 5)(*[t.data_ptr() for t in outs])
        norm = torch.empty(2, dtype=torch.float64, device=DEV)
        torch.cuda.synchronize()
        zo_amd.zo_kernel_grad_clip(src_t, dst_t, n, 5, dtype, 0.5, norm, ws, s)
        torch.cuda.synchronize()
        assert norm.tolist() == first[1] and all(torch.equal(a, b) for a, b in zip(outs, first[0]))


def test_more_elements_than_32_bits_count():
    n, max_norm = (1 << 32) + 9, 0.5
    src = torch.empty(n, dtype=torch.bfloat16, device=DEV).normal_(0.0, 0.01, generator=generator(31))
    out = Out((n,), torch.bfloat16)
    norm = torch.empty(2, dtype=torch.float64, device=DEV)
    zo_amd.zo_kernel_grad_clip([src], [out.t], [n], 1, zi.BF16, max_norm, norm, scratch())
    torch.cuda.synchronize()
    assert out.whole()
    want = float(sum(t.double().square().sum() for t in src.split(1 << 28)))**0.5
    assert abs(float(norm[0]) - want) <= 2.0**-40 * want             # 2^12 in a chain here, and the oracle's own sums
    for t, o in zip(src.split(1 << 28), out.t.split(1 << 28)):
        w = max_norm / want * t.double()
        assert ((o.double() - w).abs() <= (half(t.dtype) * (1 + 2.0**-20) + 2.0**-22) * w.abs() + least(t.dtype)).all()


def test_bytes_of_a_model():
    """The tensors of a 3-layer model side by side in one buffer, clipped into another: nothing between them is touched."""
    d, f = 96, 384
    numels = [5000 * d, 64 * d] + 3 * [d, d, d * d, d, d * d, d, d * d, d, d * d, d, d, d, f * d, f, d * f, d] + [d, d + 3]
    firsts, total = [], 0
    for n in numels:
        firsts.append(total)
        total += (n + 7) // 8 * 8 + 8                              # a gap behind each
    flat = normal((total,), torch.bfloat16, generator(5), 0.02)
    out = torch.full_like(flat, 7.0)
    src = [flat[a:a + n] for a, n in zip(firsts, numels)]
    dst = [out[a:a + n] for a, n in zip(firsts, numels)]
    norm = torch.empty(2, dtype=torch.float64, device=DEV)
    zo_amd.zo_kernel_grad_clip(src, dst, numels, len(numels), zi.BF16, 0.25, norm, scratch())
    torch.cuda.synchronize()
    check(zi.BF16, src, 0.25, (dst, norm.tolist()))
    hit = torch.zeros(total, dtype=torch.bool, device=DEV)
    for a, n in zip(firsts, numels):
        hit[a:a + n] = True
    assert (out[~hit] == 7.0).all()


@pytest.mark.parametrize("dtype,size,max_norm", [
    (zi.BF16, 1e38, 1.0), (zi.BF16, 1e38, 1e-3), (zi.BF16, 1e38, 1e-6), (zi.BF16, 1e38, 2.0**-126), (zi.BF16, 1e30, 2.0**-100), (zi.BF16, 1.0, 2.0**-120),
    (zi.FP16, 1e4, 2.0**-10), (zi.FP16, 1e4, 2.0**-20), (zi.FP32, 1e38, 1e-6), (zi.FP32, 1e38, 2.0**-126)])
@pytest.mark.parametrize("in_place", [False, True])
def test_coefficients_below_fp32s_range(dtype, size, max_norm, in_place):
    """Norms up to 2^250 times the limit: the coefficient itself is beyond fp32 (bf16, fp32), what it makes of a gradient is not."""
    g = generator(12)
    src = [(normal((n,), torch.float64, g).clamp(-3, 3) * size).to(param_dtype(dtype)) for n in (40000, 77, 1)]
    max_norm = float(torch.tensor(max_norm, dtype=torch.float32))
    check(dtype, src, max_norm, clip(dtype, src, max_norm, in_place))
