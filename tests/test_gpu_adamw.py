"""AdamW over many tensors: bit for bit against the same fp32 operations one by one on the host, and against the formula in 64 bits.

The tolerance against 64 bits (32-bit moments): m is two products and a sum, each off by 2^-24 of itself: 2^-23 of |b1 m| + |c1 g|, and the scalars
and the clipped gradient by as much again; v likewise with one product more.  The root halves v's relative error; the step (a product, a root, a
product, a sum, a division) is off by at most 8 x 2^-24 of itself beside m's error.  The parameter's own fp32 sum and its rounding to its type come on top.
"""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2507_03211_amd as zo_amd
import zo_inputs as zi
from oracle import zo_oracle as zo
from gpu_util import DEV
from grad_util import Out, generator, half, least, normal, param_dtype

pytestmark = pytest.mark.gpu
DTYPES = [zi.FP32, zi.BF16, zi.FP16]
LISTS = [[1], [256], [257, 3], [4096, 4097], [5, 0, 100001, 8, 64], [0, 0, 300, 0], [1000] + [40] * 39, [1000] + [40] * 40, [33] * 141, [700] + [17] * 299]
LR, B1, B2, EPS, WD = 1e-2, 0.9, 0.95, 1e-8, 0.1
F = np.float32


class Tensors:
    """Parameters, gradients and moments of a list, the moments from earlier steps (or zeros); guarded ends."""

    def __init__(self, dtype, bits, numels, seed=0, fresh=False, std=0.01):
        g = generator(seed + sum(numels) + bits)
        self.dtype, self.bits, self.numels = dtype, bits, numels
        self.param = [Out((n,), param_dtype(dtype)) for n in numels]
        self.grad = [normal((n,), param_dtype(dtype), g, std) for n in numels]
        self.state = [Out((zo_amd.zo_kernel_adamw_state_bytes(n, bits),), torch.uint8, 0) for n in numels]
        for p in self.param:
            p.t.copy_(normal(tuple(p.t.shape), param_dtype(dtype), g, 0.02))
        if not fresh:
            for n, s in zip(numels, self.state):
                m, v = (torch.zeros((n + 255) // 256 * 256) for _ in range(2))
                m[:n] = normal((n,), torch.float32, g, std).cpu()
                v[:n] = normal((n,), torch.float32, g, std).cpu().square()
                s.t.copy_(torch.from_numpy(pack(m.numpy(), v.numpy(), bits)))

    def host(self):
        return [p.t.cpu().clone() for p in self.param], [s.t.cpu().numpy().copy() for s in self.state]

    def step(self, t, **more):
        zo_amd.zo_kernel_adamw([p.t for p in self.param], self.grad, [s.t for s in self.state], self.numels, len(self.numels), self.dtype, self.bits, LR,
                               B1, B2, EPS, WD, t, **more)
        torch.cuda.synchronize()
        assert all(o.whole() for o in self.param + self.state)


def hold8(x, low):
    x = x.reshape(-1, 256)
    with np.errstate(all="ignore"):
        top = np.abs(x).max(1, keepdims=True)
        scale = (top * F(1.0 / 448.0)).astype(F)
        scale[scale < F(2.0**-126)] = 0
        inverse = np.where(scale > 0, F(1) / scale, F(0)).astype(F)
        y = (x * inverse).astype(F)
    if low:
        y = np.where((x > 0) & (scale > 0), np.maximum(y, F(2.0**-9)), y)
    bad = ~np.isfinite(x).all(1, keepdims=True)
    scale, y = np.where(bad, F(np.nan), scale), np.where(bad, F(0), y)
    return torch.from_numpy(y.astype(F)).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), scale


def pack(m, v, bits):
    if bits == 32:
        return np.concatenate([m.reshape(-1, 256), v.reshape(-1, 256)], 1).astype(F).view(np.uint8).reshape(-1)
    (mq, ms), (vq, vs) = hold8(m, False), hold8(np.sqrt(v), True)
    return np.concatenate([mq, vq, np.concatenate([ms, vs], 1).view(np.uint8)], 1).reshape(-1)


def unpack(state, bits):
    if bits == 32:
        s = state.view(F).reshape(-1, 512)
        return s[:, :256].reshape(-1).copy(), s[:, 256:].reshape(-1).copy()
    s = state.reshape(-1, 520)
    scale = s[:, 512:].copy().view(F)
    m, r = (torch.from_numpy(s[:, a:a + 256].copy()).view(torch.float8_e4m3fn).float().numpy() * scale[:, i:i + 1] for i, a in ((0, 0), (1, 256)))
    return m.reshape(-1), (r * r).reshape(-1)


def words(seed, tensor, n):
    """Word i % 4 of Philox4x32-10 at (i / 4, tensor, 3), for i < n."""
    j = np.arange((n + 3) // 4, dtype=np.uint64)
    low, s32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [j & low, j >> s32, np.full_like(j, tensor), np.full_like(j, 3)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> s32) ^ c[1] ^ np.uint64(k0), b & low, (a >> s32) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, 1).reshape(-1)[:n].astype(np.uint32)


def scalars(t):
    return dict(b1=F(B1), c1=F(1 - B1), b2=F(B2), c2=F(1 - B2), decay=F(LR * WD), rate=F(LR / -math.expm1(t * math.log(B1))),
                root=F(1 / math.sqrt(-math.expm1(t * math.log(B2)))), eps=F(EPS))


def expect(ts, param, state, t, coef=F(1), stochastic=False, seed=0):
    """One step by the stated fp32 operations; new parameters and states."""
    c, out = scalars(t), ([], [])
    for i, (n, p, g, s) in enumerate(zip(ts.numels, param, ts.grad, state)):
        m, v = unpack(s, ts.bits)
        m, v, p, g = m[:n], v[:n], p.float().numpy(), g.float().cpu().numpy()
        with np.errstate(all="ignore"):
            g = (F(coef) * g).astype(F)
            m = c["b1"] * m + c["c1"] * g
            v = c["b2"] * v + (c["c2"] * g) * g
            p = p - (c["decay"] * p + (c["rate"] * m) / (c["root"] * np.sqrt(v) + c["eps"]))
        assert p.dtype == m.dtype == v.dtype == F
        if stochastic:
            p = torch.from_numpy(zo.sr_round(p, words(seed, i, n), ts.dtype).view(np.int16).copy()).view(param_dtype(ts.dtype))
        else:
            p = torch.from_numpy(p).to(param_dtype(ts.dtype))
        out[0].append(p)
        pad = np.zeros((n + 255) // 256 * 256 - n, F)
        out[1].append(pack(np.concatenate([m, pad]), np.concatenate([v, pad]), ts.bits))
    return out


def same(ts, want):
    got = ts.host()
    bits = lambda x: x.contiguous().view(torch.uint8) if x.numel() else x  # noqa: E731
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip(got[0], want[0]))
    assert all(np.array_equal(a, b) for a, b in zip(got[1], want[1]))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("numels", LISTS, ids=lambda v: "%dx%d" % (len(v), max(v)))
def test_bits(dtype, bits, numels):
    ts = Tensors(dtype, bits, numels)
    for t in (1, 7, 100000):
        before = ts.host()
        ts.step(t)
        same(ts, expect(ts, *before, t))


@pytest.mark.parametrize("dtype", [zi.BF16, zi.FP16])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("numels", [[1], [5, 0, 100001, 8], [33] * 150], ids=lambda v: "%dx%d" % (len(v), max(v)))
def test_stochastic_bits(dtype, bits, numels):
    ts = Tensors(dtype, bits, numels, 1)
    for t, seed in ((1, 5), (2, 2**64 - 3)):
        before = ts.host()
        ts.step(t, rounding=zo_amd.ZO_ROUND_STOCHASTIC, seed=seed)
        same(ts, expect(ts, *before, t, stochastic=True, seed=seed))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits", [32, 8])
def test_clipped_on_the_way(dtype, bits):
    """The coefficient of the norm alone, and what the clipping call's own norm gives; none where max_norm is infinite or the norm below it."""
    ts = Tensors(dtype, bits, [5000, 3, 777], 2)
    norm = torch.empty(2, dtype=torch.float64, device=DEV)
    scratch = torch.empty(zo_amd.zo_kernel_grad_clip_scratch_bytes(), dtype=torch.uint8, device=DEV)
    zo_amd.zo_kernel_grad_clip(ts.grad, ts.grad, ts.numels, 3, dtype, float("inf"), norm, scratch)
    n = float(norm[0])
    for t, max_norm in ((3, n / 3), (4, 1e-3), (5, 2 * n), (6, float("inf"))):
        max_norm = float(F(max_norm))
        before = ts.host()
        ts.step(t, norm=norm, max_norm=max_norm)
        same(ts, expect(ts, *before, t, coef=F(max_norm / n) if n > max_norm else F(1)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_norm_that_is_not_finite_writes_nothing(dtype, bits, bad):
    ts = Tensors(dtype, bits, [5000, 3], 3)
    before = ts.host()
    for max_norm in (1.0, math.inf):
        ts.step(2, norm=torch.tensor([bad], dtype=torch.float64, device=DEV), max_norm=max_norm)
    same(ts, before)


@pytest.mark.parametrize("dtype", DTYPES)
def test_against_64_bits(dtype):
    """Steps from zero moments, each from the state before it."""
    ts = Tensors(dtype, 32, [100003], 4, fresh=True)
    u = 2.0**-24
    for t in range(1, 6):
        param, state = ts.host()
        p, g = param[0].double().numpy(), ts.grad[0].double().cpu().numpy()
        m, v = (x[:100003].astype(np.float64) for x in unpack(state[0], 32))
        m64, v64 = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
        # the hand-written step of the definition: bias-corrected moments, decay on the weight itself
        step = LR * (m64 / (1 - B1**t)) / (np.sqrt(v64 / (1 - B2**t)) + EPS)
        want = p - LR * WD * p - step
        ts.step(t)
        got_m, got_v = (x[:100003] for x in unpack(ts.state[0].t.cpu().numpy(), 32))
        m_off = 4 * u * (np.abs(B1 * m) + np.abs((1 - B1) * g))
        assert (np.abs(got_m - m64) <= m_off + 2.0**-149).all()
        assert (np.abs(got_v - v64) <= 5 * u * v64 + 2.0**-148).all()
        got = ts.param[0].t.double().cpu().numpy()
        fp32 = m_off * np.abs(step / np.where(m64 == 0, 1, m64)) + 12 * u * np.abs(step) + 3 * u * np.abs(LR * WD * p) + 2 * u * (np.abs(want) + np.abs(p - want))
        rounding = half(param_dtype(dtype)) if dtype != zi.FP32 else 0.0
        assert (np.abs(got - want) <= fp32 + rounding * (np.abs(want) + fp32) + least(param_dtype(dtype))).all()
        ts.grad[0].copy_(normal((100003,), param_dtype(dtype), generator(t), 0.01))


def test_first_step_is_the_gradients_sign():
    """From zero moments m / (1 - b1) = g and v / (1 - b2) = g^2: every weight moves by lr, against its gradient (8-bit moments hold each only
    afterwards, so they say the same)."""
    for bits in (8, 32):
        ts = Tensors(zi.FP32, bits, [5000], 5, fresh=True)
        ts.param[0].t.zero_()
        ts.step(1)
        want = -LR * torch.sign(ts.grad[0].double())
        assert ((ts.param[0].t.double() - want).abs() <= LR * (2.0**-20 + EPS / ts.grad[0].double().abs().clamp(min=EPS))).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_not_finite_in_8_bits_stays_in_its_block(bad):
    ts = Tensors(zi.BF16, 8, [1000, 300], 6)
    ts.grad[0][300] = bad
    before = ts.host()
    ts.step(3)
    want = expect(ts, *before, 3)
    got = ts.host()
    nan = torch.isnan(got[0][0])
    assert nan[300] and int(nan.sum()) == 1
    assert all(torch.equal(a[~torch.isnan(b)], b[~torch.isnan(b)]) for a, b in zip(got[0], want[0]))
    scale = got[1][0].reshape(-1, 520)[:, 512:].copy().view(F)
    assert np.isnan(scale[1]).all() and np.isfinite(scale[[0, 2, 3]]).all()
    other = [0, 2, 3]
    assert np.array_equal(got[1][0].reshape(-1, 520)[other], want[1][0].reshape(-1, 520)[other]) and np.array_equal(got[1][1], want[1][1])


def test_small_beside_a_blocks_largest():
    """A block whose gradients span 2^40: roots that e4m3 cannot reach are held as its least number, never as zero, and the next step does not
    divide by eps alone.  Magnitudes below 2^-117 are held as zeros."""
    ts = Tensors(zi.FP32, 8, [256, 256], 7, fresh=True)
    ts.grad[0].copy_(torch.exp2(-torch.arange(256, device=DEV) * (40.0 / 255)))
    ts.grad[1].fill_(2.0**-140)
    ts.param[0].t.zero_()
    before = ts.host()
    ts.step(1)
    same(ts, expect(ts, *before, 1))
    rows = [s.t.cpu().numpy().reshape(-1, 520) for s in ts.state]
    assert (rows[0][0, 256:512] > 0).all() and not rows[1].any()
    ts.grad[0].zero_()
    old = ts.param[0].t.clone()
    ts.step(2)
    assert float((ts.param[0].t - old).abs().max()) <= 2 * LR


def test_what_lies_behind_a_tensor_in_its_last_block_does_not_count():
    ts = Tensors(zi.BF16, 8, [300], 8)
    row = ts.state[0].t.view(-1, 520)[1]
    row[44:256] = 0x7E                                              # 448, behind the end
    row[256 + 44:512] = 0x7E
    before = ts.host()
    ts.step(4)
    same(ts, expect(ts, *before, 4))
    assert not bool(row[44:256].any()) and not bool(row[256 + 44:512].any())


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_and_replayed(bits):
    """A replay is a call with the same scalars: replays, with other gradients in the same buffers, give what eager calls do."""
    a, b = (Tensors(zi.BF16, bits, [5000, 3, 70000] + [20] * 60, 9) for _ in range(2))
    keep = a.host()
    norm = torch.tensor([3.0, 1.0], dtype=torch.float64, device=DEV)
    a.step(5, norm=norm, max_norm=1.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        zo_amd.zo_kernel_adamw([p.t for p in a.param], a.grad, [s.t for s in a.state], a.numels, len(a.numels), zi.BF16, bits, LR, B1, B2, EPS, WD, 5, norm, 1.0,
                               stream=torch.cuda.current_stream())
    for p, s, kp, ks in zip(a.param, a.state, *keep):
        p.t.copy_(kp)
        s.t.copy_(torch.from_numpy(ks))
    for i in range(4):
        for x, y in zip(a.grad, b.grad):
            x.copy_(normal(tuple(x.shape), torch.bfloat16, generator(i), 0.01))
            y.copy_(x)
        norm[0] = 0.5 + i
        graph.replay()
        torch.cuda.synchronize()
        b.step(5, norm=norm, max_norm=1.0)
        same(a, b.host())


def test_two_streams_and_tables_kept():
    ts = [Tensors(zi.FP16, 8, [70000, 5, 123456], 10) for _ in range(3)]
    ts[0].step(2)
    tables = []
    for x in ts[1:]:
        tables.append([(ctypes.c_void_p * 3)(*[t.data_ptr() for t in lst]) for lst in ([p.t for p in x.param], x.grad, [s.t for s in x.state])])
    n = (ctypes.c_uint64 * 3)(*ts[0].numels)
    streams = [torch.cuda.Stream(device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    for s, t in zip(streams, tables):
        zo_amd.zo_kernel_adamw(*t, n, 3, zi.FP16, 8, LR, B1, B2, EPS, WD, 2, stream=s)
    torch.cuda.synchronize()
    for x in ts[1:]:
        same(x, ts[0].host())


def test_more_elements_than_32_bits_count():
    """A tensor's end beyond 2^32 elements (and 2^33 bytes) takes the step that it takes alone."""
    n = (1 << 32) + 777
    tail = 256 * 5 + n % 256
    param = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    grad = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    state = torch.zeros(zo_amd.zo_kernel_adamw_state_bytes(n, 8), dtype=torch.uint8, device=DEV)
    g = generator(11)
    param[-tail:] = normal((tail,), torch.bfloat16, g, 0.02)
    grad[-tail:] = normal((tail,), torch.bfloat16, g, 0.01)
    alone = Tensors(zi.BF16, 8, [tail], 11, fresh=True)
    alone.param[0].t.copy_(param[-tail:])
    alone.grad[0].copy_(grad[-tail:])
    alone.step(1)
    zo_amd.zo_kernel_adamw([param], [grad], [state], [n], 1, zi.BF16, 8, LR, B1, B2, EPS, WD, 1)
    torch.cuda.synchronize()
    assert torch.equal(param[-tail:], alone.param[0].t) and torch.equal(state[-alone.state[0].t.numel():], alone.state[0].t)
    assert not bool(param[:1 << 20].any()) and not bool(state[:1 << 20].any())


def test_8_bit_states_side_by_side():
    """Blocks of 520 bytes, tensor behind tensor: states on odd multiples of 8."""
    ts = Tensors(zi.BF16, 8, [256, 700, 5, 300], 12)
    flat = torch.cat([s.t for s in ts.state])
    sizes = [s.t.numel() for s in ts.state]
    views = list(flat.split(sizes))
    assert any(v.data_ptr() % 16 for v in views)
    before = ts.host()
    zo_amd.zo_kernel_adamw([p.t for p in ts.param], ts.grad, views, ts.numels, 4, zi.BF16, 8, LR, B1, B2, EPS, WD, 6)
    torch.cuda.synchronize()
    for s, v in zip(ts.state, views):
        s.t.copy_(v)
    same(ts, expect(ts, *before, 6))


def test_nothing_to_do():
    zo_amd.zo_kernel_adamw([], [], [], [], 0, zi.BF16, 32, LR, B1, B2, EPS, WD, 1)
    zo_amd.zo_kernel_adamw([None], [None], [None], [0], 1, zi.BF16, 8, LR, B1, B2, EPS, WD, 1)


@pytest.mark.parametrize("first", [2.0**-40, 2.0**-89, 2.0**116, 2.0**-126])
def test_roots_of_every_mantissa(first):
    """v through two powers of two, in each of its fp32 numbers: halved exactly, its root, and a division that shows the root's last bit."""
    n = 1 << 24
    v = torch.arange(n, dtype=torch.int32, device=DEV).add_(int(np.float32(2 * first).view(np.int32))).view(torch.float32)
    state = torch.stack([torch.full((n // 256, 256), 1.0 + 2.0**-20, device=DEV), v.view(-1, 256)], 1).contiguous()
    param, grad = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    zo_amd.zo_kernel_adamw([param], [grad], [state], [n], 1, zi.FP32, 32, 2.0**-30, 0.5, 0.5, 2.0**-100, 0.0, 1 << 20)
    half_v = v.cpu().numpy() * F(0.5)
    step = F(2.0**-30) * F(0.5 * (1.0 + 2.0**-20)) / (np.sqrt(half_v) + F(2.0**-100))
    assert step.dtype == F
    assert np.array_equal(param.cpu().numpy().view(np.uint32), (F(0) - step).view(np.uint32))
    assert np.array_equal(state[:, 1].reshape(-1).cpu().numpy(), half_v)


@pytest.mark.parametrize("before", [39, 40, 139, 140, 141, 300])
def test_a_table_of_empty_tensors_in_front(before):
    """Nothing but empty tensors in a launch's table: no launch, and the numbering goes on."""
    ts = Tensors(zi.BF16, 32, [0] * before + [5, 700] + [0] * 150)
    at = ts.host()
    ts.step(3, rounding=zo_amd.ZO_ROUND_STOCHASTIC, seed=9)
    same(ts, expect(ts, *at, 3, stochastic=True, seed=9))
