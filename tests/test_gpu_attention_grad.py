"""The causal attention's backward pass against 64 bits.

Tolerance, 16-bit types on the matrix cores (u = half a step of the type, all other arithmetic fp32): P and dS enter their products rounded by u each;
D is summed from `out`, each element off by u of itself: by at most u |dO| |O| (absolute sums), which P multiplies.  With |dP| and |D| bounded by
the same absolute sums, a gradient's element is off by at most
    dV: u P^T |dO|,   dQ, dK: (2 u |dS| + u P D_abs) against |K|, |Q| / sqrt(d_head)
plus fp32's share (the exponent's error is some 2^-24 of the scaled scores and logsumexp, relative to P) and the result's own rounding.
"""
import math

import pytest
import torch

import paper_2507_03211_amd as zo_amd
import zo_inputs as zi
from gpu_util import DEV, act_dtype
from grad_util import Out, generator, half, least, normal

pytestmark = pytest.mark.gpu
DTYPES = [zi.FP32, zi.BF16, zi.FP16]
MATRIX = [64, 80, 96, 112, 128]


class Attention:
    def __init__(self, dtype, n_seq, seq, heads, d_head, seed=0, size=1.0, dsize=0.1, qkv=None):
        g = generator(seed + 1000 * n_seq + seq + 31 * heads + d_head)
        self.dtype, self.n_seq, self.seq, self.heads, self.d_head = dtype, n_seq, seq, heads, d_head
        self.shape = (dtype, n_seq, seq, heads, d_head)
        a, rows, d = act_dtype(dtype), n_seq * seq, heads * d_head
        self.qkv = normal((rows, 3 * d), a, g, size) if qkv is None else qkv
        self.dout = normal((rows, d), a, g, dsize)
        self.out = torch.empty((rows, d), dtype=a, device=DEV)
        zo_amd.zo_kernel_attention(self.qkv, self.out, *self.shape)
        self.dqkv = Out((rows, 3 * d), a)
        self.scratch = torch.full((zo_amd.zo_kernel_attention_grad_scratch_bytes(*self.shape),), 0xFF, dtype=torch.uint8, device=DEV)

    def run(self, stream=None):
        zo_amd.zo_kernel_attention_grad(self.qkv, self.out, self.dout, self.dqkv.t, self.scratch, *self.shape, stream)

    def split(self, t, i):
        """[parts, heads, positions, channels] of sequence i, in fp64."""
        return t.view(self.n_seq, self.seq, -1, self.heads, self.d_head)[i].double().permute(1, 2, 0, 3).contiguous()

    def want(self, i):
        """Gradients of sequence i and how far off they may be."""
        q, k, v = self.split(self.qkv, i)
        (do,), (o,) = self.split(self.dout, i), self.split(self.out, i)
        scale = 1.0 / math.sqrt(self.d_head)
        score = (q @ k.transpose(1, 2)) * scale
        seen = torch.ones(self.seq, self.seq, dtype=torch.bool, device=DEV).tril()
        score = score.masked_fill(~seen, -math.inf)
        p = torch.softmax(score, 2)
        dp = do @ v.transpose(1, 2)
        delta = (p * dp).sum(2, keepdim=True)
        ds = p * (dp - delta)
        grads = [scale * ds @ k, scale * ds.transpose(1, 2) @ q, p.transpose(1, 2) @ do]
        matrix = self.dtype != zi.FP32 and self.d_head in MATRIX
        u16 = half(act_dtype(self.dtype)) if self.dtype != zi.FP32 else 0.0
        u = 2.0**-53 if self.dtype == zi.FP32 else 2.0**-24
        terms = self.seq + self.d_head + 64
        # P: relative to itself, by its exponent: sums of d_head products, a multiplication by the scale, logsumexp
        size = (q.abs() @ k.abs().transpose(1, 2)) * scale
        top = torch.where(seen, size, 0.0).amax(2, keepdim=True)
        p_rel = u * ((self.d_head + 8) * (size + top) + terms)
        dp_abs, d_abs = do.abs() @ v.abs().transpose(1, 2), (do.abs() * o.abs()).sum(2, keepdim=True)
        # D: `out` is off by its rounding and by what the forward call's own P was (rounded too, on the matrix cores)
        d_off = (3 * u16 + terms * u) * (do.abs() * (p @ v.abs())).sum(2, keepdim=True) + terms * u * d_abs
        if matrix and self.seq <= 128:                          # (D is summed from P dP there, P in fp32)
            d_off = (p * (p_rel + terms * u) * dp_abs).sum(2, keepdim=True)
        ds_off = ds.abs() * (p_rel + (2 * u16 if matrix else 0.0)) + p * (d_off + terms * u * (dp_abs + d_abs))
        p_off = p * (p_rel + (u16 if matrix else 0.0))
        if matrix and self.dtype == zi.FP16:
            # numbers below the type's normal ones: 2^-25 of a P scaled by 2^14, of a dS scaled to 2^12 / (A B) and more
            p_off = p_off + torch.where(seen, 2.0**-39, 0.0)
            bound = do.norm(dim=2).amax(1) * v.norm(dim=2).amax(1)
            ds_off = ds_off + torch.where(seen, (2.0**-25 * 2.0**-7) * bound[:, None, None], 0.0)
        offs = [scale * ds_off @ k.abs(), scale * ds_off.transpose(1, 2) @ q.abs(), p_off.transpose(1, 2) @ do.abs()]
        sums = [scale * ds.abs() @ k.abs(), scale * ds.abs().transpose(1, 2) @ q.abs(), p.transpose(1, 2) @ do.abs()]
        return grads, [a + terms * u * b for a, b in zip(offs, sums)]

    def check(self, sequences=None):
        t = act_dtype(self.dtype)
        for i in range(self.n_seq) if sequences is None else sequences:
            grads, offs = self.want(i)
            for got, want, off in zip(self.split(self.dqkv.t, i), grads, offs):
                assert bool(((got - want).abs() <= off * (1 + 2.0**-6) + (half(t) if self.dtype != zi.FP32 else 0.0) * (want.abs() + off) + least(t) + 1e-300).all())


def ran(a):
    a.run()
    torch.cuda.synchronize()
    assert a.dqkv.whole()
    return a


@pytest.mark.parametrize("dtype", [zi.BF16, zi.FP16])
@pytest.mark.parametrize("d_head", MATRIX)
@pytest.mark.parametrize("seq", [1, 2, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129, 200, 257, 511])
def test_lengths(dtype, d_head, seq):
    ran(Attention(dtype, 3, seq, 3, d_head)).check()


@pytest.mark.parametrize("dtype", [zi.BF16, zi.FP16])
@pytest.mark.parametrize("d_head", MATRIX)
@pytest.mark.parametrize("seq", [1, 33, 64, 65, 128, 129])
def test_short_sequences_do_without_out(dtype, d_head, seq):
    a = ran(Attention(dtype, 3, seq, 2, d_head, size=2.0))
    a.check()
    want = a.dqkv.t.clone()
    a.out.fill_(math.nan)
    ran(a)
    assert torch.equal(a.dqkv.t, want) if seq <= 128 else bool(torch.isnan(a.dqkv.t).any())


@pytest.mark.parametrize("dtype,d_head", [(zi.FP32, c) for c in (1, 4, 16, 33, 64, 128)] + [(t, c) for t in (zi.BF16, zi.FP16) for c in (8, 40, 72, 120)])
@pytest.mark.parametrize("seq", [1, 2, 32, 127, 129, 300])
def test_other_heads(dtype, d_head, seq):
    ran(Attention(dtype, 2, seq, 3, d_head)).check()


@pytest.mark.parametrize("dtype", [zi.BF16, zi.FP16])
@pytest.mark.parametrize("n_seq,seq,heads,d_head", [(1, 2048, 2, 128), (1, 4096, 1, 64), (9, 70, 5, 96), (1, 1500, 3, 80), (17, 130, 1, 112), (40, 3, 16, 64)])
def test_sizes(dtype, n_seq, seq, heads, d_head):
    ran(Attention(dtype, n_seq, seq, heads, d_head)).check(None if n_seq < 10 else (0, n_seq - 1))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d_head", [64, 128])
@pytest.mark.parametrize("size", [0.05, 3.0])
def test_flat_and_peaked(dtype, d_head, size):
    """Scores near zero everywhere, and of deviation 9 sqrt(d_head) / sqrt(d_head) x sqrt(d_head): one key has nearly all."""
    ran(Attention(dtype, 2, 200, 2, d_head, size=size)).check()


@pytest.mark.parametrize("d_head", MATRIX)
@pytest.mark.parametrize("dsize", [2.0**-20, 2.0**-10, 1.0, 2.0**9])
@pytest.mark.parametrize("seq", [65, 1024])
def test_fp16_gradients_of_any_size(d_head, dsize, seq):
    """dS follows dO's size; the results are 16-bit numbers again."""
    a = Attention(zi.FP16, 1, seq, 2, d_head, dsize=dsize)
    ran(a).check()
    assert bool(torch.isfinite(a.dqkv.t).all())


@pytest.mark.parametrize("dtype", [zi.BF16, zi.FP16])
@pytest.mark.parametrize("d_head", [64, 80, 128])
def test_scores_that_rise_along_the_keys(dtype, d_head):
    """The reference maximum is raised again and again; and never, with scores that fall."""
    for sign in (1, -1):
        g = generator(3)
        seq, heads = 300, 2
        qkv = normal((seq, 3, heads, d_head), torch.float64, g, 0.3)
        ramp = torch.linspace(0, 6, seq, device=DEV, dtype=torch.float64)[:, None]
        qkv[:, 0, :, 0], qkv[:, 1, :, 0] = 4.0, sign * ramp * math.sqrt(d_head) / 4
        ran(Attention(dtype, 1, seq, heads, d_head, qkv=qkv.reshape(seq, -1).to(act_dtype(dtype)))).check()


@pytest.mark.parametrize("dtype,d_head", [(zi.BF16, 64), (zi.FP16, 128), (zi.BF16, 80), (zi.FP32, 16), (zi.BF16, 40)])
def test_not_finite_stays_in_its_sequence_and_head(dtype, d_head):
    a, b = (Attention(dtype, 3, 100, 3, d_head) for _ in range(2))
    d = 3 * d_head
    for t, col in ((b.qkv, d_head + 3), (b.qkv, d + d_head + 1), (b.qkv, 2 * d + d_head), (b.dout, d_head + 7), (b.out, d_head + 2)):
        keep = t[150, col].clone()
        for bad in (math.nan, math.inf):
            t[150, col] = bad
            ran(a)
            ran(b)
            x, y = (s.dqkv.t.view(3, 100, 3, 3, d_head) for s in (a, b))
            for i in range(3):
                for h in range(3):
                    if (i, h) != (1, 1):
                        assert torch.equal(x[i, :, :, h], y[i, :, :, h])
        t[150, col] = keep


@pytest.mark.parametrize("dtype,d_head", [(zi.BF16, 64), (zi.FP16, 96), (zi.BF16, 128), (zi.FP16, 40), (zi.FP32, 20)])
def test_neighbours_in_memory_stay_out(dtype, d_head):
    for n_seq, seq in ((1, 33), (2, 130), (3, 64)):
        a = Attention(dtype, n_seq, seq, 2, d_head)
        for name in ("qkv", "out", "dout"):
            t = getattr(a, name)
            around = torch.full((t.numel() + (1 << 17),), float("nan"), dtype=t.dtype, device=DEV)
            inside = around[1 << 16:(1 << 16) + t.numel()].view(t.shape)
            inside.copy_(t)
            setattr(a, name, inside)
        ran(a).check()


def test_gradient_by_differences():
    """fp32 (fp64 activations): the forward call's own central difference along a direction.  Its error is a sixth of the third derivative, found from a
    step twice as long (the two differ by three times the finer one's error, 4/3 with the next order's), beside fp64's rounding."""
    a = ran(Attention(zi.FP32, 2, 24, 2, 12))
    g = generator(8)
    direction = normal(tuple(a.qkv.shape), torch.float64, g)

    def difference(eps):
        losses = []
        for s in (eps, -eps):
            out = torch.empty_like(a.out)
            zo_amd.zo_kernel_attention(a.qkv + s * direction, out, *a.shape)
            losses.append(out)
        return float((a.dout * (losses[0] - losses[1])).sum()) / (2 * eps)
    coarse, fine = difference(2.0**-10), difference(2.0**-11)
    got = float((direction * a.dqkv.t).sum())
    assert abs(got - fine) <= abs(coarse - fine) + 2.0**-40 * float((direction * a.dqkv.t).abs().sum())


@pytest.mark.parametrize("dtype,d_head", [(zi.BF16, 64), (zi.FP16, 80), (zi.BF16, 128), (zi.FP32, 16)])
def test_captured_and_replayed(dtype, d_head):
    a = Attention(dtype, 2, 150, 3, d_head)
    a.run(torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run(torch.cuda.current_stream())
    g = generator(3)
    for i in range(4):
        a.qkv.copy_(normal(tuple(a.qkv.shape), torch.float64, g))
        a.dout.copy_(normal(tuple(a.dout.shape), torch.float64, g, 0.1 * (i + 1)))
        zo_amd.zo_kernel_attention(a.qkv, a.out, *a.shape, torch.cuda.current_stream())
        a.dqkv.t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = a.dqkv.t.clone()
        a.scratch.fill_(85 * i)
        a.run(torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(got, a.dqkv.t)


def test_two_streams():
    many = [Attention(zi.BF16, 2, 700, 4, 64) for _ in range(3)]
    ran(many[0])
    streams = [torch.cuda.Stream(device=DEV) for _ in many[1:]]
    torch.cuda.synchronize()
    for a, s in zip(many[1:], streams):
        a.run(s)
    torch.cuda.synchronize()
    assert all(torch.equal(a.dqkv.t, many[0].dqkv.t) for a in many[1:])


def test_more_bytes_than_32_bits_count():
    """qkv of 2^32 bytes and more; the last sequence has the gradient that it has alone."""
    n_seq, seq, heads, d_head = 2100, 70, 80, 128
    g = generator(2)
    last = normal((seq, 3 * heads * d_head), torch.bfloat16, g)
    qkv = torch.zeros((n_seq * seq, 3 * heads * d_head), dtype=torch.bfloat16, device=DEV)
    qkv[-seq:] = last
    assert qkv.numel() * 2 > 1 << 32
    a = Attention(zi.BF16, n_seq, seq, heads, d_head, qkv=qkv)
    alone = Attention(zi.BF16, 1, seq, heads, d_head, qkv=last)
    alone.dout.copy_(a.dout[-seq:])
    ran(a)
    ran(alone)
    assert torch.equal(a.dqkv.t[-seq:], alone.dqkv.t)
