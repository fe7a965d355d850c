"""The causal attention's backward pass at scores of any size.

Where a row's largest scores belong to copies of one key and all others lie far behind, P is known to the last bit whatever the scores are: one over the copies
that the row sees.  Scores of copies are the same bits, sums of the same products in the same order, so nothing of their size may show in P.

Tolerance.  Copies: P is exp of exactly zero over the sum, by way of a logarithm in base two of at most 2^10, whose last place is 2^-20, in an exponent of at most 2^4,
rounded to 2^-21; ln 2 times that, the exponential's and the quotient's last places, 2^-23 each, and `terms` roundings of the sum come to less than P_REL = 2^-19 + terms 2^-24
(fp64: 2^-48 and terms 2^-53).  Others: their scores and the copies' are off by E = (d_head + 8) 2^-24 of the largest sum of magnitudes each, so their P, e^(s - top), is at
most e^(s - top + 2 E) before and after, which vanishes beside half a step here for every gap used.  On top, as for any scores (u = half a step of the type): P and dS rounded
by u each, `out` by u where D comes from it, fp32 sums, the result's rounding.
"""
import math

import pytest
import torch

import zo_inputs as zi
from gpu_util import act_dtype
from grad_util import generator, half, least, normal
from test_gpu_attention_grad import MATRIX, Attention, ran

pytestmark = pytest.mark.gpu


def levels_of(kind, seq):
    """Copies of a key by position, as (positions, size beside the largest)."""
    if kind == "one":
        return [([0], 1.0)]
    if kind == "two":
        return [([0, seq // 3], 1.0)]
    if kind == "all":
        return [(list(range(seq)), 1.0)]
    if kind == "all below zero":
        return [(list(range(seq)), -1.0)]
    return [([0, 5], 0.25), ([seq // 3, seq // 3 + 2], 0.5), ([2 * seq // 3, seq - 1], 1.0)]           # "rising"


class Led(Attention):
    def __init__(self, dtype, seq, d_head, top, kind, heads=2, n_seq=2):
        g = generator(seq + d_head)
        a = act_dtype(dtype)
        uniform = lambda *shape: 1.0 + 0.5 * torch.rand(shape, device=g.device, dtype=torch.float64, generator=g)  # noqa: E731
        signs = torch.sign(normal((n_seq, 1, heads, d_head), torch.float64, g))
        size = math.sqrt(top / (1.5625 * math.sqrt(d_head)))                        # (1.25 twice: the mean products of the two)
        qkv = normal((n_seq, seq, 3, heads, d_head), torch.float64, g)
        qkv[:, :, 0] = size * signs * uniform(n_seq, seq, heads, d_head)
        # (others' scores: sums of d_head terms of either sign, 1 / (32 sqrt(d_head)) of the largest each deviation)
        qkv[:, :, 1] *= size / 32
        self.levels = levels_of(kind, seq)
        lead = size * signs[:, 0] * uniform(n_seq, heads, d_head)
        for places, factor in self.levels:
            qkv[:, places, 1] = factor * lead[:, None]
        super().__init__(dtype, n_seq, seq, heads, d_head, dsize=2.0**-10, qkv=qkv.reshape(n_seq * seq, -1).to(a))
        # `out` as 64 bits have it: the forward call has limits of its own
        self.out = torch.cat([(self.probabilities(i)[0] @ self.split(self.qkv, i)[2]).permute(1, 0, 2).reshape(seq, -1) for i in range(n_seq)]).to(a)

    def probabilities(self, i):
        """P of sequence i, the largest P that anything but a copy may have, and which are copies."""
        q, k, _ = self.split(self.qkv, i)
        scale = 1.0 / math.sqrt(self.d_head)
        score, size = (q @ k.transpose(1, 2)) * scale, (q.abs() @ k.abs().transpose(1, 2)) * scale
        for places, _ in self.levels:
            score[:, :, places] = score[:, :, places[:1]]
        seen = torch.ones(self.seq, self.seq, dtype=torch.bool, device=q.device).tril()
        score = score.masked_fill(~seen, -math.inf)
        top = score.amax(2, keepdim=True)
        lead = score == top
        u = 2.0**-53 if self.dtype == zi.FP32 else 2.0**-24
        e = (self.d_head + 8) * u * torch.where(seen, size, 0.0).amax(2, keepdim=True)
        return torch.softmax(score, 2), torch.where(lead | ~seen, 0.0, torch.exp(torch.minimum(score - top + 2 * e, torch.zeros_like(score)))), lead

    def want(self, i):
        q, k, v = self.split(self.qkv, i)
        (do,), (o,) = self.split(self.dout, i), self.split(self.out, i)
        scale = 1.0 / math.sqrt(self.d_head)
        p, others, lead = self.probabilities(i)
        assert float(others.max()) <= 2.0**-13          # (of the inputs: rows with one or more keys far ahead)
        dp = do @ v.transpose(1, 2)
        ds = p * (dp - (p * dp).sum(2, keepdim=True))
        grads = [scale * ds @ k, scale * ds.transpose(1, 2) @ q, p.transpose(1, 2) @ do]
        matrix = self.dtype != zi.FP32 and self.d_head in MATRIX
        u16 = half(act_dtype(self.dtype)) if self.dtype != zi.FP32 else 0.0
        u, terms = 2.0**-53 if self.dtype == zi.FP32 else 2.0**-24, self.seq + self.d_head + 64
        # (others: all the rest of their own P, and what theirs changes of the copies')
        rest = others.sum(2, keepdim=True)
        p_rel = 32 * u + terms * u + rest
        dp_abs, d_abs = do.abs() @ v.abs().transpose(1, 2), (do.abs() * o.abs()).sum(2, keepdim=True)
        p_arith = torch.where(lead, p * p_rel, 0.0) + others
        if matrix and self.seq <= 128:                  # (D from P in fp32 there)
            d_off = (p_arith * dp_abs).sum(2, keepdim=True)
        else:
            d_off = u16 * d_abs + (p_arith * dp_abs).sum(2, keepdim=True)
        ds_off = ds.abs() * ((2 * u16 if matrix else 0.0) + p_rel) + others * (dp_abs + d_abs) + p * (d_off + terms * u * (dp_abs + d_abs))
        p_off = p_arith + p * (u16 if matrix else 0.0)
        if matrix and self.dtype == zi.FP16:            # numbers below the type's normal ones
            seen = torch.ones_like(p[0], dtype=torch.bool).tril()
            p_off = p_off + torch.where(seen, 2.0**-39, 0.0)
            bound = do.norm(dim=2).amax(1) * v.norm(dim=2).amax(1)
            ds_off = ds_off + torch.where(seen, (2.0**-25 * 2.0**-7) * bound[:, None, None], 0.0)
        offs = [scale * ds_off @ k.abs(), scale * ds_off.transpose(1, 2) @ q.abs(), p_off.transpose(1, 2) @ do.abs()]
        sums = [scale * ds.abs() @ k.abs(), scale * ds.abs().transpose(1, 2) @ q.abs(), p.transpose(1, 2) @ do.abs()]
        return grads, [a + terms * u * b for a, b in zip(offs, sums)]

    def hold(self):
        ran(self)
        assert bool(torch.isfinite(self.dqkv.t).all())
        t = act_dtype(self.dtype)
        for i in range(self.n_seq):
            grads, offs = self.want(i)
            for name, got, want, off in zip(("dq", "dk", "dv"), self.split(self.dqkv.t, i), grads, offs):
                far = (got - want).abs() - (off * (1 + 2.0**-6) + (half(t) if self.dtype != zi.FP32 else 0.0) * (want.abs() + off) + least(t))
                assert float(far.max()) <= 0, name


KINDS = ["one", "two", "rising", "all", "all below zero"]


@pytest.mark.parametrize("dtype,top", [(t, 2.0**e) for t in (zi.BF16, zi.FP16) for e in (6, 10, 14, 18, 22, 26, 29)] + [(zi.FP16, 2.0**32), (zi.BF16, 2.0**60), (zi.BF16, 2.0**100)])
@pytest.mark.parametrize("d_head", [64, 80, 128])
@pytest.mark.parametrize("seq", [100, 300])
@pytest.mark.parametrize("kind", KINDS)
def test_matrix_cores(dtype, top, d_head, seq, kind):
    Led(dtype, seq, d_head, top, kind).hold()


@pytest.mark.parametrize("dtype,d_head,top", [(t, c, 2.0**e) for t, c in ((zi.BF16, 40), (zi.FP16, 8), (zi.FP32, 16)) for e in (6, 14, 22, 29)])
@pytest.mark.parametrize("seq", [40, 300])
@pytest.mark.parametrize("kind", KINDS)
def test_other_kernel(dtype, d_head, top, seq, kind):
    Led(dtype, seq, d_head, top, kind).hold()
