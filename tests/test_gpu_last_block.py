"""The gradient carried from the head through the last decoder block, and the step, as a program takes them: forward calls, head, LayerNorm, both
projections, attention, LayerNorm, clipping's norm and AdamW, one after the other on one stream; held to 64-bit automatic differentiation of
the same block, and to itself when captured and replayed.
"""
import math

import pytest
import torch

import paper_2507_03211_amd as zo_amd
import zo_inputs as zi
from gpu_util import DEV, act_dtype, resid_dtype
from grad_util import generator, half, normal, param_dtype

pytestmark = pytest.mark.gpu
LN_EPS = float(torch.tensor(1e-5, dtype=torch.float32))
NAMES = ["ln1_g", "ln1_b", "wqkv", "bqkv", "wo", "bo", "ln2_g", "ln2_b", "w1", "b1", "w2", "b2", "lnf_g", "lnf_b", "e"]


class Block:
    def __init__(self, dtype, batch, seq, heads, d_head, ffn, vocab, seed=0):
        d, rows = heads * d_head, batch * seq
        g = generator(seed + d + rows + ffn)
        self.dtype, self.batch, self.seq, self.heads, self.d_head, self.d, self.ffn, self.vocab, self.rows = dtype, batch, seq, heads, d_head, d, ffn, vocab, rows
        p, a, r = param_dtype(dtype), act_dtype(dtype), resid_dtype(dtype)
        shapes = dict(ln1_g=(d,), ln1_b=(d,), wqkv=(3 * d, d), bqkv=(3 * d,), wo=(d, d), bo=(d,), ln2_g=(d,), ln2_b=(d,), w1=(ffn, d), b1=(ffn,), w2=(d, ffn), b2=(d,),
                      lnf_g=(d,), lnf_b=(d,), e=(vocab, d))
        self.w = {n: ((1.0 if n.endswith("_g") else 0.0) + normal(shapes[n], torch.float64, g, 0.1 if len(shapes[n]) == 1 else 1.5 / math.sqrt(shapes[n][1]))).to(p)
                  for n in NAMES}
        self.grad = {n: torch.empty_like(t) for n, t in self.w.items()}
        self.h0 = normal((rows, d), r, g)
        self.target = torch.randint(0, vocab, (rows,), device=DEV, generator=g).to(torch.int32)
        self.target.view(batch, seq)[:, -1] = -1
        self.count = int((self.target >= 0).sum())
        empty = lambda shape, t: torch.empty(shape, dtype=t, device=DEV)  # noqa: E731
        self.h, self.mid_h, self.dh = (empty((rows, d), r) for _ in range(3))
        self.x1, self.att, self.x2, self.xf, self.dx, self.datt = (empty((rows, d), a) for _ in range(6))
        self.qkv, self.dqkv, self.up, self.dup = empty((rows, 3 * d), a), empty((rows, 3 * d), a), empty((rows, ffn), a), empty((rows, ffn), a)
        self.stats = [(empty((rows,), r), empty((rows,), r)) for _ in range(3)]
        self.loss, self.norm = empty((rows,), r), empty((2,), torch.float64)
        n = [zo_amd.zo_kernel_lmhead_grad_scratch_bytes(dtype, rows, d, vocab), zo_amd.zo_kernel_layernorm_grad_scratch_bytes(dtype, rows, d),
             zo_amd.zo_kernel_grad_clip_scratch_bytes(), zo_amd.zo_kernel_attention_grad_scratch_bytes(dtype, batch, seq, heads, d_head)]
        n += [zo_amd.zo_kernel_linear_grad_scratch_bytes(dtype, rows, *s) for s in ((3 * d, d, 0), (d, d, 2), (ffn, d, 0), (d, ffn, 2))]
        self.scratch = empty((max(n),), torch.uint8)             # calls of one stream share it
        self.state = {k: torch.zeros(zo_amd.zo_kernel_adamw_state_bytes(t.numel(), 32), dtype=torch.uint8, device=DEV) for k, t in self.w.items()}

    def forward(self, s=None):
        half_rows, w, dt = self.rows // 2, self.w, self.dtype

        def linear(x, name, bias, y, epilogue):
            zo_amd.zo_kernel_linear_pm(x, w[name], w[name], w[bias], w[bias], y, dt, half_rows, *w[name].shape, epilogue, s)

        def norm(x, name, y, stats):
            zo_amd.zo_kernel_layernorm(x, w[name + "_g"], w[name + "_b"], y, *stats, dt, self.rows, self.d, LN_EPS, s)
        self.mid_h.copy_(self.h0)
        norm(self.h0, "ln1", self.x1, self.stats[0])
        linear(self.x1, "wqkv", "bqkv", self.qkv, 0)
        zo_amd.zo_kernel_attention(self.qkv, self.att, dt, self.batch, self.seq, self.heads, self.d_head, s)
        linear(self.att, "wo", "bo", self.mid_h, 2)
        norm(self.mid_h, "ln2", self.x2, self.stats[1])
        linear(self.x2, "w1", "b1", self.up, 1)
        self.h.copy_(self.mid_h)
        linear(self.up, "w2", "b2", self.h, 2)
        norm(self.h, "lnf", self.xf, self.stats[2])

    def backward(self, s=None, scale=1.0, relu_x=True):
        w, g, dt, rows = self.w, self.grad, self.dtype, self.rows
        zo_amd.zo_kernel_lmhead_grad(self.xf, w["e"], self.target, self.loss, self.dx, g["e"], self.scratch, dt, rows, self.d, self.vocab, scale / self.count, s)

        def norm(x, name, stats, more):
            zo_amd.zo_kernel_layernorm_grad(self.dx, x, w[name + "_g"], *stats, self.dh, g[name + "_g"], g[name + "_b"], self.scratch, dt, rows, self.d, more, s)

        def linear(x, name, bias, y, dy, dx, epilogue, relu=False):
            zo_amd.zo_kernel_linear_grad(x, w[name], y, dy, dx, g[name], g[bias], self.scratch, dt, rows, *w[name].shape, epilogue, relu, s)
        norm(self.h, "lnf", self.stats[2], False)
        linear(self.up, "w2", "b2", None, self.dh, self.dup, 2, relu_x)
        linear(self.x2, "w1", "b1", None if relu_x else self.up, self.dup, self.dx, 0 if relu_x else 1)
        norm(self.mid_h, "ln2", self.stats[1], True)
        linear(self.att, "wo", "bo", None, self.dh, self.datt, 2)
        zo_amd.zo_kernel_attention_grad(self.qkv, self.att, self.datt, self.dqkv, self.scratch, dt, self.batch, self.seq, self.heads, self.d_head, s)
        linear(self.x1, "wqkv", "bqkv", None, self.dqkv, self.dx, 0)
        norm(self.h0, "ln1", self.stats[0], True)

    def update(self, t, lr, s=None, max_norm=math.inf):
        names = list(NAMES)
        numel, grads = [self.w[n].numel() for n in names], [self.grad[n] for n in names]
        zo_amd.zo_kernel_grad_clip(grads, grads, numel, len(names), self.dtype, math.inf, self.norm, self.scratch, s)
        zo_amd.zo_kernel_adamw([self.w[n] for n in names], grads, [self.state[n] for n in names], numel, len(names), self.dtype, 32, lr, 0.9, 0.95, 1e-8, 0.0, t,
                               self.norm, max_norm, stream=s)

    def loss64(self, h0, w):
        def norm(x, name):
            m = x.mean(1, keepdim=True)
            return (x - m) * ((x - m).square().mean(1, keepdim=True) + LN_EPS).rsqrt() * w[name + "_g"] + w[name + "_b"]
        q, k, v = (norm(h0, "ln1") @ w["wqkv"].t() + w["bqkv"]).view(self.batch, self.seq, 3, self.heads, self.d_head).permute(2, 0, 3, 1, 4)
        score = q @ k.transpose(2, 3) / math.sqrt(self.d_head)
        score = score.masked_fill(torch.ones(self.seq, self.seq, dtype=torch.bool, device=DEV).triu(1), -math.inf)
        att = (torch.softmax(score, 3) @ v).permute(0, 2, 1, 3).reshape(self.rows, self.d)
        h = h0 + att @ w["wo"].t() + w["bo"]
        # on the ReLU's branches that the forward calls took: an input that rounds to the other side of zero switches its whole term, not by a rounding
        h = h + ((norm(h, "ln2") @ w["w1"].t() + w["b1"]) * (self.up > 0)) @ w["w2"].t() + w["b2"]
        l = norm(h, "lnf") @ w["e"].t()
        at = self.target.clamp(min=0).long()[:, None]
        return torch.where(self.target >= 0, torch.logsumexp(l, 1) - l.gather(1, at).squeeze(1), 0.0).sum() / self.count


@pytest.mark.parametrize("dtype", [zi.FP32, zi.BF16, zi.FP16])
@pytest.mark.parametrize("batch,seq,heads,d_head,ffn,vocab", [(2, 32, 4, 16, 256, 512), (2, 65, 3, 64, 768, 1000), (4, 131, 2, 128, 1024, 2056)])
def test_chain(dtype, batch, seq, heads, d_head, ffn, vocab):
    """By 64-bit automatic differentiation.  On its way from the head to the block's input a gradient passes eleven roundings to 16 bits (probabilities, dx of
    head, two projections, dS, dqkv, two more projections' operands and dx, itself), the activations it meets nine; each is half a step at most, independent
    from element to element and spread over sums, so that 20 half steps of the norm bound what is compared, on the branches of the ReLU that the forward calls
    took (a fraction f of its inputs on the other side of zero changes a gradient by sqrt(f) of its norm: 2^-11 of them by 2 %).  fp32: each result's own rounding, and fp64 sums."""
    m = Block(dtype, batch, seq, heads, d_head, ffn, vocab)
    scale = 1024.0 if dtype == zi.FP16 else 1.0
    m.forward()
    m.backward(scale=scale)
    leaves = {n: t.double().requires_grad_() for n, t in m.w.items()}
    h0 = m.h0.double().requires_grad_()
    m.loss64(h0, leaves).backward()
    step = half(act_dtype(dtype)) if dtype != zi.FP32 else 2.0**-24
    for got, leaf in [(m.dh, h0)] + [(m.grad[n], leaves[n]) for n in NAMES]:
        want = scale * leaf.grad
        assert float(torch.linalg.vector_norm(got.double() - want)) <= 20 * step * float(torch.linalg.vector_norm(want))


@pytest.mark.parametrize("dtype", [zi.FP32, zi.BF16])
def test_relu_taken_back_by_either_call(dtype):
    m = Block(dtype, 2, 65, 2, 64, 520, 512, 1)
    m.forward()
    m.backward()
    want = {n: t.clone() for n, t in m.grad.items()}
    m.backward(relu_x=False)
    assert all(torch.equal(want[n], m.grad[n]) for n in NAMES)


@pytest.mark.parametrize("dtype", [zi.FP32, zi.BF16, zi.FP16])
def test_captured_steps(dtype):
    """Forward, backward and step in one graph, replayed: the eager program's bits, weights and moments moving on from step to step."""
    a, b = (Block(dtype, 2, 40, 2, 64, 264, 520, 4) for _ in range(2))

    def step(m, s):
        m.forward(s)
        m.backward(s, 64.0 if dtype == zi.FP16 else 1.0)
        m.update(3, 1e-3, s, 0.5)
    for m in (a, b):
        step(m, torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, torch.cuda.current_stream())
    for i in range(4):
        for m in (a, b):
            m.h0.copy_(normal(tuple(m.h0.shape), torch.float64, generator(50 + i)))
        a.scratch.fill_(85 * i)
        graph.replay()
        torch.cuda.synchronize()
        step(b, torch.cuda.current_stream())
        torch.cuda.synchronize()
        for n in NAMES:
            assert torch.equal(a.w[n], b.w[n]) and torch.equal(a.state[n], b.state[n]) and torch.equal(a.grad[n], b.grad[n])
        assert float(a.norm[0]) == float(b.norm[0]) and math.isfinite(float(a.norm[0]))
