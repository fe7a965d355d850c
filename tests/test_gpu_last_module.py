"""The last module's gradient as a program takes it: LayerNorm, head, LayerNorm's backward pass and clipping, one after the other
on one stream; held to the whole chain in 64 bits, to z . grad L as a zeroth-order step's g sees it, and to itself when captured into a
graph and replayed.
"""
import pytest
import torch

import paper_2507_03211_amd as zo_amd
import zo_inputs as zi
from gpu_util import DEV, act_dtype, resid_dtype
from grad_util import generator, half, normal, param_dtype

pytestmark = pytest.mark.gpu
EPS = float(torch.tensor(1e-5, dtype=torch.float32))            # as the call gets it


class Module:
    """Buffers of one last module: parameters, a batch, everything a step needs beside them."""

    def __init__(self, dtype, rows, d, vocab, seed=0):
        g = generator(seed + rows + d + vocab)
        self.dtype, self.rows, self.d, self.vocab = dtype, rows, d, vocab
        p, a, r = param_dtype(dtype), act_dtype(dtype), resid_dtype(dtype)
        self.h = normal((rows, d), r, g, 2.0)
        self.gain, self.bias = (1.0 + normal((d,), torch.float64, g, 0.2)).to(p), normal((d,), p, g, 0.2)
        self.e = normal((vocab, d), p, g, 0.05)
        self.target = torch.randint(0, vocab, (rows,), device=DEV, generator=g).to(torch.int32)
        self.target[rows - 1::7] = -1
        self.count = int((self.target >= 0).sum())
        empty = lambda shape, t: torch.empty(shape, dtype=t, device=DEV)  # noqa: E731
        self.y, self.dy, self.dh = empty((rows, d), a), empty((rows, d), a), empty((rows, d), r)
        self.mean, self.rstd, self.loss = (empty((rows,), r) for _ in range(3))
        self.de, self.dg, self.db = torch.empty_like(self.e), torch.empty_like(self.gain), torch.empty_like(self.bias)
        self.norm = empty((2,), torch.float64)
        n = [zo_amd.zo_kernel_lmhead_grad_scratch_bytes(dtype, rows, d, vocab), zo_amd.zo_kernel_layernorm_grad_scratch_bytes(dtype, rows, d),
             zo_amd.zo_kernel_grad_clip_scratch_bytes()]
        self.scratch = empty((max(n),), torch.uint8)             # calls of one stream share it

    def step(self, max_norm=float("inf"), scale=1.0):
        s, a = torch.cuda.current_stream(), (self.dtype, self.rows, self.d)
        zo_amd.zo_kernel_layernorm(self.h, self.gain, self.bias, self.y, self.mean, self.rstd, *a, EPS, s)
        zo_amd.zo_kernel_lmhead_grad(self.y, self.e, self.target, self.loss, self.dy, self.de, self.scratch, *a, self.vocab, scale / self.count, s)
        zo_amd.zo_kernel_layernorm_grad(self.dy, self.h, self.gain, self.mean, self.rstd, self.dh, self.dg, self.db, self.scratch, *a, False, s)
        grads = [self.de, self.dg, self.db]
        zo_amd.zo_kernel_grad_clip(grads, grads, [t.numel() for t in grads], 3, self.dtype, max_norm, self.norm, self.scratch, s)

    def outs(self):
        return [self.loss, self.dh, self.de, self.dg, self.db, self.norm]

    def loss64(self, h, gain, bias, e):
        m = h.mean(1, keepdim=True)
        y = (h - m) * ((h - m).square().mean(1, keepdim=True) + EPS).rsqrt() * gain + bias
        l = y @ e.t()
        at = self.target.clamp(min=0).long()[:, None]
        return torch.where(self.target >= 0, torch.logsumexp(l, 1) - l.gather(1, at).squeeze(1), 0.0).sum() / self.count


@pytest.mark.parametrize("dtype", [zi.FP32, zi.BF16, zi.FP16])
@pytest.mark.parametrize("rows,d,vocab", [(62, 64, 512), (331, 192, 2056), (16, 768, 9000)])
def test_chain(dtype, rows, d, vocab):
    """The whole chain by 64-bit automatic differentiation.  A gradient passes four roundings to 16 bits (y, the
    probabilities, dy, itself), each independent from element to element and half a step at most, three of them spread over
    sums: 4 half steps of the norm of what is compared; fp32: its own rounding, 2^-24, and fp64 sums."""
    m = Module(dtype, rows, d, vocab)
    scale = 1024.0 if dtype == zi.FP16 else 1.0
    m.step(scale=scale)
    leaves = [t.double().requires_grad_() for t in (m.h, m.gain, m.bias, m.e)]
    loss = m.loss64(*leaves)
    loss.backward()
    step = half(act_dtype(dtype)) if dtype != zi.FP32 else 2.0**-24
    assert abs(float(m.loss.double().sum()) / m.count - float(loss.detach())) <= 4 * step * (1.0 + abs(float(loss.detach())))
    for got, leaf in zip((m.dh, m.dg, m.db, m.de), leaves):
        want = scale * leaf.grad
        assert float(torch.linalg.vector_norm(got.double() - want)) <= 4 * step * float(torch.linalg.vector_norm(want))
    whole = float(torch.sqrt(sum(t.double().square().sum() for t in (m.de, m.dg, m.db))))
    assert abs(float(m.norm[0]) - whole) <= 1e-11 * whole


def test_z_dot_gradient():
    """Eq. 2's g, with the last module alone perturbed by the library's own z, against z . grad L: (L+ - L-) / 2 eps at eps and eps / 2,
    the finer one off by a third of what they differ by.  Losses and gradient come from the same calls; parameters are fp32, their
    perturbed values rounded by 2^-24 of at most 1.5 each, independently."""
    m = Module(zi.FP32, 62, 64, 512, 3)
    m.step()
    grads = [(0, m.e, m.de.clone()), (1, m.gain, m.dg.clone()), (2, m.bias, m.db.clone())]
    seed, g, zs = 1234, [], []
    for tid, t, _ in grads:
        z = torch.empty(t.numel(), device=DEV)
        zo_amd.zo_kernel_z(z, t.numel(), seed, tid)
        zs.append(z.double())
    keep = [t.clone() for _, t, _ in grads]
    for eps in (1e-2, 5e-3):
        loss = []
        for sign in (eps, -eps):
            for (tid, t, _), k in zip(grads, keep):
                zo_amd.zo_kernel_axpy_z(k, t, zi.FP32, t.numel(), seed, tid, sign)
            m.step()
            loss.append(float(m.loss.sum()) / m.count)
        g.append((loss[0] - loss[1]) / (2 * eps))
    want = sum(float((z * d.double().reshape(-1)).sum()) for z, (_, _, d) in zip(zs, grads))
    size = float(torch.sqrt(sum(d.double().square().sum() for _, _, d in grads)))
    assert abs(g[1] - want) <= abs(g[0] - g[1]) + 7 * 2.0**-24 * 1.5 * size / 5e-3


@pytest.mark.parametrize("dtype", [zi.FP32, zi.BF16, zi.FP16])
@pytest.mark.parametrize("rows,d,vocab", [(62, 64, 512), (24, 768, 9000), (700, 256, 4104)])
def test_captured_and_replayed(dtype, rows, d, vocab):
    """Replays of a captured chain give the eager call's bits, with other inputs in the same buffers, eager work between."""
    m = Module(dtype, rows, d, vocab, 1)
    m.step(0.5)                                                   # (what a first launch sets up, outside the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.step(0.5)
    g = generator(9)
    for i in range(4):
        m.h.copy_(normal((rows, d), torch.float64, g, 1.0 + i))
        m.target.copy_(torch.randint(0, vocab, (rows,), device=DEV, generator=g))
        m.target[i] = -1
        for t in m.outs():
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in m.outs()]
        m.scratch.fill_(i * 85)
        m.step(0.5)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, m.outs()))


def test_two_graphs_with_workspaces_of_their_own():
    """Two captured chains replayed at the same time on two streams."""
    ms = [Module(zi.BF16, 400, 256, 4104, s) for s in (1, 2)]
    graphs, want = [], []
    for m in ms:
        m.step(0.5)
        torch.cuda.synchronize()
        want.append([t.clone() for t in m.outs()])
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            m.step(0.5)
    streams = [torch.cuda.Stream(device=DEV) for _ in ms]
    for _ in range(3):
        for m in ms:
            for t in m.outs():
                t.zero_()
        torch.cuda.synchronize()
        for s, gr in zip(streams, graphs):
            with torch.cuda.stream(s):
                gr.replay()
        torch.cuda.synchronize()
        for m, w in zip(ms, want):
            assert all(torch.equal(a, b) for a, b in zip(m.outs(), w))
