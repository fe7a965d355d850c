"""The linear layer's backward pass against 64 bits, element by element.

A result is a sum of terms of magnitude sum S.  16-bit types: the products' fp32 sums are off by at most (terms + 64) 2^-24 S whatever their order (64:
shares added up), G's rounding from fp32 (epilogues 2 and 3) by half a step of each term, and the result's own rounding comes on top.  db has no
rounding of G.  fp32: fp64 sums, and fp32's rounding of dw and db.
"""
import pytest
import torch

import paper_2507_03211_amd as zo_amd
import zo_inputs as zi
from gpu_util import DEV, act_dtype, resid_dtype
from grad_util import Out, generator, half, least, normal, param_dtype

pytestmark = pytest.mark.gpu
DTYPES = [zi.FP32, zi.BF16, zi.FP16]
# sizes that take every tile of both products, with one share and with several (test_every_tile_is_taken)
TILES = [(300, 264, 8192, 0), (4100, 72, 2048, 0), (300, 1288, 3000, 0), (2050, 264, 3848, 0), (129, 1536, 3000, 0), (4100, 4096, 264, 0), (129, 2304, 3848, 0),
         (4100, 8192, 264, 0), (129, 1288, 8192, 0), (4100, 1000, 5120, 0), (1000, 8, 8, 0), (515, 264, 3848, 0), (65, 3000, 3000, 0), (4100, 200, 768, 0),
         (2050, 8192, 8, 0), (2050, 200, 3000, 0), (4100, 4096, 8, 1), (2050, 200, 3848, 0), (1000, 8192, 1288, 0), (1500, 200, 8192, 0), (1048, 8192, 3000, 0), (1, 1288, 8, 0), (2050, 3000, 768, 0), (5000, 1000, 1288, 0), (8200, 1288, 2048, 0), (1000, 8192, 8192, 0)]
# sizes that have both products in one launch: each of its tiles, dw in one share and in several (test_every_joint_launch_is_taken)
JOINT = [(200, 200, 8, 0), (300, 264, 8, 1), (700, 520, 8192, 0), (1000, 264, 8, 0), (1500, 200, 520, 2), (6000, 1000, 768, 2), (2000, 2304, 768, 0), (1500, 1536, 1536, 1)]
SMALL = [(1, 8, 8), (1, 64, 64), (2, 72, 8), (3, 8, 200), (20, 768, 768), (63, 64, 128), (64, 128, 64), (65, 136, 72), (100, 1000, 1048), (257, 512, 256), (513, 2048, 640)]


class Layer:
    def __init__(self, dtype, rows, n, k, epilogue, relu_x, seed=0, dy=None):
        g = generator(seed + rows + 3 * n + 7 * k + epilogue)
        self.dtype, self.rows, self.n, self.k, self.epilogue, self.relu_x = dtype, rows, n, k, epilogue, relu_x
        a, p, r = act_dtype(dtype), param_dtype(dtype), resid_dtype(dtype)
        self.x = normal((rows, k), a, g)
        if relu_x:
            self.x.clamp_(min=0)
        self.w = normal((n, k), p, g, 0.05)
        self.y = normal((rows, n), a, g).clamp_(min=0) if epilogue == 1 else None
        self.dy = normal((rows, n), r if epilogue >= 2 else a, g, 0.02) if dy is None else dy
        self.dx, self.dw = Out((rows, k), a), Out((n, k), p)
        self.db = Out((n,), p) if epilogue != 3 else None
        self.scratch = self.workspace()

    def workspace(self):
        return torch.full((zo_amd.zo_kernel_linear_grad_scratch_bytes(self.dtype, self.rows, self.n, self.k, self.epilogue),), 0xFF, dtype=torch.uint8, device=DEV)

    def run(self, dx=True, dw=True, db=True, stream=None, x=True, w=True):
        at = lambda o, on: o.t if o is not None and on else None  # noqa: E731
        zo_amd.zo_kernel_linear_grad(self.x if x else None, self.w if w else None, self.y, self.dy, at(self.dx, dx), at(self.dw, dw), at(self.db, db), self.scratch,
                                     self.dtype, self.rows, self.n, self.k, self.epilogue, self.relu_x, stream)

    def outs(self):
        return [self.dx.t, self.dw.t] + ([self.db.t] if self.db else [])

    def whole(self):
        return self.dx.whole() and self.dw.whole() and (self.db is None or self.db.whole())

    def check(self, rows=None):
        """`rows`: of dx and dw, those compared (all, if None)."""
        u = 2.0**-53 if self.dtype == zi.FP32 else 2.0**-24
        grad = self.dy.double() if self.y is None else torch.where(self.y > 0, self.dy.double(), 0.0)
        x, w = self.x.double(), self.w.double()
        rounded = half(param_dtype(self.dtype)) if self.epilogue >= 2 and self.dtype != zi.FP32 else 0.0
        for out, left, right, keep in ((self.dx, grad, w, self.x if self.relu_x else None), (self.dw, grad.t(), x, None)):
            if rows is not None:
                left, keep = left[rows], keep if keep is None else keep[rows]
            got = out.t.double() if rows is None else out.t[rows].double()
            want, size = left @ right, left.abs() @ right.abs()
            if keep is not None:
                want = torch.where(keep > 0, want, 0.0)
                assert bool((got[~(keep > 0)] == 0).all())
            off = ((left.shape[1] + 64) * u + rounded) * size
            # (a 16-bit dy below the type's normal numbers is itself; an fp32 one rounds by the least step)
            tiny = least(out.t.dtype) + (least(out.t.dtype) * right.abs().sum(0) if rounded else 0.0)
            own = 0.0 if out.t.dtype == torch.float64 else half(out.t.dtype)
            assert bool(((got - want).abs() <= off + own * (want.abs() + off) + tiny).all())
        if self.db is not None:
            want, off = grad.sum(0), (self.rows + 64) * u * grad.abs().sum(0)
            assert bool(((self.db.t.double() - want).abs() <= off + half(self.db.t.dtype) * (want.abs() + off) + least(self.db.t.dtype)).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("epilogue", [0, 1, 2, 3])
@pytest.mark.parametrize("rows,n,k", SMALL)
def test_against_64_bits(dtype, epilogue, rows, n, k):
    for relu_x in (False, True):
        l = Layer(dtype, rows, n, k, epilogue, relu_x)
        l.run()
        torch.cuda.synchronize()
        assert l.whole()
        l.check()


@pytest.mark.parametrize("rows,n,k", [(1, 1, 1), (17, 3, 5), (65, 33, 31), (33, 300, 7), (300, 501, 203), (700, 520, 510)])
@pytest.mark.parametrize("epilogue", [0, 1, 2, 3])
def test_fp32_takes_any_size(rows, n, k, epilogue):
    l = Layer(zi.FP32, rows, n, k, epilogue, epilogue == 2)
    l.run()
    torch.cuda.synchronize()
    assert l.whole()
    l.check()


def test_every_tile_is_taken():
    seen = set()
    for shape in TILES:
        p = zo_amd.zo_kernel_linear_grad_plan(*shape)
        seen |= {("dx", p["dx"], p["dx_shares"] > 1), ("dw", p["dw"], p["dw_shares"] > 1)}
    tiles = [(256, 256), (256, 192), (256, 128), (192, 128), (128, 128), (64, 64)]
    assert seen == {(what, t, several) for what in ("dx", "dw") for t in tiles for several in (False, True)}


@pytest.mark.parametrize("dtype", [zi.BF16, zi.FP16])
@pytest.mark.parametrize("rows,n,k,epilogue", TILES)
@pytest.mark.parametrize("relu_x", [False, True])
def test_tiles(dtype, rows, n, k, epilogue, relu_x):
    l = Layer(dtype, rows, n, k, epilogue, relu_x)
    l.run()
    torch.cuda.synchronize()
    assert l.whole()
    step = lambda m: slice(None, None, max(1, m // 700))  # noqa: E731
    l.check(step(min(rows, n)))


def test_every_joint_launch_is_taken():
    seen = set()
    for shape in JOINT:
        p = zo_amd.zo_kernel_linear_grad_plan(*shape)
        assert p["both"] and 0 < p["both_dw"] < 256 and p["both_dw"] % 8 == 0 and p["dx_shares"] == 1
        seen.add((p["both"], p["dw_shares"] > 1))
    assert seen == {(t, several) for t in ((256, 256), (256, 128), (128, 128)) for several in (False, True)}


@pytest.mark.parametrize("dtype", [zi.BF16, zi.FP16])
@pytest.mark.parametrize("rows,n,k,epilogue", JOINT)
@pytest.mark.parametrize("relu_x", [False, True])
def test_both_products_in_one_launch(dtype, rows, n, k, epilogue, relu_x):
    l = Layer(dtype, rows, n, k, epilogue, relu_x)
    l.run()
    torch.cuda.synchronize()
    assert l.whole()
    l.check(slice(None, None, max(1, min(rows, n) // 500)))


@pytest.mark.parametrize("dtype", [zi.BF16, zi.FP16])
@pytest.mark.parametrize("rows,n,k,epilogue", TILES + JOINT)
def test_one_product_without_the_other(dtype, rows, n, k, epilogue):
    """dx alone and dw alone, in launches of their own: the bits of the call for both."""
    for relu_x in (False, True):
        l = Layer(dtype, rows, n, k, epilogue, relu_x)
        l.run()
        torch.cuda.synchronize()
        want = [t.clone() for t in (l.dx.t, l.dw.t)]
        for dx in (True, False):
            for t in l.outs():
                t.fill_(3.0)
            l.scratch.fill_(0xFF)
            l.run(dx, not dx, False, w=dx)
            torch.cuda.synchronize()
            assert l.whole()
            assert torch.equal(l.dx.t, want[0]) if dx else torch.equal(l.dw.t, want[1])


@pytest.mark.parametrize("dtype", [zi.BF16, zi.FP16])
@pytest.mark.parametrize("rows,n,k", [(1, 768, 768), (3, 576, 4096), (64, 768, 768), (200, 768, 768), (100, 1024, 1024), (20, 8192, 2048)])
@pytest.mark.parametrize("epilogue", [0, 2, 3])
@pytest.mark.parametrize("relu_x", [False, True])
def test_both_products_of_few_rows(dtype, rows, n, k, epilogue, relu_x):
    p = zo_amd.zo_kernel_linear_grad_plan(rows, n, k, epilogue)
    assert p["both"] == (64, 64) and (p["dx_shares"] > 1) == (n == 8192)
    l = Layer(dtype, rows, n, k, epilogue, relu_x)
    l.run()
    torch.cuda.synchronize()
    assert l.whole()
    l.check(slice(None, None, max(1, min(rows, n) // 50)))
    want = [t.clone() for t in (l.dx.t, l.dw.t)]
    l.run(dw=False, db=False)
    l.run(dx=False, db=False)
    torch.cuda.synchronize()
    assert torch.equal(l.dx.t, want[0]) and torch.equal(l.dw.t, want[1])


def test_plans_kept_stay_their_sizes_own():
    """More sizes than a thread keeps, in turn and over again, from two threads: the same bits as alone."""
    import threading
    layers = [Layer(zi.BF16, 40 + 13 * i, 64 + 8 * (i % 7), 72 + 8 * (i % 5), i % 3, False, i) for i in range(48)]
    want = []
    for l in layers:
        l.run()
        torch.cuda.synchronize()
        want.append([t.clone() for t in l.outs()])
    for l in layers:
        for t in l.outs():
            t.fill_(5.0)
        l.scratch.fill_(0xFF)
    torch.cuda.synchronize()

    def work(mine):
        for _ in range(3):
            for l in mine:
                l.run()
    threads = [threading.Thread(target=work, args=(layers[i::2],)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert all(l.whole() for l in layers)
    assert all(torch.equal(a, b) for l, w in zip(layers, want) for a, b in zip(l.outs(), w))


@pytest.mark.parametrize("dtype", [zi.BF16, zi.FP16])
@pytest.mark.parametrize("rows,n,k,epilogue", [(1048, 5000, 4096, 0), (2050, 13000, 1288, 2), (700, 13000, 3000, 1)])
def test_rows_behind_whole_rounds_of_tiles(dtype, rows, n, k, epilogue):
    p = zo_amd.zo_kernel_linear_grad_plan(rows, n, k, epilogue)
    assert p["dw_rows"] < n
    l = Layer(dtype, rows, n, k, epilogue, False)
    l.run()
    torch.cuda.synchronize()
    assert l.whole()
    step = max(1, rows // 300)
    l.check(slice(None, rows, step))                           # (dx's rows, and as many of dw's first)
    cut = p["dw_rows"]
    last = torch.cat([torch.arange(cut - 40, min(cut + 300, n)), torch.arange(n - 40, n)])
    grad = l.dy.double() if l.y is None else torch.where(l.y > 0, l.dy.double(), 0.0)
    left, right = grad.t()[last.to(DEV)], l.x.double()
    want, size = left @ right, left.abs() @ right.abs()
    off = ((rows + 64) * 2.0**-24 + (half(param_dtype(dtype)) if epilogue >= 2 else 0.0)) * size
    own = half(param_dtype(dtype))
    tiny = least(param_dtype(dtype)) * (1.0 + (right.abs().sum(0) if epilogue >= 2 else 0.0))
    assert bool(((l.dw.t[last.to(DEV)].double() - want).abs() <= off + own * (want.abs() + off) + tiny).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,n,k", [(65, 136, 72), (20, 768, 768), (700, 520, 256)])
def test_subsets_of_the_outputs(dtype, rows, n, k):
    """Any of the three alone, and those inputs NULL that it does not need: the same bits, nothing else written."""
    for epilogue in (0, 1, 2):
        l = Layer(dtype, rows, n, k, epilogue, False)
        l.run()
        torch.cuda.synchronize()
        want = [t.clone() for t in l.outs()]
        for on in range(1, 7):
            dx, dw, db = bool(on & 1), bool(on & 2), bool(on & 4)
            for t in l.outs():
                t.fill_(3.0)
            l.scratch.fill_(0xFF)
            l.run(dx, dw, db, x=dw, w=dx)
            torch.cuda.synchronize()
            for t, w, asked in zip(l.outs(), want, (dx, dw, db)):
                assert torch.equal(t, w) if asked else bool((t == 3.0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,n,k", [(65, 136, 72), (130, 256, 128)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_a_relu_holds_back_does_not_count(dtype, rows, n, k, bad):
    """dy where y is zero, and W's words where every G is: whatever they hold."""
    a, b = (Layer(dtype, rows, n, k, 1, True) for _ in range(2))
    a.dy[~(a.y > 0)] = bad
    b.dy[~(b.y > 0)] = 0.0
    for l in (a, b):
        l.run()
    torch.cuda.synchronize()
    assert all(torch.equal(s, t) for s, t in zip(a.outs(), b.outs()))
    a.check()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("epilogue", [0, 2])
@pytest.mark.parametrize("rows,n,k", [(65, 136, 72), (64, 128, 64), (200, 1000, 264)])
def test_what_is_not_finite_reaches_its_results(dtype, epilogue, rows, n, k):
    """A NaN in dy: its row of dx, its row of dw, its element of db; one in x: its column of dw; one in w: its column of dx; no other."""
    l = Layer(dtype, rows, n, k, epilogue, False)
    l.dy[rows // 2, n // 3] = float("nan")
    l.x[3, k - 1] = float("nan")
    l.w[n - 1, 5] = float("nan")
    l.run()
    torch.cuda.synchronize()
    want = [torch.zeros(s, dtype=torch.bool, device=DEV) for s in ((rows, k), (n, k), (n,))]
    want[0][rows // 2] = want[0][:, 5] = want[1][n // 3] = want[1][:, k - 1] = want[2][n // 3] = True
    assert all(torch.equal(torch.isnan(t), w) for t, w in zip(l.outs(), want))


@pytest.mark.parametrize("dtype", [zi.BF16, zi.FP16])
@pytest.mark.parametrize("epilogue", [0, 2])
def test_neighbours_in_memory_stay_out(dtype, epilogue):
    """Operands between buffers of NaN: nothing behind or in front of them is summed (sizes that end inside tiles and slabs)."""
    for rows, n, k in ((65, 136, 72), (33, 64, 200), (190, 72, 1032), (1048, 200, 264), (129, 1536, 3000)):
        l = Layer(dtype, rows, n, k, epilogue, False)
        for name in ("x", "w", "dy"):
            t = getattr(l, name)
            around = torch.full((t.numel() + (1 << 17),), float("nan"), dtype=t.dtype, device=DEV)
            inside = around[1 << 16:(1 << 16) + t.numel()].view(t.shape)
            inside.copy_(t)
            setattr(l, name, inside)
        l.run()
        torch.cuda.synchronize()
        assert l.whole()
        l.check(slice(None, None, max(1, min(rows, n) // 200)))


@pytest.mark.parametrize("epilogue", [0, 1, 2])
def test_gradients_by_differences(epilogue):
    """fp32: the derivative of sum(c y) along a direction of x, w and b at once, by central differences of the forward call itself.  y is at most
    bilinear in them, so the difference is exact but for fp64's rounding; weights lie on a grid of 2^-10 and directions on one of
    2^-2, so that a weight and 2^-22 of a direction add up exactly in fp32; outputs nearer zero than 2^-12 have no weight in the sum: no other changes sign."""
    rows, n, k, scale = 24, 40, 56, 2.0**-22
    l = Layer(zi.FP32, 2 * rows, n, k, epilogue, False, 5)
    g = generator(17)
    grid = lambda t, step: (t.double() / step).round() * step  # noqa: E731
    l.w.copy_(grid(l.w, 2.0**-10))
    b = grid(normal((n,), torch.float64, g, 0.1), 2.0**-10).float()
    dirs = [grid(normal(tuple(t.shape), torch.float64, g), 0.25) for t in (l.x, l.w, b)]
    base = normal((2 * rows, n), torch.float64, g)

    def forward(s):
        x, w, bias = l.x + s * dirs[0], (l.w.double() + s * dirs[1]).float(), (b.double() + s * dirs[2]).float()
        y = base.clone() if epilogue == 2 else torch.empty_like(base)
        zo_amd.zo_kernel_linear_pm(x, w, w, bias, bias, y, zi.FP32, rows, n, k, epilogue)
        return y
    l.dy[(l.x @ l.w.double().t() + b.double()).abs() < 2.0**-12] = 0.0
    if epilogue == 1:
        l.y = forward(0.0)
    l.run()
    plus, minus = forward(scale), forward(-scale)
    want = float((l.dy * (plus - minus)).sum()) / (2 * scale)
    got = sum(float((d * t.double()).sum()) for d, t in zip(dirs, l.outs()))
    size = sum(float((d * t.double()).abs().sum()) for d, t in zip(dirs, l.outs()))
    # dw and db rounded to fp32; y's fp64 sums of k terms
    y_off = (k + 4) * 2.0**-53 * float((l.dy.abs() * (l.x.abs() @ l.w.double().abs().t() + b.double().abs() + base.abs())).sum())
    assert abs(got - want) <= size * 2.0**-23 + 2 * y_off / (2 * scale)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,n,k,epilogue", [(20, 768, 768, 1), (700, 512, 640, 2), (65, 136, 72, 0)])
def test_captured_and_replayed(dtype, rows, n, k, epilogue):
    l = Layer(dtype, rows, n, k, epilogue, True)
    l.run(stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        l.run(stream=torch.cuda.current_stream())
    g = generator(3)
    for i in range(4):
        l.dy.copy_(normal((rows, n), torch.float64, g, 0.1))
        l.x.copy_(normal((rows, k), torch.float64, g).clamp(min=0))
        for t in l.outs():
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in l.outs()]
        l.scratch.fill_(85 * i)
        l.run(stream=torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, l.outs()))


def test_two_streams():
    ls = [Layer(zi.BF16, 700, 512, 640, 2, False) for _ in range(3)]
    ls[0].run()
    streams = [torch.cuda.Stream(device=DEV) for _ in ls[1:]]
    torch.cuda.synchronize()
    for l, s in zip(ls[1:], streams):
        l.run(stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for l in ls[1:] for a, b in zip(l.outs(), ls[0].outs()))


def test_more_bytes_than_32_bits_count():
    """dy, x and both results beyond 2^32 bytes; sampled rows."""
    l = Layer(zi.BF16, 262144 + 8, 8200, 8200, 0, False, dy=torch.zeros(1, device=DEV))
    g = generator(1)
    l.dy = torch.empty((l.rows, l.n), dtype=torch.bfloat16, device=DEV).normal_(0.0, 0.02, generator=g)
    l.run()
    torch.cuda.synchronize()
    assert l.whole()
    w = l.w.double()
    for r in (0, 131071, l.rows - 1):
        grad = l.dy[r].double()
        want, size = grad @ w, grad.abs() @ w.abs()
        off = (l.n + 64) * 2.0**-24 * size
        assert bool(((l.dx.t[r].double() - want).abs() <= off + half(torch.bfloat16) * (want.abs() + off)).all())
    for c in (0, l.n - 1):
        grad = l.dy[:, c].double()
        want, size = (sum((f(grad[i:i + 16384]) @ f(l.x[i:i + 16384].double())) for i in range(0, l.rows, 16384)) for f in (lambda t: t, torch.abs))
        # sums over rows: their order is a tree of shares, slabs and matrix instructions, each chain at most rows / 16 long
        off = (l.rows / 16 + 64) * 2.0**-24 * size
        assert bool(((l.dw.t[c].double() - want).abs() <= off + half(torch.bfloat16) * (want.abs() + off)).all())
