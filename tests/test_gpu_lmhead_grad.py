"""Cross entropy of the tied LM head with its gradient against the formulas in 64 bits, element by element.

Tolerances (16-bit types).  A logit is a sum of d products in fp32: off by A u sum |x e|, A = 16 + d / 8 (the matrix
instructions add sixteen products at a time; the row's largest such error is `dl`).  A probability is off by 2 dl + 2^-21 of itself: its
own logit, the row's logsumexp, and exponential, sums and roundings of 32 bits.  A logit may be kept as a distance in steps of 32 / 65535,
which moves the probability by half of that, and counts as none from 32 on (e^-32 of a neighbour's probability); the probability enters the
products rounded to the 16-bit type, by half a step.  `h` is the root of both squared.  These roundings are independent, so a sum of n such terms is off by 7 h sqrt(sum of squares) (bounded
independent terms pass that once in 10^10), everything else by its worst case; then the result is rounded, half a step.
fp32 parameters: all in fp64, results of the parameters' type rounded once.
"""
import math

import pytest
import torch

import paper_2507_03211_amd as zo_amd
import zo_inputs as zi
from gpu_util import DEV, act_dtype, resid_dtype
from grad_util import Out, generator, half, least, normal, param_dtype, unit

pytestmark = pytest.mark.gpu
HALVES = [zi.BF16, zi.FP16]


def inputs(dtype, rows, d, vocab, seed=0, lean=12.0, std=0.05):
    g = generator(seed + 7 * rows + 13 * d + vocab)
    e = normal((vocab, d), param_dtype(dtype), g, std)
    target = torch.randint(0, vocab, (rows,), device=DEV, generator=g)
    x = normal((rows, d), torch.float64, g)
    x = (x + lean / (std * std * d) * torch.rand((rows, 1), device=DEV, generator=g, dtype=torch.float64) * e[target].double()).to(act_dtype(dtype))
    if rows > 2:
        target[torch.randperm(rows, device=DEV, generator=g)[:max(1, rows // 7)]] = -1
    return x, e, target.to(torch.int32)


def call(dtype, x, e, target, scale, stream=None):
    (rows, d), vocab = x.shape, e.shape[0]
    loss, dx, de = Out((rows,), resid_dtype(dtype)), Out((rows, d), act_dtype(dtype)), Out((vocab, d), param_dtype(dtype))
    scratch = Out((zo_amd.zo_kernel_lmhead_grad_scratch_bytes(dtype, rows, d, vocab),), torch.uint8)
    zo_amd.zo_kernel_lmhead_grad(x, e, target, loss.t, dx.t, de.t, scratch.t, dtype, rows, d, vocab, scale, stream)
    torch.cuda.synchronize()
    assert loss.whole() and dx.whole() and de.whole() and scratch.whole()
    return loss.t, dx.t, de.t


def check(dtype, x, e, target, scale, got, words=slice(None)):
    """x's rows of targets < 0 are taken as zeros; the scale is an fp32 number, as the call gets it.  `words`: whose de is looked at."""
    scale = float(torch.tensor(scale, dtype=torch.float32))
    loss, dx, de = got
    (rows, d), vocab = x.shape, e.shape[0]
    live = target >= 0
    xd, ed = torch.where(live[:, None], x.double(), 0.0), e.double()
    at = target.clamp(min=0).long()[:, None]
    logits = xd @ ed.t()
    lse = torch.logsumexp(logits, 1, keepdim=True)
    p = torch.exp(logits - lse)
    hit = logits.gather(1, at)
    G = p.clone()
    G.scatter_(1, at, torch.expm1(hit - lse))
    G[~live] = 0.0
    want_loss = torch.where(live, (lse - hit).squeeze(1), 0.0)
    u = unit(dtype)
    dl = ((16 + d / 8) * u * (xd.abs() @ ed.abs().t()).amax(1, keepdim=True))
    rel = 2 * dl + (2.0**-21 if dtype != zi.FP32 else 2.0**-48)
    # beside the roundings to 16 bits, in absolute size: every probability by `rel` of itself, the target's by that of p
    off_G = 1.1 * rel * p
    off_G[~live] = 0.0
    assert ((loss.double() - want_loss).abs() <= 2 * dl.squeeze(1) + 8 * u * (1.0 + lse.abs() + hit.abs()).squeeze(1)).all()
    assert (loss[~live] == 0).all() and (dx[~live] == 0).all()
    h = 0.0 if dtype == zi.FP32 else (half(act_dtype(dtype))**2 + (16.0 / 65535)**2)**0.5
    tiny = 0.0 if dtype == zi.FP32 else math.exp(-32.0) + (2.0**-39 if dtype == zi.FP16 else 0.0)    # the latter: half the step of probabilities below fp16's normal numbers, 2^15 times enlarged
    for out, A, B, n in ((dx, G, ed, vocab), (de[words], G[:, words].t().contiguous(), xd, rows)):
        off = off_G if out is dx else off_G[:, words].t().contiguous()
        want = scale * (A @ B)
        t = out.dtype
        tol = half(t) * want.abs() + abs(scale) * (
            7 * h * torch.sqrt(A.square() @ B.square()) + (off + tiny * (A != 0)) @ B.abs() + (24 + n / 8) * u * (A.abs() @ B.abs()))
        assert ((out.double() - want).abs() <= 1.02 * tol + least(t)).all(), "dx" if out is dx else "de"


SHAPES = [
    (1, 64, 8), (1, 768, 50272), (2, 8, 16), (5, 72, 200), (20, 768, 50272), (33, 64, 520), (62, 128, 512), (64, 64, 64), (65, 200, 1000),
    (130, 192, 4104), (257, 320, 2600), (300, 384, 8008), (513, 1024, 3000), (700, 264, 5000), (1048, 640, 6824), (2100, 128, 2056), (2049, 576, 4160),
]


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("rows,d,vocab", SHAPES)
def test_sixteen_bits(dtype, rows, d, vocab):
    x, e, target = inputs(dtype, rows, d, vocab)
    scale = (4096.0 if dtype == zi.FP16 else 1.0) / rows
    check(dtype, x, e, target, scale, call(dtype, x, e, target, scale))


@pytest.mark.parametrize("rows,d,vocab", [(1, 1, 2), (3, 7, 11), (62, 64, 512), (65, 130, 517), (300, 96, 1001)])
def test_fp32_parameters(rows, d, vocab):
    x, e, target = inputs(zi.FP32, rows, d, vocab)
    check(zi.FP32, x, e, target, 1.0 / rows, call(zi.FP32, x, e, target, 1.0 / rows))


def test_fp32_parameters_in_pieces():
    """More logits than a piece holds: 2^25 of them are worked at a time."""
    rows, d, vocab = 2100, 16, 17000
    x, e, target = inputs(zi.FP32, rows, d, vocab)
    check(zi.FP32, x, e, target, 0.5, call(zi.FP32, x, e, target, 0.5))


@pytest.mark.parametrize("dtype", [zi.FP32, zi.BF16, zi.FP16])
@pytest.mark.parametrize("rows", [40, 600])
def test_rows_that_do_not_count(dtype, rows):
    """Whatever such a row holds, all else is as if it held zeros."""
    d, vocab = 128, 1000
    x, e, target = inputs(dtype, rows, d, vocab, 3)
    target[rows // 3:rows // 2] = -1
    target[rows - 1] = -7
    x[target < 0] = 0.0
    a = call(dtype, x, e, target, 0.25)
    x[target < 0] = float("nan")
    x[rows // 3] = float("inf")
    b = call(dtype, x, e, target, 0.25)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    check(dtype, x, e, target, 0.25, b)
    target[:] = -1
    assert all((t == 0).all() for t in call(dtype, x, e, target, 0.25))


@pytest.mark.parametrize("dtype", [zi.FP32, zi.BF16, zi.FP16])
@pytest.mark.parametrize("rows", [9, 400])
def test_targets_beyond_the_vocabulary(dtype, rows):
    d, vocab = 64, 520
    x, e, target = inputs(dtype, rows, d, vocab, 4)
    target[4], target[5] = vocab, 5
    loss, dx, de = call(dtype, x, e, target, 1.0)
    assert torch.isnan(loss[4]) and torch.isnan(dx[4]).all() and torch.isnan(de).all()
    keep = torch.arange(rows, device=DEV) != 4
    assert torch.isfinite(loss[keep]).all() and torch.isfinite(dx[keep]).all()


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("rows", [12, 384])
@pytest.mark.parametrize("size", [1.0, 50.0, 3000.0])
def test_logits_of_all_sizes(dtype, rows, size):
    """Rows of one word's embedding times `size`: from soft answers to ones that are certain, and certainly wrong."""
    d, vocab = 128, 776
    x, e, target = inputs(dtype, rows, d, vocab, 5, std=0.3)
    word = torch.arange(rows, device=DEV) * 3 % vocab
    x = (e[word].double() * size).to(act_dtype(dtype))
    target[::2] = word[::2].int()                              # half the rows answer with the target
    target[3] = -1
    check(dtype, x, e, target, 1.0 / rows, call(dtype, x, e, target, 1.0 / rows))


@pytest.mark.parametrize("dtype", [zi.FP32, zi.BF16, zi.FP16])
@pytest.mark.parametrize("rows", [10, 300])
def test_numbers_that_are_not_finite(dtype, rows):
    """A NaN or infinite row that counts spoils its loss, its dx and de; the other rows' losses and dx stay."""
    d, vocab = 64, 304
    for bad in (float("nan"), float("inf")):
        x, e, target = inputs(dtype, rows, d, vocab, 6)
        target[2], target[3] = 17, 18
        x[2, 5] = bad
        loss, dx, de = call(dtype, x, e, target, 1.0)
        keep = torch.arange(rows, device=DEV) != 2
        assert torch.isnan(loss[2]) and torch.isnan(dx[2]).all() and torch.isnan(de).any()
        assert torch.isfinite(loss[keep]).all() and torch.isfinite(dx[keep]).all()


@pytest.mark.parametrize("dtype,rows,d,vocab", [
    (zi.BF16, 10, 64, 1000), (zi.FP16, 10, 64, 1000), (zi.BF16, 600, 128, 4096), (zi.FP16, 600, 128, 4096), (zi.BF16, 140, 320, 1 << 22), (zi.FP32, 10, 64, 304),
    (zi.FP32, 100, 16, 6000), (zi.FP32, 2100, 16, 17000)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_words_that_are_not_finite(dtype, rows, d, vocab, bad):
    """Whole neighbourhoods of words that are not finite, and no others: a row that counts has a loss only where the formula has one."""
    x, e, target = inputs(dtype, rows, d, vocab, 16)
    for words in (slice(0, 512), slice(vocab - 512, vocab)) if vocab > 1024 else (slice(0, 256),):
        if (dtype, rows) == (zi.FP32, 2100):
            words = slice(0, 16000) if words.start == 0 else slice(16000, vocab)         # a whole piece of logits, and a part of one
        bent = e.clone()
        bent[words] = bad
        loss, dx, de = call(dtype, x, bent, target, 1.0)
        live = target >= 0
        logits = torch.where(live[:, None], x.double(), 0.0) @ bent.double().t()
        want = torch.logsumexp(logits, 1) - logits.gather(1, target.clamp(min=0).long()[:, None]).squeeze(1)
        assert torch.equal(torch.isfinite(loss[live]), torch.isfinite(want[live])) and (loss[~live] == 0).all() and torch.isnan(dx[live]).all()


@pytest.mark.parametrize("dtype", [zi.FP32, zi.BF16, zi.FP16])
@pytest.mark.parametrize("rows,d,vocab", [(16, 256, 4096), (520, 256, 4096)])
def test_same_bits_every_time_on_any_stream(dtype, rows, d, vocab):
    x, e, target = inputs(dtype, rows, d, vocab, 8)
    first = call(dtype, x, e, target, 0.01)
    streams = [torch.cuda.Stream(device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    # two calls under way at once, each with a workspace of its own, other bytes in it
    outs = []
    for i, s in enumerate(streams):
        o = [Out((rows,), resid_dtype(dtype)), Out((rows, d), act_dtype(dtype)), Out((vocab, d), param_dtype(dtype))]
        scratch = torch.full((zo_amd.zo_kernel_lmhead_grad_scratch_bytes(dtype, rows, d, vocab),), 0xFF * i, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        outs.append((o, scratch))
    for s, (o, scratch) in zip(streams, outs):
        zo_amd.zo_kernel_lmhead_grad(x, e, target, o[0].t, o[1].t, o[2].t, scratch, dtype, rows, d, vocab, 0.01, s)
    torch.cuda.synchronize()
    for o, _ in outs:
        assert all(torch.equal(a.t, b) for a, b in zip(o, first))


def test_same_word_many_times():
    """All rows ask for one word, and all rows are alike: its gradient is the sum of as many equal shares."""
    dtype, rows, d, vocab = zi.BF16, 333, 192, 1024
    x, e, target = inputs(dtype, rows, d, vocab, 9)
    target[:] = 1021
    check(dtype, x, e, target, 1.0 / rows, call(dtype, x, e, target, 1.0 / rows))


@pytest.mark.parametrize("dtype", [zi.FP32, zi.BF16])
def test_against_differences(dtype):
    """The mean loss by its own row losses in 64 bits along a direction of (x, e), at two steps: the finer central difference is off by a
    third of what the two differ by."""
    rows, d, vocab = 24, 64, 304
    x, e, target = inputs(dtype, rows, d, vocab, 10)
    live = int((target >= 0).sum())
    _, dx, de = call(dtype, x, e, target, 1.0 / live)
    g = generator(77)
    vx, ve = normal((rows, d), torch.float64, g), normal((vocab, d), torch.float64, g, 0.1)

    def f(t):
        xx, ee = x.double() + t * vx, e.double() + t * ve
        if dtype == zi.FP32:                                     # the call's own losses, at parameters of its type
            ee32 = ee.float()
            return call(dtype, xx, ee32, target, 1.0)[0].sum() / live
        l = xx @ ee.t()
        at = target.clamp(min=0).long()[:, None]
        return torch.where(target >= 0, torch.logsumexp(l, 1) - l.gather(1, at).squeeze(1), 0.0).sum() / live

    step = 2.0**-6
    coarse, fine = ((f(s) - f(-s)) / (2 * s) for s in (step, step / 2))
    got = (dx.double() * vx).sum() + (de.double() * ve).sum()
    # 16-bit: the gradient's own rounding and its probabilities', two independent half steps a term; fp32: the parameters the
    # losses were taken at are off by 2^-24 of 0.05 + step ve, a loss by as much of its slope, and that over the step
    h = half(act_dtype(dtype)) if dtype != zi.FP32 else 2.0**-24
    terms = torch.sqrt((dx.double() * vx).square().sum() + (de.double() * ve).square().sum())
    off = 7 * 1.5 * h * terms
    if dtype == zi.FP32:
        off = off + 7 * 2.0**-24 * (e.abs().max().double() + step * ve.abs().max()) * torch.sqrt(de.double().square().sum()) / step
    assert (got - fine).abs() <= (coarse - fine).abs() + off


@pytest.mark.parametrize("rows,d,vocab", [(6, 520, 1 << 22), (1 << 20, 2056, 16)])
def test_more_bytes_than_32_bits_count(rows, d, vocab):
    g = generator(51)
    x = torch.empty((rows, d), dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g)
    e = torch.empty((vocab, d), dtype=torch.bfloat16, device=DEV).normal_(0.0, 0.05, generator=g)
    target = torch.randint(0, vocab, (rows,), device=DEV, generator=g).to(torch.int32)
    target[rows // 2], target[rows - 1], target[0] = -1, vocab - 1, (1 << 31) // d % vocab
    words = slice(None)
    if vocab > 1 << 20:
        middle = (1 << 30) // d                                     # its bytes pass 2^31 there, and 2^32 near the end
        words = torch.cat([torch.arange(a, b, device=DEV) for a, b in ((0, 1000), (middle - 1000, middle + 1000), (2 * middle - 1000, vocab))])
    check(zi.BF16, x, e, target, 1.0 / rows, call(zi.BF16, x, e, target, 1.0 / rows), words)


TILES = [
    ("logits", (64, 64), 30, 136, 520), ("logits", (128, 128), 2049, 320, 1000), ("logits", (192, 128), 1048, 200, 3000), ("logits", (256, 128), 1000, 136, 4104),
    ("logits", (256, 192), 513, 136, 12000), ("logits", (256, 256), 3000, 512, 4104),
    ("de", (64, 64), 30, 136, 520), ("de", (128, 128), 257, 768, 3000), ("de", (192, 128), 200, 768, 4104), ("de", (256, 128), 131, 1024, 4104),
    ("de", (256, 192), 131, 136, 33000), ("de", (256, 256), 131, 200, 33000),
    ("dx", (64, 64), 30, 136, 520), ("dx", (128, 128), 1048, 1024, 1000), ("dx", (192, 128), 2049, 2048, 520), ("dx", (256, 128), 4096, 1536, 520),
    ("dx", (256, 192), 4096, 1536, 3000), ("dx", (256, 256), 2049, 2048, 6824),
]


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("product,tile,rows,d,vocab", TILES)
def test_every_tile(dtype, product, tile, rows, d, vocab):
    """Every product in every tile shape, at a size that takes it, and with ends that fill no tile."""
    assert zo_amd.zo_kernel_lmhead_grad_plan(rows, d, vocab)[product] == tile
    for r, v in ((rows, vocab), (rows - 3, vocab - 8)):
        x, e, target = inputs(dtype, r, d, v, 21)
        check(dtype, x, e, target, 0.03125, call(dtype, x, e, target, 0.03125))


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("rows,d,vocab,slabs", [(100, 512, 20000, 20), (300, 64, 8192, 5), (65, 72, 50272, 13), (512, 8, 64, 8), (4000, 8, 64, 63), (64, 2048, 50272, 99)])
def test_small_tiles_together_and_apart(dtype, rows, d, vocab, slabs):
    """de and dx in 64 x 64 tiles: one launch up to 512 rows and shares of 64 slabs, two beyond."""
    p = zo_amd.zo_kernel_lmhead_grad_plan(rows, d, vocab)
    assert p["de"] == p["dx"] == (64, 64) and p["de_words"] == vocab
    assert max(-(-(-(-vocab // 64)) // p["shares"]), -(-rows // 64)) == slabs
    for r, v in ((rows, vocab), (rows - 3, vocab - 8)):
        x, e, target = inputs(dtype, r, d, v, 24)
        scale = min(0.03125, 1e3 / float(x.abs().max()))
        check(dtype, x, e, target, scale, call(dtype, x, e, target, scale))


@pytest.mark.parametrize("dtype,rows,d,vocab,words,rest", [
    (zi.BF16, 520, 648, 50272, 43520, (192, 128)), (zi.FP16, 520, 968, 20000, 16384, (128, 128)), (zi.BF16, 1024, 392, 33000, 32768, (64, 64)),
    (zi.FP16, 1024, 520, 50272, 43520, (192, 128)), (zi.BF16, 1024, 1032, 33000, 26112, (256, 128)), (zi.FP16, 2048, 264, 33000, 32768, (64, 64)),
    (zi.BF16, 2048, 648, 33000, 21760, (256, 192))])
def test_words_behind_whole_rounds(dtype, rows, d, vocab, words, rest):
    """de's last words in a launch and tiles of their own."""
    p = zo_amd.zo_kernel_lmhead_grad_plan(rows, d, vocab)
    assert (p["de_words"], p["de_rest"]) == (words, rest)
    for r, v in ((rows, vocab), (rows - 3, vocab - 8)):
        x, e, target = inputs(dtype, r, d, v, 23)
        target[0], target[1], target[2] = words - 1, words, v - 1
        check(dtype, x, e, target, 0.03125, call(dtype, x, e, target, 0.03125))


@pytest.mark.parametrize("rows,d,vocab", [(16, 768, 9000), (40, 512, 20000), (131, 2048, 12000), (5, 64, 50272)])
def test_shares_of_the_vocabulary(rows, d, vocab):
    """Few rows: the contraction over the words is cut into shares, some of which reach past the last word."""
    assert zo_amd.zo_kernel_lmhead_grad_plan(rows, d, vocab)["shares"] > 1
    for v in (vocab, vocab - 64, vocab - 72):
        x, e, target = inputs(zi.BF16, rows, d, v, 22)
        target[-1] = v - 1                                       # the last word counts
        check(zi.BF16, x, e, target, 1.0, call(zi.BF16, x, e, target, 1.0))


@pytest.mark.parametrize("dtype,rows,d,vocab", [(zi.BF16, 8300, 64, 66008), (zi.FP16, 8300, 64, 66008), (zi.BF16, 8300, 264, 66008), (zi.FP16, 8300, 576, 66008),
                                                (zi.BF16, 140, 320, 1 << 22)])
def test_sixteen_bits_in_pieces(dtype, rows, d, vocab):
    """More words than the workspace holds probabilities for at once (2^30 bytes): the logits are worked again for each piece, and the later
    pieces' share of dx is added to the first's."""
    assert zo_amd.zo_kernel_lmhead_grad_plan(rows, d, vocab)["pieces"] > 1
    x, e, target = inputs(dtype, rows, d, vocab, 12)
    check(dtype, x, e, target, 1.0 / 64, call(dtype, x, e, target, 1.0 / 64))


# words of a strip's last, partly filled part and of a strip's halves: a strip of 32 to 128 words is held by two halves of a wavefront, in turns of four
PARTS = {"first of the last eight": lambda v: torch.arange(v - 8, v - 4), "last four": lambda v: torch.arange(v - 4, v), "last eight": lambda v: torch.arange(v - 8, v),
         "last one": lambda v: torch.arange(v - 1, v), "last strip": lambda v: torch.arange((v - 1) // 128 * 128, v),
         "one half's": lambda v: torch.arange(256, 384)[(torch.arange(128) >> 2) % 2 == 0], "other half's": lambda v: torch.arange(256, 384)[(torch.arange(128) >> 2) % 2 == 1]}


@pytest.mark.parametrize("dtype,rows,d,vocab", [
    (zi.BF16, 10, 64, 520), (zi.FP16, 10, 64, 1000), (zi.BF16, 2049, 320, 1000), (zi.FP16, 1048, 200, 3000), (zi.BF16, 1000, 136, 4104), (zi.FP16, 513, 136, 12008),
    (zi.BF16, 3000, 512, 4104), (zi.BF16, 8300, 64, 66056), (zi.FP16, 8300, 264, 66008), (zi.FP32, 10, 64, 504), (zi.FP32, 100, 16, 6000), (zi.FP32, 2100, 16, 17000)])
def test_a_few_words_that_are_nan(dtype, rows, d, vocab):
    """Fewer NaN words than a strip has: every row that counts is NaN throughout, as the formula has it."""
    x, e, target = inputs(dtype, rows, d, vocab, 17)
    live = target >= 0
    for name, words in PARTS.items():
        bent = e.clone()
        bent[words(vocab).to(DEV)] = float("nan")
        loss, dx, de = call(dtype, x, bent, target, 1.0)
        assert torch.isnan(loss[live]).all() and (loss[~live] == 0).all(), name
        assert torch.isnan(dx[live]).all() and torch.isnan(de).all(), name


@pytest.mark.parametrize("dtype,rows,d,vocab", [(zi.BF16, 40, 64, 1000), (zi.FP16, 600, 128, 4096), (zi.BF16, 8300, 64, 66008), (zi.FP16, 8300, 64, 66008),
                                                (zi.FP32, 100, 16, 6000), (zi.FP32, 2100, 16, 17000)])
def test_no_row_counts_and_words_are_nan(dtype, rows, d, vocab):
    """G is 0 throughout: no word gets a gradient, whatever words hold."""
    x, e, target = inputs(dtype, rows, d, vocab, 19)
    e[7], e[vocab - 1], e[vocab // 2] = float("nan"), float("inf"), float("nan")
    target[:] = -1
    loss, _, de = call(dtype, x, e, target, 1.0)
    assert (loss == 0).all() and (de == 0).all()


@pytest.mark.parametrize("words", [slice(0, 15936), slice(15936, 17000), slice(0, 9000)])
def test_fp32_pieces_of_no_probability(words):
    """A piece of the vocabulary (15936 words of 2100 rows) whose logits are all minus infinity, while those of the other are about -1000."""
    rows, d, vocab = 2100, 16, 17000
    x, e, target = inputs(zi.FP32, rows, d, vocab, 18, lean=0.0)
    x[:, 0], x[:, 1], e[:, 1] = 1.0, 1000.0, -1.0
    e[words, 0] = -float("inf")
    lost = torch.zeros(vocab, dtype=torch.bool, device=DEV)
    lost[words] = True
    rest = torch.nonzero(~lost).squeeze(1)
    live = target >= 0
    target[live] = rest[target[live].long() % len(rest)].int()
    loss, _, de = call(zi.FP32, x, e, target, 1.0)
    # over the words that are left: a sum of d products and of len(rest) exponentials in fp64, values of 1000
    logits = x @ e[rest].double().t()
    place = (torch.cumsum(~lost, 0) - 1).clamp(min=0)             # (a row that does not count has none)
    hit = logits.gather(1, place[target.clamp(min=0).long()][:, None])
    lse = torch.logsumexp(logits, 1, keepdim=True)
    want = torch.where(live, (lse - hit).squeeze(1), 0.0)
    assert ((loss - want).abs() <= 2.0**-50 * 1000 * (16 + d)).all()
    assert (de[lost] == 0).all() and torch.isfinite(de).all()


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("rows", [12, 384])
@pytest.mark.parametrize("size", [1.5, 2.0, 2.5, 3.0])
def test_small_probabilities(dtype, rows, size):
    """Rows sure of one word, the others' probabilities from about 2^-20 to 2^-45: in fp16 G holds those below 2^-29 as subnormal numbers, and
    most words' gradient is made of them alone."""
    d, vocab = 128, 776
    x, e, target = inputs(dtype, rows, d, vocab, 20, std=0.3)
    word = torch.arange(rows, device=DEV) % 12 * 3
    x = (e[word].double() * size).to(act_dtype(dtype))
    target = torch.where(target >= 0, word, -1).int()
    scale = 2.0**24
    check(dtype, x, e, target, scale / rows, call(dtype, x, e, target, scale / rows))
