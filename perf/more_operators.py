"""Performance cases of what carries the exact gradient on from the last module: the linear layer's backward pass (bias, ReLU and
residual as its forward call has them), the causal attention's, and the AdamW step over many tensors, its moments held in 32 bits or in 8.

A program that trains the last decoder blocks, the final LayerNorm and the head by their gradient makes these calls between the
LayerNorm's backward pass and the next forward pass.  bf16 and fp16 parameters go with 16-bit activations and an fp32 residual stream, fp32
parameters with fp64 activations, as everywhere in this library; moments are fp32 numbers, or e4m3 ones in blocks of 256 with a scale each.
"""
import ctypes
import math

import torch

own = False

DEV = "cuda:0"
VOCAB = 50272
CODES = {"fp32": 0, "bf16": 1, "fp16": 2}
PARAM = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
ACT = {"fp32": torch.float64, "bf16": torch.bfloat16, "fp16": torch.float16}
RESID = {"fp32": torch.float64, "bf16": torch.float32, "fp16": torch.float32}
BLOCK = 256                                 # elements that share a scale
LR, BETA1, BETA2, EPS, DECAY, MAX_NORM = 1e-4, 0.9, 0.95, 1e-8, 0.1, 1.0


def listed():
    return [
        # Up-projection of a tiny fp32 model (fp64 activations), 2 x 32 tokens: all latency.
        dict(name="linear_tiny_fp32", kind="linear", rows=64, n=256, k=64, epilogue=1, relu_x=False, dtype="fp32"),
        # Up-projection of the 1.3b shape with its ReLU for four short prompts: W read once and its gradient written.
        dict(name="linear_few_rows", kind="linear", rows=20, n=8192, k=2048, epilogue=1, relu_x=False, dtype="bf16"),
        # Attention's output projection, 125m shape, 16 x 512 tokens: few output tiles, a long sum over the rows.
        dict(name="linear_125m_out", kind="linear", rows=8192, n=768, k=768, epilogue=2, relu_x=False, dtype="bf16"),
        # Down-projection onto the residual stream behind a ReLU, eight prompts of 131 tokens, 1.3b shape, fp16 with a scaled loss: ragged rows.
        dict(name="linear_1.3b_ragged", kind="linear", rows=1048, n=2048, k=8192, epilogue=2, relu_x=True, dtype="fp16"),
        # Up-projection of the 13B shape, 4 x 2048 tokens, its ReLU taken back by the layer behind it: 3.4 TFLOP.
        dict(name="linear_13b_up", kind="linear", rows=8192, n=20480, k=5120, epilogue=0, relu_x=False, dtype="bf16"),
        # Attention of a tiny fp32 model, 2 x 32 tokens, 4 heads of 16.
        dict(name="attention_tiny_fp32", kind="attention", n_seq=2, seq=32, heads=4, d_head=16, dtype="fp32"),
        # An ordinary batch of the 125m shape, 16 x 512 tokens.
        dict(name="attention_125m", kind="attention", n_seq=16, seq=512, heads=12, d_head=64, dtype="bf16"),
        # Eight prompts of 131 tokens, heads of 80 channels, fp16 with a scaled loss: ragged tiles.
        dict(name="attention_ragged", kind="attention", n_seq=8, seq=131, heads=32, d_head=80, dtype="fp16"),
        # 4 x 2048 tokens of the 13B shape.
        dict(name="attention_13b", kind="attention", n_seq=4, seq=2048, heads=40, d_head=128, dtype="bf16"),
        # Every tensor of a tiny fp32 model, 36 of them.
        dict(name="adamw_tiny_fp32", kind="adamw", numels=_model(2, 64, 256, 512, 32), bits=32, stochastic=False, clip=True, dtype="fp32"),
        # The tied embedding, the final LayerNorm and the last feed-forward layer, 125m shape, fp32 moments.
        dict(name="adamw_125m_module", kind="adamw", numels=_module(768, 4 * 768, VOCAB), bits=32, stochastic=False, clip=True, dtype="bf16"),
        # The same tensors as 125m_module's of the 1.3b shape, moments in 8 bits, weights without a master copy rounded stochastically.
        dict(name="adamw_1.3b_module_8bit", kind="adamw", numels=_module(2048, 8192, VOCAB), bits=8, stochastic=True, clip=True, dtype="bf16"),
    ]


def _text(numels):
    return " ".join(str(n) for n in numels)


def _model(layers, d, ffn, vocab, max_pos):
    block = [d, d, d * d, d, d * d, d, d * d, d, d * d, d, d, d, ffn * d, ffn, d * ffn, d]
    return _text([vocab * d, max_pos * d] + block * layers + [d, d])


def _module(d, ffn, vocab):
    return _text([vocab * d, d, d, ffn * d, ffn, d * ffn, d, d, d])


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    half = rng.choice(["bf16", "bf16", "fp16"])
    kind = rng.choice(["linear", "linear", "attention", "attention", "adamw"])
    if kind == "attention":
        if rng.random() < 0.15:
            return dict(kind=kind, n_seq=rng.randint(1, 8), seq=_log(rng, 1, 128), heads=rng.randint(1, 8), d_head=4 * rng.randint(1, 16), dtype="fp32")
        heads, d_head, seq = rng.randint(4, 40), rng.choice([64, 64, 80, 96, 112, 128, 128]), _log(rng, 1, 4096)
        n_seq = _log(rng, 1, max(1, min(32, 4 * 2048 * 2048 * 40 * 128 // (seq * seq * heads * d_head))))
        return dict(kind=kind, n_seq=n_seq, seq=seq, heads=heads, d_head=d_head, dtype=half)
    if kind == "linear":
        epilogue = rng.choice([0, 0, 1, 2, 2, 3])
        relu_x = rng.random() < 0.4
        if rng.random() < 0.15:
            return dict(kind="linear", rows=_log(rng, 1, 512), n=_log(rng, 16, 512), k=_log(rng, 16, 512), epilogue=epilogue, relu_x=relu_x, dtype="fp32")
        step = 8 if rng.random() < 0.3 else 64
        n, k = step * _log(rng, 512 // step, 20480 // step), step * _log(rng, 512 // step, 20480 // step)
        return dict(kind="linear", rows=_log(rng, 1, min(8192, max(64, 8192 * 20480 * 5120 // (n * k)))), n=n, k=k, epilogue=epilogue, relu_x=relu_x, dtype=half)
    dtype = rng.choice([half, half, "fp32"])
    bits = rng.choice([8, 32])
    if rng.random() < 0.5:
        d = 64 * _log(rng, 1, 24)
        numels = _module(d, 4 * d, 8 * _log(rng, 64, 6284))
    else:
        numels = _text([_log(rng, 1, 3_000_000) for _ in range(_log(rng, 1, 30))])
    return dict(kind="adamw", numels=numels, bits=bits, stochastic=dtype == "bf16" and rng.random() < 0.4, clip=rng.random() < 0.7, dtype=dtype)


def _normal(shape, dtype, g, std=1.0):
    return torch.empty(shape, device=DEV, dtype=torch.float32).normal_(0.0, std, generator=g).to(dtype)


def _coefficients(s):
    """What a step's scalars come to, each worked in 64 bits and rounded to fp32 once, as the call does."""
    f = lambda v: float(torch.tensor(v, dtype=torch.float32))  # noqa: E731
    t = s["step"]
    return dict(b1=f(BETA1), c1=f(1.0 - BETA1), b2=f(BETA2), c2=f(1.0 - BETA2), decay=f(LR * DECAY), rate=f(LR / (1.0 - BETA1 ** t)),
                root=f(1.0 / math.sqrt(1.0 - BETA2 ** t)), eps=f(EPS))


def _held(x, low):
    """Rows of 256 fp32 numbers as e4m3 ones and a scale; `low`: what is above zero stays above it."""
    scale = x.abs().amax(1, keepdim=True) * float(torch.tensor(1.0 / 448.0, dtype=torch.float32))
    scale = torch.where(scale < 2.0 ** -126, 0.0, scale)
    y = x * torch.where(scale > 0, torch.reciprocal(scale), 0.0)
    y = torch.where((x > 0) & (scale > 0), y.clamp(min=2.0 ** -9), y) if low else y
    return y.to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = case["dtype"]
    s = dict(case)
    if case["kind"] == "linear":
        rows, n, k = case["rows"], case["n"], case["k"]
        # normalised rows, or a ReLU's output; a mean loss's gradients, scaled up as fp16 training does
        x = _normal((rows, k), torch.float32, g)
        s["x"] = (x.clamp(min=0) if case["relu_x"] else x).to(ACT[dt])
        s["w"] = _normal((n, k), PARAM[dt], g, 0.02)
        s["y"] = _normal((rows, n), torch.float32, g).clamp(min=0).to(ACT[dt]) if case["epilogue"] == 1 else None
        size = (64.0 if dt == "fp16" else 1.0) / rows
        s["dy"] = (_normal((rows, n), torch.float32, g, size) * (0.5 + torch.rand((rows, 1), device=DEV, generator=g))).to(
            (RESID if case["epilogue"] >= 2 else ACT)[dt])
        s["dx"] = torch.empty((rows, k), device=DEV, dtype=ACT[dt])
        s["dw"] = torch.empty((n, k), device=DEV, dtype=PARAM[dt])
        s["db"] = torch.empty(n, device=DEV, dtype=PARAM[dt]) if case["epilogue"] != 3 else None
        return s
    if case["kind"] == "attention":
        rows, d = case["n_seq"] * case["seq"], case["heads"] * case["d_head"]
        s["qkv"] = _normal((rows, 3 * d), ACT[dt], g)
        s["out"] = _merge(_probabilities(s) @ _heads(s, s["qkv"], 2).to(RESID[dt]), s).to(ACT[dt])            # the forward call's
        s["dout"] = _normal((rows, d), ACT[dt], g, (64.0 if dt == "fp16" else 1.0) / rows)
        s["dqkv"] = torch.empty((rows, 3 * d), device=DEV, dtype=ACT[dt])
        return s
    # tensors side by side, each on a block's boundary, so that the plain form takes all of them at once; zeros behind their ends
    numels = [int(n) for n in case["numels"].split()]
    blocks = [(n + BLOCK - 1) // BLOCK for n in numels]
    total = sum(blocks)
    counts = torch.tensor(blocks, device=DEV)
    s["tensor"] = torch.repeat_interleave(torch.arange(len(numels), device=DEV), counts)                 # of a block
    s["within"] = torch.arange(total, device=DEV) - (torch.cumsum(counts, 0) - counts)[s["tensor"]]      # its number in the tensor
    left = torch.tensor(numels, device=DEV)[s["tensor"]] - BLOCK * s["within"]
    real = torch.arange(BLOCK, device=DEV)[None] < left[:, None]
    s["param"] = torch.where(real, _normal((total, BLOCK), torch.float32, g, 0.02), 0.0).to(PARAM[dt])
    # gradients and moments of earlier ones: rows of unlike size, as embeddings of rare and common words have
    size = torch.exp(torch.randn((total, 1), device=DEV, generator=g)) / math.sqrt(sum(numels))
    grad = torch.where(real, _normal((total, BLOCK), torch.float32, g) * size, 0.0)
    m = torch.where(real, _normal((total, BLOCK), torch.float32, g, 0.3) * size, 0.0)
    r = torch.where(real, (0.5 + torch.rand((total, BLOCK), device=DEV, generator=g)) * size, 0.0)
    s["grad"] = grad.to(PARAM[dt])
    if case["bits"] == 32:
        s["state"] = torch.cat([m, r * r], 1).contiguous()
        s["m"], s["v"] = s["state"][:, :BLOCK], s["state"][:, BLOCK:]
        each = 4 * 2 * BLOCK
    else:
        each = 2 * BLOCK + 8
        s["state"] = torch.empty((total, each), device=DEV, dtype=torch.uint8)
        s["m"], s["v"] = (s["state"][:, at:at + BLOCK].view(torch.float8_e4m3fn) for at in (0, BLOCK))
        s["scale"] = s["state"].view(torch.float32)[:, BLOCK // 2:]
        for held, x, at in ((s["m"], m, 0), (s["v"], r, 1)):
            y, scale = _held(x, at == 1)
            held.view(torch.uint8).copy_(y.view(torch.uint8))
            s["scale"][:, at:at + 1] = scale
    s["step"], s["seed"] = 100, seed * 0x9E3779B97F4A7C15 % 2 ** 64
    norm = s["grad"].double().square().sum().sqrt()
    s["norm"] = torch.stack([norm, torch.clamp(MAX_NORM / norm, max=1.0)]) if case["clip"] else None      # as the clipping call leaves them
    firsts = [sum(blocks[:i]) for i in range(len(blocks))]
    tables = [(s["param"], BLOCK * PARAM[dt].itemsize), (s["grad"], BLOCK * PARAM[dt].itemsize), (s["state"], each)]
    s["tables"] = [(ctypes.c_void_p * len(numels))(*[t.data_ptr() + f * b for f in firsts]) for t, b in tables]
    s["numel"] = (ctypes.c_uint64 * len(numels))(*numels)
    return s


def _heads(s, x, part):
    """Queries (0), keys (1) or values (2) of [rows, 3 d], or all of [rows, d], as [sequences and heads, positions, channels]."""
    x = x.view(s["n_seq"], s["seq"], -1, s["heads"], s["d_head"])[:, :, part]
    return x.permute(0, 2, 1, 3).reshape(-1, s["seq"], s["d_head"])


def _merge(x, s):
    return x.view(s["n_seq"], s["heads"], s["seq"], s["d_head"]).permute(0, 2, 1, 3).reshape(s["n_seq"] * s["seq"], -1)


def _probabilities(s):
    q, k = (_heads(s, s["qkv"], part).to(RESID[s["dtype"]]) for part in (0, 1))
    score = (q @ k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(s["d_head"]))
    score.masked_fill_(torch.ones(s["seq"], s["seq"], device=DEV, dtype=torch.bool).triu_(1), -math.inf)
    score = score.sub_(score.amax(2, keepdim=True)).exp_()
    return score.div_(score.sum(2, keepdim=True))


def _outputs(s):
    return [s["param"], s["m"], s["v"]] + ([s["scale"]] if s["bits"] == 8 else [])


def _run_own(s):
    import paper_2507_03211_amd as zo
    code, stream = CODES[s["dtype"]], torch.cuda.current_stream()
    if s["kind"] == "linear":
        if "scratch" not in s:              # a workspace the program keeps
            s["scratch"] = torch.empty(zo.zo_kernel_linear_grad_scratch_bytes(code, s["rows"], s["n"], s["k"], s["epilogue"]), device=DEV, dtype=torch.uint8)
        zo.zo_kernel_linear_grad(s["x"], s["w"], s["y"], s["dy"], s["dx"], s["dw"], s["db"], s["scratch"], code, s["rows"], s["n"], s["k"], s["epilogue"],
                                 s["relu_x"], stream)
        return [s["dx"], s["dw"]] + ([s["db"]] if s["db"] is not None else [])
    if s["kind"] == "attention":
        if "scratch" not in s:
            s["scratch"] = torch.empty(zo.zo_kernel_attention_grad_scratch_bytes(code, s["n_seq"], s["seq"], s["heads"], s["d_head"]), device=DEV, dtype=torch.uint8)
        zo.zo_kernel_attention_grad(s["qkv"], s["out"], s["dout"], s["dqkv"], s["scratch"], code, s["n_seq"], s["seq"], s["heads"], s["d_head"], stream)
        return s["dqkv"]
    zo.zo_kernel_adamw(*s["tables"], s["numel"], len(s["numel"]), code, s["bits"], LR, BETA1, BETA2, EPS, DECAY, s["step"], s["norm"], MAX_NORM,
                       zo.ZO_ROUND_STOCHASTIC if s["stochastic"] else zo.ZO_ROUND_NEAREST, s["seed"], stream)
    return _outputs(s)


def _words(s):
    """A random 32-bit number for each element: word i % 4 of Philox4x32-10 at counter (i / 4, tensor, 3), 64-bit key = the seed."""
    low = 0xFFFFFFFF
    j = (BLOCK // 4 * s["within"])[:, None] + torch.arange(BLOCK // 4, device=DEV)[None]
    c0, c1, c2, c3 = j & low, j >> 32, s["tensor"][:, None].expand_as(j), torch.full_like(j, 3)
    k0, k1 = s["seed"] & low, s["seed"] >> 32

    def both(a, m):                         # high and low half of a 64-bit product
        first = a * (m & 0xFFFF)
        second = a * (m >> 16) + (first >> 16)
        return second >> 16, (second & 0xFFFF) << 16 | first & 0xFFFF
    for _ in range(10):
        h0, l0 = both(c0, 0xD2511F53)
        h1, l1 = both(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack([c0, c1, c2, c3], 2).reshape(-1, BLOCK)


def _stored(p, s):
    """fp32 numbers in the parameters' type."""
    if not s["stochastic"]:
        return p.to(PARAM[s["dtype"]])
    bits = p.view(torch.int32).long()       # bf16: the upper half of fp32, one step further out where the lower half says so
    up = (_words(s) >> 8) < (bits & 0xFFFF) << 8
    return ((bits >> 16) + up).to(torch.int16).view(torch.bfloat16)


def run(s):
    if own:
        return _run_own(s)
    dt = s["dtype"]
    acc = RESID[dt]
    if s["kind"] == "linear":
        grad = s["dy"].to(acc)
        if s["epilogue"] == 1:
            grad = torch.where(s["y"] > 0, grad, 0.0)
        dx = grad @ s["w"].to(acc)
        if s["relu_x"]:
            dx = torch.where(s["x"] > 0, dx, 0.0)
        out = [dx.to(ACT[dt]), (grad.t() @ s["x"].to(acc)).to(PARAM[dt])]
        return out + ([grad.sum(0).to(PARAM[dt])] if s["db"] is not None else [])
    if s["kind"] == "attention":
        q, k, v = (_heads(s, s["qkv"], part).to(acc) for part in range(3))
        p, dout = _probabilities(s), _heads(s, s["dout"], 0).to(acc)
        dv = p.transpose(1, 2).contiguous() @ dout
        ds = dout @ v.transpose(1, 2).contiguous()
        ds.sub_((dout * (p @ v)).sum(2, keepdim=True)).mul_(p).mul_(1.0 / math.sqrt(s["d_head"]))
        return torch.cat([_merge(t, s) for t in (ds @ k, ds.transpose(1, 2).contiguous() @ q, dv)], 1).to(ACT[dt])
    c = _coefficients(s)
    grad, p = s["grad"].float(), s["param"].float()
    if s["clip"]:
        grad = grad * torch.where(s["norm"][0] > MAX_NORM, MAX_NORM / s["norm"][0], 1.0).float()
    m, v = s["m"].float(), s["v"].float()
    if s["bits"] == 8:
        m, v = m * s["scale"][:, :1], v * s["scale"][:, 1:]
        v = v * v
    m = m * c["b1"] + grad * c["c1"]
    v = v * c["b2"] + grad * c["c2"] * grad
    r = torch.sqrt(v)
    p = p - (p * c["decay"] + m * c["rate"] / (r * c["root"] + c["eps"]))
    s["param"].copy_(_stored(p, s))
    if s["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return _outputs(s)
    for held, x, at in ((s["m"], m, 0), (s["v"], r, 1)):
        y, scale = _held(x, at == 1)
        held.view(torch.uint8).copy_(y.view(torch.uint8))
        s["scale"][:, at:at + 1] = scale
    return _outputs(s)


def work(case):
    param = PARAM[case["dtype"]].itemsize
    if case["kind"] == "linear":
        act, resid = ACT[case["dtype"]].itemsize, RESID[case["dtype"]].itemsize
        rows, n, k = case["rows"], case["n"], case["k"]
        dy = {0: act, 1: 2 * act, 2: resid, 3: resid}[case["epilogue"]]          # and y, for its sign
        return {"bytes": 2 * rows * k * act + 2 * n * k * param + rows * n * dy + (n * param if case["epilogue"] != 3 else 0), "flops": 4 * rows * n * k}
    if case["kind"] == "attention":
        seq, n = case["seq"], case["n_seq"] * case["heads"]
        # qkv, out and dout read, dqkv written; S, dP, dQ, dK, dV over the half that is not masked
        return {"bytes": 8 * n * seq * case["d_head"] * ACT[case["dtype"]].itemsize, "flops": 5 * n * seq * (seq + 1) * case["d_head"]}
    n = sum(int(t) for t in case["numels"].split())
    return {"bytes": n * 3 * param + n * (16 if case["bits"] == 32 else 4) + (16 * n // BLOCK if case["bits"] == 8 else 0), "flops": 16 * n}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "linear":
        live = s["dy"].double()
        if s["y"] is not None:
            live = live * (s["y"] > 0).double()
        dx = torch.matmul(live, s["w"].double())
        dw = torch.matmul(s["x"].double().t(), live).t()
        if case["relu_x"]:
            dx = dx * (s["x"] > 0).double()
        return [dx, dw] + ([torch.ones(case["rows"], device=DEV, dtype=torch.float64) @ live] if s["db"] is not None else [])
    if case["kind"] == "attention":
        # a sequence and head at a time would take long: a few of them together, so that 64-bit scores stay small
        parts, scale = [], case["d_head"] ** -0.5
        seen = torch.ones(case["seq"], case["seq"], device=DEV, dtype=torch.bool).tril()
        qkv = s["qkv"].double().view(case["n_seq"], case["seq"], 3, case["heads"], case["d_head"])
        dout = s["dout"].double().view(case["n_seq"], case["seq"], case["heads"], case["d_head"])
        for i in range(case["n_seq"]):
            q, k, v = (qkv[i, :, j].transpose(0, 1).contiguous() for j in range(3))
            do = dout[i].transpose(0, 1).contiguous()
            logp = torch.where(seen, torch.matmul(q, k.mT.contiguous()) * scale, -math.inf)
            p = torch.exp(logp - torch.logsumexp(logp, 2, keepdim=True))
            dp = torch.matmul(do, v.mT.contiguous())
            ds = p * dp - p * (p * dp).sum(2, keepdim=True)
            grads = [torch.matmul(ds, k) * scale, torch.matmul(ds.mT.contiguous(), q) * scale, torch.matmul(p.mT.contiguous(), do)]
            parts.append(torch.stack(grads, 0).permute(2, 0, 1, 3).reshape(case["seq"], -1))
        return torch.cat(parts, 0)
    t = s["step"]
    grad, p = s["grad"].double(), s["param"].double()
    if case["clip"]:
        grad = grad * min(1.0, MAX_NORM / float(s["norm"][0]))
    if case["bits"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        scale = s["scale"].double()
        m, v = s["m"].double() * scale[:, :1], (s["v"].double() * scale[:, 1:]).square()
    m = m + (1.0 - BETA1) * (grad - m)
    v = v + (1.0 - BETA2) * (grad.square() - v)
    step = LR * (m / (1.0 - BETA1 ** t)) / (torch.sqrt(v / (1.0 - BETA2 ** t)) + EPS)
    p = (1.0 - LR * DECAY) * p - step
    # (stochastic rounding is to either neighbour: the value itself stands between)
    if case["bits"] == 32:
        return [p, m, v]
    r = v.sqrt()
    tops = [x.abs().amax(1, keepdim=True) / 448.0 for x in (m, r)]
    held = []
    for x, top in zip((m, r), tops):
        y = torch.where(top > 0, x / top, 0.0)
        unit = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)           # of e4m3: three bits behind the first, 2^-9 at the least
        held.append(torch.round(y / unit) * unit)
    held[1] = torch.where((r > 0) & (held[1] == 0), 2.0 ** -9, held[1])
    return [p, held[0], held[1], torch.cat(tops, 1)]
