"""Performance cases of the last module's gradient: LayerNorm with its statistics and its backward pass, the tied LM head's
cross entropy with its gradient, and the global norm and clipping of many gradients.

A program that trains the final LayerNorm and the head by their exact gradient (the blocks by zeroth-order steps), or that
compares a step's g with z . grad L, makes these calls.  bf16 and fp16 parameters go with 16-bit activations and an fp32
residual stream, fp32 parameters with fp64 activations, as everywhere in this library.
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
EPS = float(torch.tensor(1e-5, dtype=torch.float32))      # calls take it, and the loss's scale, as an fp32 number


def listed():
    return [
        # The final LayerNorm of eight label positions: a call that is all latency.
        dict(name="norm_few", kind="norm", rows=8, d=768, dtype="fp16"),
        # The final LayerNorm of an ordinary batch of the 125m shape, 16 x 512 tokens.
        dict(name="norm_125m", kind="norm", rows=8192, d=768, dtype="bf16"),
        # Backward of a tiny fp32 model's LayerNorm (fp64 activations), 2 x 32 tokens: launches count.
        dict(name="norm_grad_tiny_fp32", kind="norm_grad", rows=64, d=64, dtype="fp32"),
        # A ragged batch over rows whose length is no power of two.
        dict(name="norm_grad_ragged", kind="norm_grad", rows=1003, d=1100, dtype="fp16"),
        # 4 x 2048 tokens of the 13B shape: a stream of 420 MB.
        dict(name="norm_grad_13b", kind="norm_grad", rows=8192, d=5120, dtype="bf16"),
        # Head of a tiny fp32 model, 2 x 32 tokens over 512 words, in fp64.
        dict(name="head_tiny_fp32", kind="head", batch=2, seq=32, d=64, vocab=512, dtype="fp32"),
        # Four short prompts against the real vocabulary: few rows, E read and its gradient written.
        dict(name="head_few_rows", kind="head", batch=4, seq=5, d=768, vocab=VOCAB, dtype="bf16"),
        # An ordinary batch of the 125m shape, 16 x 512 tokens: short contractions, exponentials count.
        dict(name="head_125m", kind="head", batch=16, seq=512, d=768, vocab=VOCAB, dtype="bf16"),
        # Eight prompts of 131 tokens, 1.3b shape, fp16 with a scaled loss: ragged rows.
        dict(name="head_1.3b_ragged", kind="head", batch=8, seq=131, d=2048, vocab=VOCAB, dtype="fp16"),
        # 4 x 2048 tokens of the 13B shape: 12.7 TFLOP of products.
        dict(name="head_13b", kind="head", batch=4, seq=2048, d=5120, vocab=VOCAB, dtype="bf16"),
        # Gradients of a tiny fp32 model: 36 small tensors.
        dict(name="clip_tiny_fp32", kind="clip", layers=2, d=64, ffn=256, vocab=512, max_pos=32, dtype="fp32"),
        # Gradients of every tensor of the 125m model, 196 of them, clipped into one bucket.
        dict(name="clip_125m", kind="clip", layers=12, d=768, ffn=4 * 768, vocab=VOCAB, max_pos=2048, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "norm_grad", "head", "head", "head", "clip"])
    half = rng.choice(["bf16", "bf16", "fp16"])
    if kind in ("norm", "norm_grad"):
        if rng.random() < 0.2:
            return dict(kind=kind, rows=_log(rng, 8, 2048), d=_log(rng, 64, 1024), dtype="fp32")
        d = _log(rng, 64, 12288) if rng.random() < 0.3 else 8 * _log(rng, 8, 1536)
        return dict(kind=kind, rows=_log(rng, 8, min(16384, 8192 * 5120 // d)), d=d, dtype=half)
    if kind == "head":
        if rng.random() < 0.15:
            return dict(kind=kind, batch=rng.randint(1, 4), seq=rng.randint(8, 64), d=16 * rng.randint(2, 16), vocab=8 * _log(rng, 32, 256),
                        dtype="fp32")
        d = 8 * _log(rng, 32, 640) if rng.random() < 0.3 else 64 * _log(rng, 4, 80)
        vocab = VOCAB if rng.random() < 0.7 else 8 * _log(rng, 250, 6284)
        batch = _log(rng, 1, 16)
        return dict(kind=kind, batch=batch, seq=_log(rng, 5, 8192 // batch), d=d, vocab=vocab, dtype=half)
    d = 64 * _log(rng, 2, 16)
    vocab = 8 * _log(rng, 64, 6284)
    layers = rng.randint(1, 12)
    if layers * 12 * d * d + vocab * d > 120_000_000:
        layers, vocab = 1, 8192
    return dict(kind=kind, layers=layers, d=d, ffn=4 * d, vocab=vocab, max_pos=rng.randint(32, 2048), dtype=rng.choice([half, "fp32"]))


def _normal(shape, dtype, g, std=1.0):
    return torch.empty(shape, device=DEV, dtype=torch.float32).normal_(0.0, std, generator=g).to(dtype)


def _numels(case):
    d, f = case["d"], case["ffn"]
    block = [d, d, d * d, d, d * d, d, d * d, d, d * d, d, d, d, f * d, f, d * f, d]
    return [case["vocab"] * d, case["max_pos"] * d] + block * case["layers"] + [d, d]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    kind, dt = case["kind"], case["dtype"]
    s = dict(case)
    if kind in ("norm", "norm_grad"):
        rows, d = case["rows"], case["d"]
        # a residual stream: rows of unlike size around unlike means, a few channels far larger than the others
        h = _normal((rows, d), RESID[dt], g) * (0.5 + 2.0 * torch.rand((rows, 1), device=DEV, generator=g)) + 0.3 * _normal((rows, 1), RESID[dt], g)
        h[:, torch.randint(0, d, (3,), device=DEV, generator=g)] *= 12.0
        s["resid"] = h.to(RESID[dt])
        s["gain"] = (1.0 + _normal((d,), torch.float32, g, 0.2)).to(PARAM[dt])
        if kind == "norm":
            s["bias"] = _normal((d,), PARAM[dt], g, 0.2)
            s["y"] = torch.empty((rows, d), device=DEV, dtype=ACT[dt])
            s["mean"], s["rstd"] = (torch.empty(rows, device=DEV, dtype=RESID[dt]) for _ in range(2))
        else:
            s["dy"] = _normal((rows, d), ACT[dt], g, 0.01)
            s["mean"] = s["resid"].double().mean(1).to(RESID[dt])
            s["rstd"] = (s["resid"].double().var(1, unbiased=False) + EPS).rsqrt().to(RESID[dt])
            s["dresid"] = torch.empty((rows, d), device=DEV, dtype=RESID[dt])
            s["dgain"], s["dbias"] = (torch.empty(d, device=DEV, dtype=PARAM[dt]) for _ in range(2))
    elif kind == "head":
        rows, d, vocab = case["batch"] * case["seq"], case["d"], case["vocab"]
        s["e"] = _normal((vocab, d), PARAM[dt], g, 0.02)
        target = torch.randint(0, vocab, (rows,), device=DEV, generator=g)
        # final-LayerNormed rows; the target's logit stands out by 0 to 16, as in a model that has learned some of its answers
        lean = 16.0 / (0.02 * 0.02 * d) * torch.rand((rows, 1), device=DEV, generator=g)
        s["x"] = (_normal((rows, d), torch.float32, g) + lean * s["e"][target].float()).to(ACT[dt])
        target.view(case["batch"], case["seq"])[:, -1] = -1          # the last position of a prompt has no next token
        s["target"] = target.to(torch.int32)
        # the mean over the positions that count; fp16 gradients are scaled up as fp16 training does
        s["scale"] = float(torch.tensor((16384.0 if dt == "fp16" else 1.0) / (case["batch"] * (case["seq"] - 1)), dtype=torch.float32))
        s["row_loss"] = torch.empty(rows, device=DEV, dtype=RESID[dt])
        s["dx"] = torch.empty((rows, d), device=DEV, dtype=ACT[dt])
        s["de"] = torch.empty((vocab, d), device=DEV, dtype=PARAM[dt])
    else:
        # every tensor's gradient in a buffer of its own, here side by side; clipped into a bucket of the same layout
        numels = _numels(case)
        step = 16 // PARAM[dt].itemsize
        firsts, total = [], 0
        for n in numels:
            firsts.append(total)
            total += (n + step - 1) // step * step
        flat = torch.empty(total, device=DEV, dtype=PARAM[dt]).normal_(0.0, 1e-3, generator=g)
        for n, at in zip(numels, firsts):
            flat[at + n:at + (n + step - 1) // step * step] = 0
        s["flat"], s["bucket"] = flat, torch.zeros_like(flat)
        at = [f * flat.element_size() for f in firsts]
        s["src"] = (ctypes.c_void_p * len(numels))(*[flat.data_ptr() + a for a in at])
        s["dst"] = (ctypes.c_void_p * len(numels))(*[s["bucket"].data_ptr() + a for a in at])
        s["numel"] = (ctypes.c_uint64 * len(numels))(*numels)
        s["n_tensors"] = len(numels)
        s["norm"] = torch.empty(2, device=DEV, dtype=torch.float64)      # the norm and the coefficient
    return s


def _run_own(s):
    import paper_2507_03211_amd as zo
    kind, code = s["kind"], CODES[s["dtype"]]
    stream = torch.cuda.current_stream()
    if kind == "norm":
        zo.zo_kernel_layernorm(s["resid"], s["gain"], s["bias"], s["y"], s["mean"], s["rstd"], code, s["rows"], s["d"], EPS, stream)
        return [s["y"], s["mean"], s["rstd"]]
    if "scratch" not in s:                  # a workspace the program keeps
        n = zo.zo_kernel_layernorm_grad_scratch_bytes(code, s["rows"], s["d"]) if kind == "norm_grad" else \
            zo.zo_kernel_lmhead_grad_scratch_bytes(code, s["batch"] * s["seq"], s["d"], s["vocab"]) if kind == "head" else \
            zo.zo_kernel_grad_clip_scratch_bytes()
        s["scratch"] = torch.empty(n, device=DEV, dtype=torch.uint8)
    if kind == "norm_grad":
        zo.zo_kernel_layernorm_grad(s["dy"], s["resid"], s["gain"], s["mean"], s["rstd"], s["dresid"], s["dgain"], s["dbias"], s["scratch"],
                                    code, s["rows"], s["d"], False, stream)
        return [s["dresid"], s["dgain"], s["dbias"]]
    if kind == "head":
        zo.zo_kernel_lmhead_grad(s["x"], s["e"], s["target"], s["row_loss"], s["dx"], s["de"], s["scratch"], code, s["batch"] * s["seq"],
                                 s["d"], s["vocab"], s["scale"], stream)
        return [s["row_loss"], s["dx"], s["de"]]
    zo.zo_kernel_grad_clip(s["src"], s["dst"], s["numel"], s["n_tensors"], code, 1.0, s["norm"], s["scratch"], stream)
    return [s["bucket"], s["norm"]]


def run(s):
    if own:
        return _run_own(s)
    kind, dt = s["kind"], s["dtype"]
    acc = RESID[dt]
    if kind == "norm":
        h = s["resid"]
        mean = h.sum(1, keepdim=True) / s["d"]
        centred = h - mean
        rstd = 1.0 / torch.sqrt((centred * centred).sum(1, keepdim=True) / s["d"] + EPS)
        y = s["gain"].to(acc) * (centred * rstd) + s["bias"].to(acc)
        return [y.to(ACT[dt]), mean.squeeze(1), rstd.squeeze(1)]
    if kind == "norm_grad":
        xh = (s["resid"] - s["mean"][:, None]) * s["rstd"][:, None]
        dy = s["dy"].to(acc)
        a = dy * s["gain"].to(acc)
        dh = s["rstd"][:, None] * (a - a.sum(1, keepdim=True) / s["d"] - xh * ((a * xh).sum(1, keepdim=True) / s["d"]))
        return [dh, (dy * xh).sum(0).to(PARAM[dt]), dy.sum(0).to(PARAM[dt])]
    if kind == "head":
        x, e = s["x"].to(acc), s["e"].to(acc)
        counts = (s["target"] >= 0)[:, None]
        at = s["target"].clamp(min=0).long()[:, None]
        logits = x @ e.t()
        top = logits.amax(1, keepdim=True)
        hit = logits.gather(1, at)
        p = torch.exp(logits - top)
        z = p.sum(1, keepdim=True)
        loss = torch.where(counts, torch.log(z) + (top - hit), 0.0)
        p = p / z
        # p - 1 at the target as minus the others' sum would say it: exp(.) - 1 in one function, exact where p is near 1
        p.scatter_(1, at, torch.expm1(hit - top - torch.log(z)))
        p = torch.where(counts, p, 0.0)
        return [loss.squeeze(1), ((p @ e) * s["scale"]).to(ACT[dt]), ((p.t() @ x) * s["scale"]).to(PARAM[dt])]
    norm = torch.sqrt(s["flat"].double().square().sum())
    coef = torch.where(norm > 1.0, 1.0 / norm, 1.0)
    return [(s["flat"].float() * coef.float()).to(PARAM[dt]), torch.stack([norm, coef])]


def work(case):
    param = PARAM[case["dtype"]].itemsize
    act, resid = ACT[case["dtype"]].itemsize, RESID[case["dtype"]].itemsize
    if case["kind"] == "norm":
        return {"bytes": case["rows"] * (case["d"] * (resid + act) + 2 * resid) + 2 * case["d"] * param, "flops": 8 * case["rows"] * case["d"]}
    if case["kind"] == "norm_grad":
        return {"bytes": case["rows"] * (case["d"] * (2 * resid + act) + 2 * resid) + 3 * case["d"] * param, "flops": 14 * case["rows"] * case["d"]}
    if case["kind"] == "head":
        rows = case["batch"] * case["seq"]
        return {"bytes": 2 * rows * case["d"] * act + 2 * case["vocab"] * case["d"] * param + rows * (4 + resid),
                "flops": 6 * rows * case["vocab"] * case["d"]}
    return {"bytes": 2 * param * sum(_numels(case)), "flops": 3 * sum(_numels(case))}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        h = s["resid"].double()
        n = case["d"]
        first, second = h.mean(1), h.pow(2).mean(1)
        rstd = (second - first.pow(2) + EPS).pow(-0.5)
        y = h * (rstd[:, None] * s["gain"].double()[None]) + (s["bias"].double()[None] - (first * rstd)[:, None] * s["gain"].double()[None])
        return [y, first, rstd]
    if kind == "norm_grad":
        n = case["d"]
        mean, rstd, dy = s["mean"].double()[:, None], s["rstd"].double()[:, None], s["dy"].double()
        h = s["resid"].double()
        w = s["gain"].double()[None]
        # through y = w (h - mean) rstd: the direct share, and what goes through the mean and through rstd
        direct = dy * w * rstd
        by_rstd = ((dy * w * (h - mean)).sum(1, keepdim=True)) * rstd.pow(3) / n
        dh = direct - direct.mean(1, keepdim=True) - by_rstd * (h - mean)
        return [dh, ((h - mean) * rstd * dy).sum(0), dy.sum(0)]
    if kind == "head":
        x, e, t = s["x"].double(), s["e"].double(), s["target"].long()
        live = t >= 0
        x_live, t_live = x[live], t[live]
        logp = x_live @ e.t()
        logp -= torch.logsumexp(logp, 1, keepdim=True)
        loss = torch.zeros(len(t), device=DEV, dtype=torch.float64)
        loss[live] = -logp[torch.arange(len(t_live), device=DEV), t_live]
        grad = logp.exp_()
        others = grad.sum(1) - grad[torch.arange(len(t_live), device=DEV), t_live]
        grad[torch.arange(len(t_live), device=DEV), t_live] = -others
        grad *= s["scale"]
        dx = torch.zeros_like(x)
        dx[live] = grad @ e
        return [loss, dx, grad.t().contiguous() @ x_live]
    flat = s["flat"].double()
    norm = torch.linalg.vector_norm(flat)
    coef = min(1.0, 1.0 / float(norm))
    return [flat * coef, torch.tensor([float(norm), coef], dtype=torch.float64)]
