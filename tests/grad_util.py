"""Helpers of the gradient tests: types of a precision, buffers with a guarded end, and the error terms their tolerances count.

u is half a step of the type sums are taken in, `half` half a step of the type results are rounded to, `least` half of
the least subnormal number's step of that type.
"""
import torch

import zo_inputs as zi
from gpu_util import DEV, act_dtype, resid_dtype

PARAM = {zi.FP32: torch.float32, zi.BF16: torch.bfloat16, zi.FP16: torch.float16}
GUARD = 256


def param_dtype(dtype):
    return PARAM[dtype]


def unit(dtype):
    return 2.0**-53 if dtype == zi.FP32 else 2.0**-24


def half(t):
    return torch.finfo(t).eps / 2


def least(t):
    return {torch.bfloat16: 2.0**-134, torch.float16: 2.0**-25}.get(t, 0.0)


class Out:
    """An output of `shape` with bytes behind its end that a call has no business with."""

    def __init__(self, shape, t, fill=None):
        n = 1
        for s in shape:
            n *= s
        size = torch.empty((), dtype=t).element_size()
        self.raw = torch.full((n * size + GUARD,), 0xA5, dtype=torch.uint8, device=DEV)
        self.t = self.raw[:n * size].view(t).view(shape)
        if fill is not None:
            self.t.fill_(fill)

    def whole(self):
        return bool((self.raw[-GUARD:] == 0xA5).all())


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(shape, t, g, std=1.0):
    return torch.empty(shape, dtype=torch.float64, device=DEV).normal_(0.0, std, generator=g).to(t)
