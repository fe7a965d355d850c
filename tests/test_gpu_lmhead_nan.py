"""Words of the LM head that are NaN, in strips' parts and in whole strips, against the loss's definition: a sign's losses are NaN in all
rows that count, the other sign's are as ever."""
import pytest
import torch

import paper_2507_03211_amd as zo_amd
import zo_inputs as zi
from gpu_util import DEV, act_dtype
from grad_util import generator, normal, param_dtype

pytestmark = pytest.mark.gpu


def words_of(vocab):
    """Parts of a strip of 64 or 128 words, whose halves take its words in turns of four; whole strips."""
    some = torch.arange(128)
    yield torch.arange(vocab - 8, vocab - 4)
    yield torch.arange(vocab - 4, vocab)
    yield torch.arange(vocab - 1, vocab)
    yield torch.arange((vocab - 1) // 128 * 128, vocab)
    yield 256 + some
    yield 256 + some[(some >> 2) % 2 == 0]
    yield 256 + some[(some >> 2) % 2 == 1]


@pytest.mark.parametrize("dtype", [zi.FP32, zi.BF16, zi.FP16])
@pytest.mark.parametrize("m_half,d,vocab", [(5, 64, 520), (5, 64, 1000), (40, 320, 4104), (300, 192, 12008), (700, 192, 8200), (1500, 256, 4104), (5, 64, 70408), (20, 72, 1000)])
def test_losses_of_nan_words(dtype, m_half, d, vocab):
    g = generator(m_half + d + vocab)
    x = normal((2 * m_half, d), act_dtype(dtype), g)
    ep, em = (normal((vocab, d), param_dtype(dtype), g, 0.3) for _ in range(2))
    target = torch.randint(0, vocab, (2 * m_half,), device=DEV, generator=g).to(torch.int32)
    target[::7] = -1
    scratch = torch.empty(zo_amd.zo_kernel_lmhead_scratch_bytes(dtype, m_half, vocab), device=DEV, dtype=torch.uint8)

    def losses(plus, minus):
        out = torch.full((2 * m_half,), 7.0, device=DEV, dtype=torch.float64)
        zo_amd.zo_kernel_lmhead_ce(x, plus, minus, target, out, scratch, dtype, m_half, d, vocab)
        torch.cuda.synchronize()
        return out

    good = losses(ep, em)
    count = target >= 0
    assert torch.isfinite(good).all() and (good[~count] == 0).all()
    first = torch.arange(2 * m_half, device=DEV) < m_half
    for words in words_of(vocab):
        for sign in range(2):
            bent = [ep.clone(), em.clone()]
            bent[sign][words.to(DEV)] = float("nan")
            got, bad = losses(*bent), count & (first if sign == 0 else ~first)
            assert torch.isnan(got[bad]).all(), (sign, words)
            assert torch.equal(got[~bad], good[~bad])
