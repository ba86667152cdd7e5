"""Sampling where a place lies among many logits that differ in their last bits alone: few enough to be gathered, too many for a wave to sort."""
import numpy as np
import pytest
import torch

from tests.test_gpu_sample import DEV, SETTINGS, TD, call, check

pytestmark = pytest.mark.gpu


def _near(rows, vocab, n, same, dtype, seed):
    """n logits from 1.25 on in steps of their type's last bit, `same` tokens at each, at random places of a row of unlikely tokens."""
    g = torch.Generator().manual_seed(seed)
    step = {"fp32": 2.0 ** -23, "fp16": 2.0 ** -10}[dtype]
    values = 1.25 + (torch.arange(n, dtype=torch.float64) // same) * step
    if dtype == "fp16":
        values *= 2.0 ** -6  # (a step is then 2^-16: a thousand of them lie in a bin of 1 / 32)
    l = torch.empty(rows, vocab, dtype=torch.float64).uniform_(-60, -20, generator=g)
    for r in range(rows):
        l[r, torch.randperm(vocab, generator=g)[:n]] = values[torch.randperm(n, generator=g)]
    out = l.to(TD[dtype])
    assert torch.equal(out[l > 0].double(), l[l > 0])
    return out.to(DEV)


@pytest.mark.parametrize("n,same", [(129, 1), (300, 1), (1000, 1), (1000, 3), (1000, 90), (4096, 1), (4096, 7), (4096, 700)])
@pytest.mark.parametrize("rows,vocab", [(3, 6000), (3, 30000), (260, 9000)])
def test_places_among_nearly_equal_logits(rows, vocab, n, same):
    logits = _near(rows, vocab, n, same, "fp32", n + same)
    u = torch.rand(rows, generator=torch.Generator().manual_seed(n)).to(DEV)
    # min_p lies among the logits too: the largest is n / same steps of 2^-23 above the least
    inside = float(np.float32(np.exp(-n / same * 2.0 ** -24)))
    for s in [dict(), dict(top_k=n // 2), dict(top_k=n - 1, top_p=0.6), dict(top_p=0.3), dict(min_p=inside), dict(top_k=n // 3, top_p=0.9, min_p=inside), dict(temperature=0.7, top_k=n // 2 + 1, top_p=0.5)] + SETTINGS[-2:]:
        check(logits, u, *call(logits, u, **s), **s)


@pytest.mark.parametrize("n,same", [(200, 1), (500, 2), (4000, 11)])
@pytest.mark.parametrize("rows,vocab", [(3, 6000), (3, 30000)])
def test_the_same_in_binary16(rows, vocab, n, same):
    logits = _near(rows, vocab, n, same, "fp16", n)
    u = torch.rand(rows, generator=torch.Generator().manual_seed(n)).to(DEV)
    for s in [dict(), dict(top_k=n // 2), dict(top_k=n - 1, top_p=0.6), dict(top_p=0.3)]:
        check(logits, u, *call(logits, u, **s), **s)
