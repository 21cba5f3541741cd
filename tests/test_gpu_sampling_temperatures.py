"""Probabilities at temperatures that are infinite or as large as numbers are: barred tokens stay at 0."""
import math

import numpy as np
import pytest
import torch

from paper_2504_11816_amd.sampling import Sampler

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", (torch.float16, torch.float32), ids=str)
@pytest.mark.parametrize("vocab", (1, 7, 5000, 32768, 32769, 140000))
def test_infinite_temperatures(vocab, dtype):
    """Every token that is not barred is as likely as any other.  Off by the sum of n numbers that are 1 but for 2^-22 each (a difference of 2^128 at most times the smallest factor), in 32 bits, and a quotient."""
    g = torch.Generator(device=DEV).manual_seed(vocab)
    x = (torch.randn((5, vocab), generator=g, device=DEV) * 4).to(dtype)
    x[1, ::3] = -math.inf
    x[2] = -math.inf
    x[3, vocab // 2] = torch.finfo(dtype).max
    x[4, vocab // 2] = math.inf
    out = torch.full((5, vocab), math.nan, device=DEV)
    s = Sampler(max_batch=5, vocab=vocab, device=DEV)
    for t in (math.inf, torch.finfo(torch.float32).max):
        s.probs(x, out, torch.full((5,), t, device=DEV))
        got = out.double().cpu().numpy()
        for r in (0, 1, 2, 3) if t == math.inf else (0, 1, 2):
            there = (x[r] > -math.inf).cpu().numpy()
            want = there / max(1, there.sum())
            assert (np.abs(got[r] - want) <= 2.0 ** -24 * (32 + vocab / 64) * want).all(), (r, t)
        assert np.isnan(got[4]).all()
