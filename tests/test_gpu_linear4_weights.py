"""Weights that are no numbers, quantised to 4 bits: they are seen in the results."""
import numpy as np
import pytest
import torch

from oracle import linear4 as oracle
from paper_2504_11816_amd.linear4 import Linear4

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m", [1, 5, 40])
def test_a_weight_that_is_no_number_makes_its_feature_nan(m, group, zeros):
    """And nothing else: the other features' results are the bits that they are without it."""
    rng = np.random.default_rng(group)
    n_out, n_in = 48, 384
    w = (rng.standard_normal((n_out, n_in)) * 0.05).astype(np.float16)
    x = torch.tensor(rng.standard_normal((m, n_in)), dtype=torch.float16, device=DEV)
    plain, out = (torch.empty((m, n_out), dtype=torch.float16, device=DEV) for _ in range(2))
    Linear4.quantize(torch.tensor(w, device=DEV), group=group, zeros=zeros)(x, plain)
    bad = {3: (5, np.nan), 17: (n_in - 1, np.nan), 18: (200, np.inf), 40: (0, -np.inf)}
    for n, (k, value) in bad.items():
        w[n, k] = value
    w[45, 7], w[45, 300] = np.nan, np.inf
    w[20] = np.nan
    bad = [*bad, 45, 20]
    for relu in (False, True):
        q = Linear4.quantize(torch.tensor(w, device=DEV), group=group, zeros=zeros)
        q(x, out, relu=relu)
        got = out.cpu().numpy()
        assert np.isnan(got[:, bad]).all()
        others = np.setdiff1d(np.arange(n_out), bad)
        want = plain.cpu().numpy()[:, others]
        assert np.array_equal(got[:, others], np.maximum(want, 0) if relu else want)
    # which weights: those of the groups that have one
    seen = torch.empty((n_in, n_out), dtype=torch.float16, device=DEV)
    q(torch.eye(n_in, dtype=torch.float16, device=DEV), seen)
    want = oracle.quantise(w, group, zeros)
    assert np.isnan(want).any(1)[bad].all() and not np.isnan(want)[others].any()
    assert np.array_equal(seen.cpu().numpy().T[others], want[others].astype(np.float16))
