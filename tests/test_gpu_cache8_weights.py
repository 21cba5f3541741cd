"""Decode attention over the 8-bit cache where one key takes most of the softmax and its values are small, so that the result is the others': their weights,
far below the largest, have to keep their bits.  Attention sinks are of this kind.

Tolerance, relative to an output vector, values being positive.  Scores are sums of at most 4 products (the other elements of q are zero) scaled and shifted in two more
steps, up to 24 here: 7 2^-24 24.  The products of 32 keys join the sums of the others in one step, the weights' own sum takes 8 more for
its lanes: (n / 32 + 8) 2^-24 each for numerator and denominator.  The weights' own roundings, exponentials, logarithms and reciprocals: 2^-18."""
import numpy as np
import pytest
import torch

from oracle import cache8 as oracle
from paper_2504_11816_amd.cache8 import Cache8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(x, dtype=None):
    return torch.tensor(np.ascontiguousarray(x), dtype=dtype, device=DEV)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,width,B", [(768, 24, 4), (768, 40, 40), (4096, 128, None), (16384, 512, None)])
@pytest.mark.parametrize("alike,low", [(False, 1.0), (True, 1.0), (False, 2.0 ** -6)])
def test_small_weights_keep_their_bits(fmt, d, n, width, B, alike, low):
    """B None: as many sequences as there are stretches, so that a wavefront has all keys of one.  alike: the other keys have one score, and are all rounded the
    same way.  low: the other tiles' values, which the scale of the first one's, in the weights' exponent, then takes bits from as well."""
    G, R = 2, 2
    H, tol = G * R, 2 * (n / 32 + 8) * 2.0 ** -24 + 7 * 24 * 2.0 ** -24 + 2.0 ** -18
    B = B or 1024 * (128 // d) // G
    rng = np.random.default_rng(n + d)
    k = rng.standard_normal((n, G, d)).clip(-3, 3).astype(np.float16)
    k[:, :, 0], k[0, :, 0] = 0, 3
    v = (1 + 0.25 * rng.standard_normal((n, G, d))).clip(0.1, 2)
    v[32:] *= low
    v[0] = 0.02
    v = v.astype(np.float16)
    gaps = np.linspace(8, 20, B)
    q = np.zeros((B, H, d), np.float16)
    q[:, :, 0] = gaps[:, None] * d ** 0.5 / 3
    if not alike:
        q[:, :, 1:4] = (rng.standard_normal((B, H, 3)) * d ** 0.5 / 6).clip(-0.4 * d ** 0.5, 0.4 * d ** 0.5)
    c = Cache8(n_layers=1, n_q_heads=H, n_kv_heads=G, head_dim=d, page_tokens=32, n_pages=n // 32, max_seqs=B, max_pages_per_seq=width, format=fmt,
               out_dtype=torch.float32, device=DEV)
    c.table[:, :n // 32] = torch.arange(n // 32, dtype=torch.int32, device=DEV)      # all sequences share all pages
    c.lens.fill_(n)
    c.store(dev(k[None]), dev(v[None]), dev([0, n], torch.int32), c.lens, dev([0], torch.int32))
    out = torch.full((1, B, H, d), float("nan"), device=DEV)
    c.step(dev(q[None]), None, None, out, c.lens)
    got, hk, hv = out[0].double().cpu().numpy(), oracle.held(k, fmt, n), oracle.held(v, fmt, n)
    for b in sorted({0, 1, B // 4, B // 3, B // 2, 2 * B // 3, B - 1}):
        for h in range(H):
            s = hk[:, h // R] @ q[b, h].astype(np.float64) / d ** 0.5
            w = np.exp(s - s.max())
            want = w @ hv[:, h // R] / w.sum()
            err = np.linalg.norm(got[b, h] - want) / np.linalg.norm(want)
            assert err <= tol, (gaps[b], h, err, tol)
