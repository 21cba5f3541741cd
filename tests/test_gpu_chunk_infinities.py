"""Attention of several new rows over contexts that are shared out among workgroups, with values that are not finite: where rows see them, and nowhere else."""
import math

import numpy as np
import pytest
import torch

from chunk_util import DEV, Paged, ids, starts_of
from oracle import chunk as oracle

pytestmark = pytest.mark.gpu


def attend(p, q, n_new, dtype, **kw):
    out = torch.full(q.shape, math.nan, dtype=dtype, device=DEV)
    p.cache.attend(1, q, out, starts_of(n_new), p.cache.lens, ids(p.seqs), **kw)
    return out.float().cpu().numpy()


def check(p, odd, q, n_new, dtype, window=0):
    """odd: (sequence, KV head, token, value) of values whose element 7 is not finite (by turns infinite and NaN).  Rows that see one are infinite or NaN there and are otherwise, and all other rows are,
    what they are without: bit for bit."""
    clean = attend(p, q, n_new, dtype, window=window)
    saved = p.pool.copy()
    for b, g, token, value in odd:
        p.pool[p.offset(b, 1, g, token) + 7] = value
    p.upload()
    got = attend(p, q, n_new, dtype, window=window)
    p.pool[:] = saved
    p.upload()
    R, row = p.H // p.G, 0
    for b, n in enumerate(n_new):
        for j in range(n):
            pos = p.lens[b] - n + j
            seen = oracle.sees(pos, p.lens[b], window, 0)
            for h in range(p.H):
                there = [x for c, g, token, x in odd if c == b and g == h // R and seen[token]]
                a, z = got[row, h], clean[row, h]
                assert not there or not np.isfinite(a[7]), f"sequence {b} row {j} of {n} head {h} sees {there} and is {a[7]}"
                assert np.array_equal(np.delete(a, 7), np.delete(z, 7)) and (there or a[7] == z[7]), f"sequence {b} row {j} of {n} head {h}"
            row += 1


@pytest.mark.parametrize("dtype", (torch.float16, torch.float32), ids=str)
@pytest.mark.parametrize("H,G,d", [(4, 2, 128), (4, 1, 64), (3, 3, 64)])
@pytest.mark.parametrize("n_new", ([4, 1, 5, 2], [150, 1, 40, 3]), ids=("few", "many"))
def test_values_that_are_not_finite_in_long_contexts(n_new, H, G, d, dtype):
    """In the blocks of each wavefront, where some rows see them and others do not: at the end, and where a window begins.  Pieces of a sequence that has another's blocks before it are among them."""
    lens = [4100, 3333, 2600, 64]
    p = Paged(H, G, d, 32, lens, seed=d + G, room=5000)
    q = torch.randn((sum(n_new), H, d), generator=torch.Generator().manual_seed(3)).half().to(DEV)
    values = (np.inf, np.nan, -np.inf)
    for window in (0, 700):
        for part in range(3):
            odd = []
            for b, n in enumerate(n_new):
                places = sorted({t for t in (lens[b] - 1, lens[b] - 2, lens[b] - n, lens[b] - n // 2 - 1, lens[b] - window - n + 1, lens[b] - window - 1, lens[b] - window - 33) if 0 <= t < lens[b]})
                odd += [(b, (i + part) % G, t, values[(i + part) % 3]) for i, t in enumerate(places) if i % 3 == part]
            check(p, odd, q, n_new, dtype, window)


@pytest.mark.parametrize("dtype", (torch.float16, torch.float32), ids=str)
@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("n_new", ([4, 2], [200, 90]), ids=("few", "many"))
def test_values_that_are_not_finite_far_below_the_largest_score(n_new, d, dtype):
    """A key with a score of hundreds in one piece of the keys, a value that is not finite in another, whose weights are 2^-126 of the largest and less: the result is infinite or NaN however the keys were cut."""
    lens = [9000, 7000]
    p = Paged(4, 2, d, 64, lens, seed=d)
    for b in range(2):
        for g in range(2):
            p.pool[p.offset(b, 0, g, lens[b] - n_new[b] - 300)] = 2000.0
    p.upload()
    q = torch.randn((sum(n_new), 4, d), generator=torch.Generator().manual_seed(4)).half().to(DEV)
    q[:, :, 0] = 4.0                                         # 2000 * 4 / sqrt(d): 707 and more above the others
    for value in (np.inf, -np.inf, np.nan):
        check(p, [(0, 0, 5, value), (1, 1, 2000, value)], q, n_new, dtype)


@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("room", (0, 5000))
@pytest.mark.parametrize("n_new", ([4], [300]), ids=("few", "many"))
def test_values_that_are_not_finite_count_at_keys_without_weight(n_new, room, d):
    """A score of -infinity gives its key no weight; its value, where it is not finite, is seen all the same."""
    lens = [700]
    p = Paged(4, 2, d, 64, lens, seed=d, room=room)
    places = (3, 500, 697)
    for token in places:
        p.pool[p.offset(0, 0, 1, token)] = -np.inf
    p.upload()
    q = torch.randn((n_new[0], 4, d), generator=torch.Generator().manual_seed(4)).half().to(DEV)
    q[:, :, 0] = 1.0
    for dtype in (torch.float16, torch.float32):
        for token in places:
            check(p, [(0, 1, token, np.inf)], q, n_new, dtype)
