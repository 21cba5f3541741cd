"""Infinite numbers in a sequence's fp16 tail, against the definition: they are taken for what they are.  (In a tile that is quantised they make it NaN.)

Finite results: the tolerance of the attention tests, 7e-5 of a vector."""
import numpy as np
import pytest
import torch

from oracle import cache8 as oracle
from paper_2504_11816_amd.cache8 import Cache8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = np.inf


def dev(x, dtype=None):
    return torch.tensor(np.ascontiguousarray(x), dtype=dtype, device=DEV)


G, R, T = 2, 2, 32
# width: tables that hold 768 keys, whose sequences are not cut, and wider ones, whose pieces one wavefront or four join
CASES = [pytest.mark.parametrize("fmt", ["int8", "e4m3"]), pytest.mark.parametrize("d", [64, 128]), pytest.mark.parametrize("width", [24, 40, 600]),
         pytest.mark.parametrize("n,appends", [(1, True), (1, False), (9, True), (9, False), (32, True), (75, True), (75, False), (700, True), (700, False)])]


def every_case(test):
    for mark in CASES:
        test = mark(test)
    return test


def check(fmt, d, width, n, appends, changes):
    """changes(tail): lists of (k or v, token, element, value), each list for a sequence of its own; and an empty sequence behind them."""
    H = G * R
    rng = np.random.default_rng(n + d)
    q = np.abs(rng.standard_normal((H, d))).astype(np.float16) / 4 + np.float16(0.01)
    plain = [rng.standard_normal((n, G, d)).astype(np.float16) for _ in range(2)]
    cases = []
    for change in changes(range((n - appends) // 32 * 32, n)):
        k, v = (x.copy() for x in plain)
        for name, at, e, value in change:
            (k if name == "k" else v)[at, 1, e] = value
        cases.append((k, v))
    B, per, before = len(cases) + 1, -(-n // T), n - appends
    c = Cache8(n_layers=1, n_q_heads=H, n_kv_heads=G, head_dim=d, page_tokens=T, n_pages=per * B, max_seqs=B, max_pages_per_seq=width, format=fmt,
               out_dtype=torch.float32, device=DEV)
    c.table[:, :per] = torch.arange(per * B, dtype=torch.int32, device=DEV).view(B, per)
    c.lens.copy_(dev([before] * (B - 1) + [0], torch.int32))
    k, v = (np.concatenate([x[i][:before] for x in cases])[None] for i in (0, 1))
    c.store(dev(k), dev(v), dev([before * min(b, B - 1) for b in range(B + 1)], torch.int32), c.lens)
    c.lens.copy_(dev([n] * (B - 1) + [0], torch.int32))
    new = [dev(np.stack([x[i][-1] for x in cases] + [plain[i][0]])[None]) if appends else None for i in (0, 1)]
    out = torch.full((1, B, H, d), 7.0, device=DEV)
    c.step(dev(np.stack([q] * B)[None]), *new, out, c.lens)
    got = out[0].double().cpu().numpy()
    assert (got[-1] == 0).all()
    for i, (k, v) in enumerate(cases):
        with np.errstate(invalid="ignore"):
            want = oracle.attend(q, k, v, n, fmt, appends)
        for h in range(H):
            there = np.isfinite(want[h])
            assert np.array_equal(got[i, h][~there], want[h][~there], equal_nan=True), (i, h)
            assert np.linalg.norm(got[i, h][there] - want[h][there]) <= 7e-5 * np.linalg.norm(want[h][there]), (i, h)


@every_case
def test_infinite_values(fmt, d, width, n, appends):
    """Of either sign, of several keys, in one element (which is then NaN)."""
    check(fmt, d, width, n, appends, lambda tail: [
        [], [("v", tail[-1], 3, INF)], [("v", tail[len(tail) // 2], 3, -INF), ("v", tail[-1], d - 1, INF)], [("v", i, 9, INF) for i in tail],
        [("v", tail[0], 7, INF), ("v", tail[-1], 7, -INF)]])


@every_case
def test_infinite_scores(fmt, d, width, n, appends):
    """A score of -infinity leaves its key out: one of the tail's, all of them (NaN, if there are no others), all but one; one of +infinity makes NaN."""
    check(fmt, d, width, n, appends, lambda tail: [
        [], [("k", tail[-1], 5, -INF)], [("k", i, 5, -INF) for i in tail], [("k", tail[len(tail) // 2], 5, INF)],
        [("k", i, 5, -INF) for i in tail[1:]] + [("v", tail[0], 0, INF)]])
