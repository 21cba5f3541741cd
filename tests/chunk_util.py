"""A paged fp16 cache on the GPU and its tokens on the CPU, for tests of steps with several tokens a sequence; what such a step may be off by."""
import math

import numpy as np
import torch

from oracle import chunk as oracle
from oracle import kv_layout
from paper_2504_11816_amd.cache16 import Cache16

DEV = "cuda:0"


def ids(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def starts_of(n):
    return ids(np.concatenate([[0], np.cumsum(n)]))


class Paged:
    """Sequences of lens tokens, in rows `seqs` of a table of more rows, their pages shuffled; every number of the pool is set (behind a sequence's end: `behind`)."""

    def __init__(self, H, G, d, T, lens, seed=0, behind=None, room=0):
        rng = np.random.default_rng(seed)
        self.H, self.G, self.d, self.T, self.lens = H, G, d, T, list(lens)
        B = len(lens)
        self.seqs = [int(x) for x in rng.permutation(B + 2)[:B]]
        need = [-(-n // T) for n in lens]
        width, n_pages = max([*need, room // T]) + 1, sum(need) + 2      # room: tokens that a sequence can have at least (what is chosen goes by that, too)
        ids_of = rng.permutation(n_pages)
        table, at = np.full((B + 2, width), -1, dtype=np.int32), 0
        for s, n in zip(self.seqs, need):
            table[s, :n] = ids_of[at:at + n]
            at += n
        self.cache = Cache16(n_layers=2, n_q_heads=H, n_kv_heads=G, head_dim=d, page_tokens=T, n_pages=n_pages, max_seqs=B + 2, max_pages_per_seq=width,
                             table=torch.from_numpy(table).to(DEV), device=DEV)
        self.np_table = table
        pool = rng.standard_normal((n_pages, 2 * G * T * d)).astype(np.float16)
        if behind is not None:
            used = np.zeros(pool.size, dtype=bool)
            for b in range(B):
                for kv in range(2):
                    for g in range(G):
                        for i in range(lens[b]):
                            o = self.offset(b, kv, g, i)
                            used[o:o + d] = True
            pool.reshape(-1)[~used] = behind
        self.pool = pool.reshape(-1)
        self.upload()
        for s, n in zip(self.seqs, lens):
            self.cache.lens[s] = n

    def layout(self):
        return dict(kind="paged", G=self.G, d=self.d, T=self.T, block_table=self.np_table)

    def offset(self, b, kv, g, i):
        return kv_layout.token_row_offset(self.layout(), self.seqs[b], kv, g, i)

    def upload(self):
        self.cache.pool[1].copy_(torch.from_numpy(self.pool.reshape(self.cache.pool[1].shape)))

    def rows(self, b, kv, g):
        return kv_layout.gather_rows(self.pool, self.layout(), self.seqs[b], kv, g, self.lens[b])


def check_rows(p, q, out, n_new, *, scale=0.0, cap=0.0, window=0, slopes=None, prefix=None, some=None):
    """Every row (or every `some`-th) of out against the oracle.  What a result may be off by, A the weighted mean of |v|:

    weights     each off by 2^-11 of itself (fp16, half a step) or 2^-22 (two fp16 numbers), beside sums that are not:  A 2^-11 or A 2^-22
    scores      d products summed in 32 bits, the scale, the cap's tanh (4 units of what it is multiplied with; a cap above 64 is relative: 16 units of a score, which
                is at most S and cap) and the bias: e <= (d + 8) 2^-24 S + 8 cap 2^-24 + 2^-22 bias (with a cap the first is at most 2 cap), which
                changes a weight by e and the sum by e:  2 e A;  exponents are products and differences of numbers of up to 2 S: 4 S 2^-24 each, and 2^-22 of the exponential
    sums        of n numbers in 32 bits, numerator and denominator: 2 n 2^-24 A
    the result  half a step of its type, 2^-11 (2^-24), and for fp16 the smallest number, 2^-25"""
    out32 = out.dtype is torch.float32
    q, got = q.cpu().numpy().astype(np.float64), out.cpu().numpy().astype(np.float64)
    row, worst, count = 0, 0.0, 0
    for b, n in enumerate(n_new):
        kv = {g: (p.rows(b, 0, g), p.rows(b, 1, g)) for g in range(p.G)}
        for j in range(n):
            pos = p.lens[b] - n + j
            for h in range(p.H):
                count += 1
                if some and (count % some):
                    continue
                K, V = kv[h // (p.H // p.G)]
                slope = 0.0 if slopes is None else float(slopes[h])
                want, A, S = oracle.attend(q[row, h], K, V, pos, scale, cap, window, slope, 0 if prefix is None else min(prefix[b], p.lens[b]))
                bias = slope * p.lens[b]
                e = min((p.d + 8) * 2.0 ** -24 * S, 2 * cap if cap else math.inf) + (8 * cap if cap <= 64 else 16 * min(S, cap)) * 2.0 ** -24 + 2.0 ** -22 * bias
                tol = A * ((2.0 ** -22 if out32 else 2.0 ** -11) + 2 * e + 4 * (min(S, cap) if cap else S) * 2.0 ** -24 + 4 * bias * 2.0 ** -24 + 2.0 ** -22 + 2 * (p.lens[b] + 2) * 2.0 ** -24)
                tol = tol + (2.0 ** -24 if out32 else 2.0 ** -11) * np.abs(want) + (0 if out32 else 2.0 ** -25)
                same = (got[row, h] == want) | (np.isnan(got[row, h]) & np.isnan(want))
                with np.errstate(invalid="ignore"):
                    off = np.where(same, 0.0, np.abs(got[row, h] - want) / np.maximum(tol, 1e-300))
                assert np.all(off <= 1), f"sequence {b} row {j} of {n} head {h}: {off.max():.3g} times what it may be off, at {int(np.argmax(np.where(np.isnan(off), np.inf, off)))}: {got[row, h][:4]} {want[:4]}"
                worst = max(worst, float(off.max()))
            row += 1
    return worst
