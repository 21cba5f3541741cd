"""Rows whose tokens the pool has no place for: past the capacity, and in pages that the table does not name."""
import numpy as np
import pytest
import torch

from chunk_util import DEV, check_rows, ids, starts_of
from oracle import chunk as oracle
from oracle import kv_layout
from paper_2504_11816_amd.cache16 import Cache16, Rope

pytestmark = pytest.mark.gpu


def filled(H, G, d, T, per_seq, seqs=2, seed=0):
    """A cache whose sequences may have per_seq pages each, all of them in the table, every number set."""
    n_pages = per_seq * seqs
    c = Cache16(n_layers=1, n_q_heads=H, n_kv_heads=G, head_dim=d, page_tokens=T, n_pages=n_pages, max_seqs=seqs, max_pages_per_seq=per_seq, device=DEV)
    rng = np.random.default_rng(seed)
    c.table.copy_(torch.from_numpy(rng.permutation(n_pages).astype(np.int32).reshape(seqs, per_seq)))
    c.pool.copy_(torch.from_numpy(rng.standard_normal(tuple(c.pool.shape)).astype(np.float16)))
    return c


def layout_of(c):
    return dict(kind="paged", G=c.G, d=c.d, T=c.T, block_table=c.table.cpu().numpy())


def normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).half().to(DEV)


@pytest.mark.parametrize("G,d", [(2, 64), (4, 128)])
@pytest.mark.parametrize("over", (1, 2, 4, 30, 1 << 30, (1 << 31) - 1 - 64))
def test_tokens_past_the_capacity_are_not_stored(over, G, d):
    """Row i of n is token len - n + i whatever the capacity: those that fit are at their own places, turned by them, earlier tokens stay bit for bit, and queries are turned by their own positions."""
    T, per_seq, n = 16, 4, 4
    capacity = T * per_seq
    c = filled(G, G, d, T, per_seq, seed=G)
    before, layout = c.pool.cpu().numpy().reshape(-1).copy(), layout_of(c)
    k, v, q = normal(1, n, G, d), normal(2, n, G, d), normal(3, n, G, d)
    q_out = torch.empty_like(q)
    c.append(0, k, v, ids([0, n]), ids([0, capacity + over]), ids([1]), q=q, q_out=q_out, rope=Rope.of(d, device=DEV))
    tokens = [capacity + over - n + i for i in range(n)]
    freq = 10000.0 ** (-np.arange(0, d, 2) / d)
    turned, want, places = oracle.rotate(k.cpu().numpy(), tokens, freq, False), before.astype(np.float64), np.zeros(before.shape, dtype=bool)
    for i, t in enumerate(tokens):
        if t < capacity:
            for g in range(G):
                a, z = kv_layout.token_row_offset(layout, 1, 0, g, t), kv_layout.token_row_offset(layout, 1, 1, g, t)
                want[a:a + d], want[z:z + d], places[a:a + d] = turned[i, g], v[i, g].cpu().numpy(), True
    got = c.pool.cpu().numpy().reshape(-1)
    assert np.array_equal(got[~places], want[~places])
    # (a turned number: half a step of itself, factors off by 2^-22 and, of positions of 2^31, an angle off by some 2^-53 of itself: 2^-19 of numbers of up to 5)
    size = 2.0 ** -19 * 2 * 5
    assert (np.abs(got - want) <= 2.0 ** -11 * np.abs(want) + size)[places].all()
    qw = oracle.rotate(q.cpu().numpy(), tokens, freq, False)
    assert (np.abs(q_out.cpu().numpy() - qw) <= 2.0 ** -11 * np.abs(qw) + size).all()


class Tokens:
    """What check_rows asks of a cache."""

    def __init__(self, c, seq):
        self.H, self.G, self.d, self.lens = c.H, c.G, c.d, [c.T * c.table.shape[1]]
        self.pool, self.layout, self.seq = c.pool.cpu().numpy().reshape(-1), layout_of(c), seq

    def rows(self, b, kv, g):
        return kv_layout.gather_rows(self.pool, self.layout, self.seq, kv, g, self.lens[b])


@pytest.mark.parametrize("kw", [dict(), dict(window=9), dict(window=40, prefix=5), dict(slopes=True), dict(cap=4.0, window=100)], ids=str)
@pytest.mark.parametrize("n,over", [(5, 2), (150, 20), (3, 3), (4, 9), (150, 1 << 30), (70, (1 << 31) - 1 - 2048)])
@pytest.mark.parametrize("H,G,d,per_seq", [(4, 2, 64, 12), (3, 3, 128, 12), (4, 2, 64, 128)])
def test_attention_past_the_capacity(H, G, d, per_seq, n, over, kw):
    """A row's position is its token's place: rows whose tokens the pool has attend from there, as they do in a call without those behind them; rows past it attend as its last token does.  In small caches and in
    those whose keys may be cut, few rows and many."""
    T = 16
    capacity = T * per_seq
    over = min(over, (1 << 31) - 1 - capacity)
    c = filled(H, G, d, T, per_seq, seed=d + per_seq)
    q, kw = normal(n, n, H, d), dict(kw)
    how = dict(kw)
    if kw.get("slopes"):
        kw["slopes"] = [2.0 ** -(i + 1) for i in range(H)]
        how["slopes"] = torch.tensor(kw["slopes"], device=DEV)
    if kw.get("prefix"):
        how["prefix"], kw["prefix"] = ids([0, kw["prefix"]]), [kw["prefix"]]
    for dtype in (torch.float16, torch.float32):
        out = torch.full(q.shape, np.nan, dtype=dtype, device=DEV)
        c.attend(0, q, out, starts_of([n]), ids([0, capacity + over]), ids([1]), **how)
        p, there = Tokens(c, 1), max(0, n - over)
        if there:
            check_rows(p, q[:there], out[:there], [there], **kw)
        for j in {there, (there + n) // 2, n - 1}:
            check_rows(p, q[j:j + 1], out[j:j + 1], [1], **kw)


@pytest.mark.parametrize("missing", (-1, -5, 8, 1 << 30))
def test_rows_of_pages_that_the_table_does_not_name_are_not_stored(missing):
    """Nothing goes into a page that is another sequence's."""
    T, G, d = 16, 2, 64
    c = filled(G, G, d, T, 4)
    c.table[1, 2] = missing
    before, layout = c.pool.cpu().numpy().reshape(-1).copy(), layout_of(c)
    k, v = normal(1, 24, G, d), normal(2, 24, G, d)
    c.append(0, k, v, ids([0, 24]), ids([0, 52]), ids([1]))      # tokens 28 .. 51: the missing page's are 32 .. 47
    want = before.copy()
    for i, t in enumerate(range(28, 52)):
        if t // T != 2:
            for g in range(G):
                for kv, x in ((0, k), (1, v)):
                    a = kv_layout.token_row_offset(layout, 1, kv, g, t)
                    want[a:a + d] = x[i, g].cpu().numpy()
    assert np.array_equal(c.pool.cpu().numpy().reshape(-1), want)
