"""Appending with rotation and attention of several new rows a sequence, against 64 bits."""
import ctypes
import math

import numpy as np
import pytest
import torch

from chunk_util import DEV, Paged, check_rows, ids, starts_of
from oracle import chunk as oracle
from oracle import kv_layout
from paper_2504_11816_amd import binding
from paper_2504_11816_amd.cache16 import Cache16, Rope

pytestmark = pytest.mark.gpu

HEADS = [(8, 8, 64), (8, 2, 128), (16, 1, 64), (3, 3, 128), (20, 5, 64), (24, 8, 128)]


def queries(rows, H, d, seed=5, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((rows, H, d), generator=g) * size).half().to(DEV)


def attended(p, q, n_new, dtype=torch.float16, prefix=None, slopes=None, **kw):
    out = torch.full(q.shape, math.nan, dtype=dtype, device=DEV)
    at = None
    if prefix is not None:
        at = torch.zeros(len(p.lens) + 2, dtype=torch.int32, device=DEV)
        at[torch.tensor(p.seqs, device=DEV)] = ids(prefix)
    p.cache.attend(1, q, out, starts_of(n_new), p.cache.lens, ids(p.seqs), prefix=at, slopes=None if slopes is None else torch.tensor(slopes, device=DEV), **kw)
    return out


@pytest.mark.parametrize("dtype", (torch.float16, torch.float32), ids=str)
@pytest.mark.parametrize("room,times", [(0, 1), (3000, 1), (3000, 3)])
@pytest.mark.parametrize("H,G,d", HEADS)
def test_rows_of_every_kind(H, G, d, room, times, dtype):
    """One token, none, whole prompts, chunks behind long contexts; lengths about tiles' and blocks' ends.  In small caches and large ones, with few rows and with many."""
    lens, n_new = [1, 40, 17, 64, 65, 200, 129, 33], [1, 1, 17, 64, 2, 0, 40, 5]
    lens, n_new = [n * times for n in lens], [n * times for n in n_new]
    p = Paged(H, G, d, 32, lens, seed=H + d, room=room)
    q = queries(sum(n_new), H, d)
    check_rows(p, q, attended(p, q, n_new, dtype), n_new)


@pytest.mark.parametrize("T", (16, 64, 256, 1024))
def test_pages_of_every_size(T):
    p = Paged(4, 2, 128, T, [300, 15, 16], seed=T)
    q = queries(47, 4, 128)
    check_rows(p, q, attended(p, q, [20, 15, 12]), [20, 15, 12])


@pytest.mark.parametrize("kw", [dict(window=1), dict(window=7), dict(window=64), dict(window=100), dict(window=1 << 30), dict(prefix=[3, 0, 200, 30]), dict(prefix=[500, 1, 64, 33], window=20),
                                dict(prefix=[4, 4, 4, 4], window=1), dict(cap=5.0), dict(cap=30.0, window=50, prefix=[1, 2, 3, 4]), dict(slopes=True), dict(slopes=True, prefix=[90, 0, 140, 2]),
                                dict(slopes=True, cap=10.0, window=33), dict(scale=0.5), dict(scale=0.01, cap=0.3)], ids=str)
@pytest.mark.parametrize("room", (0, 3000))
@pytest.mark.parametrize("dtype", (torch.float16, torch.float32), ids=str)
def test_masks_caps_and_biases(kw, dtype, room):
    kw = dict(kw)
    if kw.get("slopes"):
        kw["slopes"] = [2.0 ** -(i + 1) for i in range(6)]
    n_new = [100, 3, 77, 40]
    p = Paged(6, 3, 64, 16, [260, 70, 141, 40], seed=11, room=room)
    q = queries(sum(n_new), 6, 64, size=3.0)
    check_rows(p, q, attended(p, q, n_new, dtype, **kw), n_new, **kw)


@pytest.mark.parametrize("kw", [dict(cap=64.5), dict(cap=1000.0), dict(cap=1e6, slopes=True), dict(cap=1e30), dict(cap=1e30, scale=1e-10), dict(scale=30.0, cap=200.0),
                                dict(scale=1e30, cap=1e-30)], ids=str)
@pytest.mark.parametrize("n_new", ([100, 3, 77, 40], [5, 3, 1, 4]), ids=("many", "few"))
@pytest.mark.parametrize("d", (64, 128))
def test_caps_far_above_and_below_the_scores(kw, n_new, d):
    kw = dict(kw)
    if kw.get("slopes"):
        kw["slopes"] = [2.0 ** -(i + 1) for i in range(6)]
    p = Paged(6, 3, d, 16, [260, 70, 141, 40], seed=12, room=3000)
    q = queries(sum(n_new), 6, d, size=3.0)
    for dtype in (torch.float16, torch.float32):
        check_rows(p, q, attended(p, q, n_new, dtype, **kw), n_new, **kw)


def test_long_contexts():
    """Few rows over tens of thousands of keys, and some hundreds of rows: cut among workgroups."""
    for n_new, lens in (([5, 1], [30001, 20000]), ([300], [9000]), ([1, 600, 2], [5, 4000, 12345])):
        p = Paged(8, 2, 128, 256, lens, seed=3)
        for dtype in (torch.float16, torch.float32):
            q = queries(sum(n_new), 8, 128, size=2.0)
            check_rows(p, q, attended(p, q, n_new, dtype), n_new, some=97)
            check_rows(p, q, attended(p, q, n_new, dtype, window=3000, prefix=[4] * len(lens)), n_new, window=3000, prefix=[4] * len(lens), some=97)


def test_one_key_takes_the_weight():
    """A first token that takes most of the softmax and has small values leaves the result to weights far below the largest."""
    for d, dtype in ((64, torch.float16), (128, torch.float32)):
        p = Paged(2, 2, d, 64, [6000], seed=4)
        for g in range(2):
            k, v = p.offset(0, 0, g, 0), p.offset(0, 1, g, 0)
            p.pool[k:k + d] = 1.6 if d == 64 else 1.2
            p.pool[v:v + d] = 0.001
        p.upload()
        q = torch.ones((9, 2, d), dtype=torch.float16, device=DEV)
        out = attended(p, q, [9], dtype)
        check_rows(p, q, out, [9])


@pytest.mark.parametrize("d", (64, 128))
@pytest.mark.parametrize("room", (0, 3000))
def test_what_rows_do_not_see_does_not_change_them(room, d):
    """Infinities and NaN behind a sequence's end, and at keys that some rows of a tile see and others do not."""
    n_new, lens = [40, 5], [90, 33]
    p = Paged(4, 2, d, 32, lens, seed=6, behind=np.float16(np.nan), room=room)
    clean = Paged(4, 2, d, 32, lens, seed=6, room=room)
    q = queries(45, 4, d)
    check_rows(p, q, attended(p, q, n_new), n_new)
    for value, kv in ((np.inf, 1), (-np.inf, 1), (np.nan, 1), (np.nan, 0)):
        for token in (70, 89):
            o = p.offset(0, kv, 1, token)
            p.pool[o + 5] = value
        p.upload()
        for dtype in (torch.float16, torch.float32):
            out = attended(p, q, n_new, dtype)
            with np.errstate(invalid="ignore"):
                early = [j for j in range(40) if 50 + j < 70]
                want = attended(clean, q, n_new, dtype)
                assert torch.equal(out[early], want[early]) and torch.equal(out[40:], want[40:])
                late = out[early[-1] + 1:40, 2:].float().cpu().numpy()
                if kv == 0:
                    assert np.isnan(late).all()
                else:
                    assert not np.isfinite(late[..., 5]).any() and np.isfinite(np.delete(late, 5, -1)).all()
                    assert np.isfinite(out[:40, :2].float().cpu().numpy()).all()
                    if value == np.inf:
                        assert (late[..., 5] == np.inf).all()
        for token in (70, 89):                               # as it was
            o = p.offset(0, kv, 1, token)
            p.pool[o + 5] = clean.pool[o + 5]
    # a window that a number has left
    o = p.offset(0, 1, 0, 45)
    p.pool[o] = np.inf
    p.upload()
    out = attended(p, q, n_new, window=6).float().cpu().numpy()
    assert np.isinf(out[0, 0, 0]) and np.isfinite(out[1:40]).all()


def test_scores_of_minus_infinity_leave_keys_out():
    p = Paged(2, 2, 64, 16, [50], seed=8)
    for i in range(50):
        if i % 2 or i < 10:
            o = p.offset(0, 0, 1, i)
            p.pool[o] = -np.inf
    p.upload()
    q = queries(50, 2, 64)
    q[:, :, 0] = 1.0
    for dtype in (torch.float16, torch.float32):
        out = attended(p, q, [50], dtype)
        check_rows(p, q, out, [50])
        assert not out[:10, 1].any() and out[:10, 0].any()


def test_rows_before_the_first_token_and_rows_of_no_sequence():
    p = Paged(4, 4, 64, 16, [3, 20], seed=9)
    q = queries(12, 4, 64)
    out = attended(p, q, [5, 4])                             # 5 rows of a sequence of 3 tokens, and 3 rows more than there are
    assert not out[:2].any() and torch.isnan(out[9:]).all()
    check_rows(p, q[2:9], out[2:9], [3, 4])
    seen = attended(p, q, [5, 4], prefix=[2, 0])
    assert seen[:2].any() and torch.equal(seen[5:9], out[5:9])
    # a row of the table that there is not
    out = torch.full(q.shape, math.nan, dtype=torch.float16, device=DEV)
    p.cache.attend(1, q, out, ids([0, 5, 9]), p.cache.lens, ids([99, p.seqs[1]]))
    assert not out[:5].any() and torch.isnan(out[9:]).all()
    check_rows(p, q[5:9], out[5:9], [0, 4])
    # lengths past the capacity and below 0
    lens = p.cache.lens.clone()
    lens[p.seqs[0]], lens[p.seqs[1]] = -7, 1 << 30
    p.cache.attend(1, q, out, ids([0, 5, 9]), lens, ids(p.seqs))
    assert not out[:5].any() and torch.isfinite(out[5:9]).all()


def test_starts_that_do_not_ascend_stay_within_the_buffers():
    for room in (0, 3000):
        p = Paged(4, 2, 64, 16, [20, 30, 40], seed=1, room=room)
        q, out = queries(12, 4, 64), torch.full((14, 4, 64), math.nan, dtype=torch.float16, device=DEV)
        for starts in ([0, 9, 3, 20], [-5, 4, 100, 7], [12, 12, 12, 12], [5, 3, 1, 0]):
            p.cache.attend(1, q, out[1:13], ids(starts), p.cache.lens, ids(p.seqs))
            p.cache.append(0, q[:, :2], q[:, 2:], ids(starts), p.cache.lens, ids(p.seqs))
        assert torch.isnan(out[0]).all() and torch.isnan(out[13]).all()


def test_scores_far_below_zero():
    """A bias that puts every score below -1e30: the nearest key takes the weight."""
    p = Paged(2, 2, 64, 16, [40], seed=1)
    q = queries(40, 2, 64)
    out = attended(p, q, [40], torch.float32, slopes=[1e31, 1e35], prefix=[0], window=0)
    v = [p.rows(0, 1, g) for g in range(2)]
    assert all(torch.equal(out[j, h].cpu(), torch.from_numpy(v[h][j].astype(np.float32))) for j in range(40) for h in range(2))


def test_many_sequences():
    rng = np.random.default_rng(1)
    n_new = [int(x) for x in rng.integers(0, 4, 150)]
    lens = [n + int(x) for n, x in zip(n_new, rng.integers(0, 90, 150))]
    p = Paged(2, 1, 64, 16, lens, seed=2)
    q = queries(sum(n_new), 2, 64)
    check_rows(p, q, attended(p, q, n_new), n_new)


@pytest.mark.parametrize("most,H,G", [(3, 4, 1), (200, 2, 2)])
def test_many_long_sequences(most, H, G):
    """More sequences than a wavefront has lanes, some of them long: few rows each, and hundreds of some."""
    rng = np.random.default_rng(most)
    n_new = [int(x) for x in rng.integers(0, 4, 130)]
    n_new[7], n_new[70], n_new[129] = most, 1, most
    lens = [n + int(x) for n, x in zip(n_new, rng.integers(0, 600, 130))]
    lens[70], lens[129], lens[12] = 9000, 2500, n_new[12]
    p = Paged(H, G, 64, 256, lens, seed=2)
    q = queries(sum(n_new), H, 64)
    for kw in (dict(), dict(window=700, prefix=[int(x) for x in rng.integers(0, 20, 130)])):
        check_rows(p, q, attended(p, q, n_new, torch.float32, **kw), n_new, some=3, **kw)


def test_strided_rows():
    p = Paged(4, 2, 128, 64, [100, 30], seed=3)
    both = queries(24, 9, 128)
    q = both[:, 3:7]
    assert q.stride(0) == 9 * 128
    check_rows(p, q.contiguous(), attended(p, q, [20, 4]), [20, 4])


def test_a_row_is_what_a_decode_step_gives():
    """One token a sequence: the same attention as okv_decode_attn_static over the same pool."""
    H, G, d, T = 16, 4, 128, 32
    lens = [77, 640, 1, 300]
    p = Paged(H, G, d, T, lens, seed=12)
    q = queries(4, H, d)
    out, other = attended(p, q, [1] * 4, torch.float32), torch.empty((4, H, d), device=DEV)
    binding.okv_decode_attn_static(n_q_heads=H, n_kv_heads=G, head_dim=d, block_tokens=T, max_blocks_per_seq=p.cache.table.shape[1], max_ctx=0, out_dtype=1, B=4, pool=p.cache.pool[1],
                                   block_table=p.cache.table[torch.tensor(p.seqs, device=DEV)].contiguous(), ctx_lens=ids(lens), q=q, out=other,
                                   stream=torch.cuda.current_stream().cuda_stream)
    check_rows(p, q, out, [1] * 4)
    torch.testing.assert_close(out, other, rtol=0, atol=2e-3)      # (its weights have 11 bits)


@pytest.mark.parametrize("H,G,d", [(4, 2, 128), (3, 3, 64)])
def test_contiguous_pools(H, G, d):
    """Through the C entry points: sequences in slices of a pool."""
    S, C, lens, n_new = 3, 208, [208, 5, 130], [30, 5, 1]
    rng = np.random.default_rng(7)
    n = 2 * G * d * C * S
    pool = rng.standard_normal(n).astype(np.float16)
    layout = dict(kind="contiguous", G=G, d=d, C=C)
    kv = [rng.standard_normal((sum(n_new), G, d)).astype(np.float16) for _ in range(2)]
    want = kv_layout.bulk_append_scatter(pool.copy(), layout, [a - b for a, b in zip(lens, n_new)], n_new, *kv)
    dev, k, v, q = torch.from_numpy(pool).to(DEV), *[torch.from_numpy(x).to(DEV) for x in kv], queries(sum(n_new), H, d)
    out, at, starts = torch.empty_like(q), ids(lens), starts_of(n_new)
    c = binding.OkvLayerPool(H, G, d, 0, 0, C, S, 0, dev.data_ptr())
    r = binding.OkvRows(3, sum(n_new), None, starts.data_ptr(), at.data_ptr())
    ws = torch.empty(max(1, int(binding.lib().okv_chunk_workspace_bytes(ctypes.byref(c)))), dtype=torch.uint8, device=DEV)
    a = binding.OkvChunk(workspace=ws.data_ptr(), workspace_bytes=ws.numel())
    s = torch.cuda.current_stream().cuda_stream
    assert binding.lib().okv_rope_append(ctypes.byref(c), ctypes.byref(r), None, k.data_ptr(), v.data_ptr(), G * d, None, 0, None, 0, s) == 0
    assert binding.lib().okv_chunk_attn(ctypes.byref(c), ctypes.byref(r), ctypes.byref(a), q.data_ptr(), H * d, out.data_ptr(), s) == 0
    assert np.array_equal(dev.cpu().numpy(), want)

    class Contiguous:
        def rows(self, b, kv, g):
            return kv_layout.gather_rows(want, layout, b, kv, g, lens[b])

    p = Contiguous()
    p.H, p.G, p.d, p.lens = H, G, d, lens
    check_rows(p, q, out, n_new)


# ---- appending ------------------------------------------------------------------------------------

def check_append(p, n_new, rope_kw, positions=None, seed=1, q_in_place=False, strided=False):
    """Values and what is not turned are moved bit for bit; a turned number is a sum of two products of 32 bits, their factors off by 2^-22 at most (the angle's turn by 2^-25 of a turn, the sine by
    two units), rounded to 11 bits: 2^-11 of itself + 2^-20 (|x| + |y|) + the smallest number's half."""
    rng = np.random.default_rng(seed)
    H, G, d, N = p.H, p.G, p.d, sum(n_new)
    q, k, v = (rng.standard_normal((N, h, d)).astype(np.float16) for h in (H, G, G))
    dev = [torch.from_numpy(x).to(DEV) for x in (q, k, v)]
    if strided:
        dev = list(torch.cat(dev, 1).split([H, G, G], 1))
    out = dev[0] if q_in_place else torch.empty((N, H, d), dtype=torch.float16, device=DEV)
    rope, inv_freq, inter = None, np.zeros(0), False
    if rope_kw is not None:
        rope = Rope.of(**rope_kw, device=DEV)
        inv_freq = rope_kw.get("base", 10000.0) ** (-np.arange(0, rope_kw["rotated"], 2) / rope_kw["rotated"])
        inter = rope_kw.get("interleaved", False)
    p.cache.append(1, dev[1], dev[2], starts_of(n_new), p.cache.lens, ids(p.seqs), q=dev[0], q_out=out, rope=rope, positions=None if positions is None else ids(positions))
    places = [p.lens[b] - n + j for b, n in enumerate(n_new) for j in range(n)]
    angles = places if positions is None else positions
    want_pool = p.pool.astype(np.float64)
    turned = np.zeros(p.pool.shape, dtype=bool)
    kw, row = oracle.rotate(k, angles, inv_freq, inter), 0
    for b, n in enumerate(n_new):
        for j in range(n):
            if places[row] >= 0:
                for g in range(G):
                    a, z = p.offset(b, 0, g, places[row]), p.offset(b, 1, g, places[row])
                    want_pool[a:a + d], want_pool[z:z + d] = kw[row, g], v[row, g]
                    turned[a:a + 2 * len(inv_freq)] = True
            row += 1
    got = p.cache.pool[1].cpu().numpy().reshape(-1)
    assert np.array_equal(got[~turned], want_pool[~turned].astype(np.float16))
    size = 2.0 ** -20 * 2 * max(np.abs(k).max(), np.abs(q).max()) + 2.0 ** -25
    assert (np.abs(got - want_pool) <= 2.0 ** -11 * np.abs(want_pool) + size)[turned].all()
    qw = oracle.rotate(q, angles, inv_freq, inter)
    assert (np.abs(out.cpu().numpy() - qw) <= 2.0 ** -11 * np.abs(qw) + size).all()
    assert not torch.any(p.cache.pool[0])                    # the other layer


@pytest.mark.parametrize("rope", [None, dict(rotated=64), dict(rotated=64, interleaved=True), dict(rotated=16), dict(rotated=32, interleaved=True, base=500000.0), dict(rotated=48)], ids=str)
@pytest.mark.parametrize("H,G,d", HEADS)
def test_appended_rows(H, G, d, rope):
    if rope and rope["rotated"] == 64:
        rope = dict(rope, rotated=d)
    p = Paged(H, G, d, 32, [5, 40, 33, 64, 100], seed=d + H)
    check_append(p, [5, 1, 0, 64, 30], rope)


@pytest.mark.parametrize("T", (16, 256))
def test_appended_rows_that_are_strided_and_turned_in_place(T):
    check_append(Paged(8, 4, 128, T, [70, 300], seed=T), [70, 3], dict(rotated=128), strided=True, q_in_place=True)


def test_far_positions():
    """Angles of positions of millions, where 32 bits would be off by some tenths."""
    rng = np.random.default_rng(2)
    p = Paged(4, 2, 64, 16, [50], seed=1)
    check_append(p, [50], dict(rotated=64), positions=[int(x) for x in rng.integers(0, 1 << 24, 50)])


def test_rows_that_do_not_fit_are_not_stored():
    p = Paged(2, 2, 64, 16, [3, 20], seed=9)
    check_append(p, [5, 4], dict(rotated=64))                # two rows of tokens before 0: queries are turned, nothing is stored
    before = p.cache.pool.clone()
    k, q = (torch.ones((9, 2, 64), dtype=torch.float16, device=DEV) for _ in range(2))
    p.cache.append(1, k, k, ids([0, 5, 9]), p.cache.lens, ids([-1, 99]))
    assert torch.equal(p.cache.pool, before)
    p.cache.pages.status[3] = binding.OKV_ENOSPC             # pages could not be taken, and nobody has looked
    p.cache.append(1, k, k, ids([0, 5, 9]), p.cache.lens, ids(p.seqs), q=q, q_out=q, rope=Rope.of(64, device=DEV))
    assert torch.equal(p.cache.pool, before) and not torch.equal(q, k)
    p.cache.pages.status[3] = 0
    p.cache.append(1, k, k, ids([0, 3, 3]), p.cache.lens, ids(p.seqs))
    assert not torch.equal(p.cache.pool, before)


def test_pools_beyond_4_gib():
    """A page and rows of queries whose places pass 2^32 bytes."""
    T, G, d = 1024, 8, 128
    n_pages = 1200                                           # 4 MiB a page
    cache = Cache16(n_layers=1, n_q_heads=8, n_kv_heads=G, head_dim=d, page_tokens=T, n_pages=n_pages, max_seqs=1, max_pages_per_seq=2, device=DEV)
    cache.table[0] = ids([n_pages - 1, n_pages - 2])
    n = 1100
    cache.lens[0] = n
    g = torch.Generator(device=DEV).manual_seed(1)
    q, k, v = (torch.randn((n, G, d), generator=g, dtype=torch.float16, device=DEV) for _ in range(3))
    starts = ids([0, n])
    cache.append(0, k, v, starts, cache.lens)
    assert not cache.pool[0, :n_pages - 2].any()
    out = torch.empty_like(q)
    cache.attend(0, q, out, starts, cache.lens)
    for j in (0, 1, 500, 1099):
        s = torch.einsum("hd,khd->hk", q[j].double(), k[:j + 1].double()) / math.sqrt(d)
        want = torch.einsum("hk,khd->hd", torch.softmax(s, -1), v[:j + 1].double())
        torch.testing.assert_close(out[j].double(), want, rtol=2.0 ** -11, atol=2.0 ** -11 + 2.0 ** -12)      # weights and result, each half a step of numbers of up to 4


def test_captured_and_on_another_stream():
    """Append and attend in a graph, replayed with other lengths and rows, and between eager work."""
    H, G, d, T = 8, 2, 128, 32
    p = Paged(H, G, d, T, [400, 90], seed=5)
    n_new = [3, 40]
    rope, starts, seqs = Rope.of(d, device=DEV), starts_of(n_new), ids(p.seqs)
    q, k, v = queries(43, H, d, 1), queries(43, G, d, 2), queries(43, G, d, 3)
    turned, out = torch.empty_like(q), torch.empty_like(q)

    def step():
        p.cache.append(1, k, v, starts, p.cache.lens, seqs, q=q, q_out=turned, rope=rope)
        p.cache.attend(1, turned, out, starts, p.cache.lens, seqs, window=200)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        q.copy_(queries(43, H, d, 10 + i))
        k.copy_(queries(43, G, d, 20 + i))
        p.cache.lens[p.seqs[0]] = 400 - 50 * i
        starts.copy_(starts_of([3, 40] if i % 2 else [20, 23]))
        graph.replay()
        torch.randn(1 << 14, device=DEV).sum().item()
        replayed, pool = out.clone(), p.cache.pool.clone()
        step()
        assert torch.equal(out, replayed) and torch.equal(p.cache.pool, pool), i


def test_wrong_tensors_are_refused():
    p = Paged(4, 2, 64, 16, [20, 30])
    c, q, k = p.cache, queries(6, 4, 64), queries(6, 2, 64)
    starts, seqs, out = ids([0, 2, 6]), ids(p.seqs), torch.empty_like(queries(6, 4, 64))
    good = dict(layer=1, q=q, out=out, starts=starts, lens=c.lens, seqs=seqs)
    c.attend(**good)
    for bad in (dict(layer=2), dict(layer=-1), dict(q=q.float()), dict(q=q[:, :3]), dict(q=q.cpu()), dict(q=q[..., ::2]), dict(out=out[:5]), dict(out=out.bfloat16()), dict(out=out.cpu()),
                dict(starts=starts.long()), dict(starts=starts[:2]), dict(starts=starts.cpu()), dict(lens=c.lens[:2]), dict(lens=c.lens.long()), dict(seqs=seqs[:1]), dict(seqs=seqs.long()),
                dict(slopes=torch.ones(3, device=DEV)), dict(slopes=torch.ones(4, device=DEV, dtype=torch.float64)), dict(prefix=ids([1])), dict(prefix=torch.ones(4, device=DEV))):
        with pytest.raises(ValueError):
            c.attend(**{**good, **bad})
    with pytest.raises(ValueError):
        c.attend(**good, window=1 << 32)
    for bad in (dict(cap=-1.0), dict(cap=math.nan), dict(cap=1e-39), dict(scale=-0.5), dict(scale=1e-40), dict(scale=1e31), dict(window=-3)):
        with pytest.raises(binding.OkvError):
            c.attend(**{**good, **bad})
    rope = Rope.of(64, device=DEV)
    good = dict(layer=0, k=k, v=k, starts=starts, lens=c.lens, seqs=seqs, q=q, q_out=out, rope=rope)
    c.append(**good)
    for bad in (dict(k=q), dict(v=k[:5]), dict(v=torch.cat([k, k], 1)[:, :2]), dict(q=None), dict(q_out=None), dict(q_out=out.float()), dict(positions=ids([1] * 5)), dict(rope=None, positions=ids([1] * 6)),
                dict(rope=Rope(torch.ones(8, dtype=torch.float64))), dict(starts=ids([])), dict(seqs=ids([1]))):
        with pytest.raises(ValueError):
            c.append(**{**good, **bad})
    with pytest.raises(binding.OkvError):
        c.append(**{**good, "rope": Rope.of(80, device=DEV)})
    with pytest.raises(ValueError):
        Rope(torch.ones(8))
    with pytest.raises(ValueError):
        Rope(torch.ones(9, dtype=torch.float64))
    for bad in (dict(page_tokens=0), dict(page_tokens=8), dict(n_layers=0), dict(pool=torch.zeros(3, device=DEV, dtype=torch.float16)), dict(table=ids([1]))):
        with pytest.raises(ValueError):
            Cache16(**{**dict(n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=4, max_seqs=2, max_pages_per_seq=2, device=DEV), **bad})
    # nothing is done over nothing
    none = torch.empty((0, 4, 64), dtype=torch.float16, device=DEV)
    c.attend(1, none, torch.empty_like(none), ids([0]), c.lens, ids([]))
    c.append(1, none[:, :2], none[:, :2], ids([0, 0, 0]), c.lens, seqs)
