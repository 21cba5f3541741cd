"""The 8-bit KV cache against its definition in 64 bits.

Codes, scales and what is read back are exact (bits).  Attention: weights go into the second product with 22 bits and scores are fp32 sums of d
products whose magnitudes add up to some 8 sqrt(d) at most here, so an output vector is within d 2^-24 8 + a few 2^-22 of the definition: 7e-5, and
2^-11 more where it is rounded to fp16.
"""
import numpy as np
import pytest
import torch

from oracle import cache8 as oracle
from paper_2504_11816_amd import binding
from paper_2504_11816_amd.cache8 import Cache8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TILE = 32


def rows_of(rng, n, G, d):
    return (rng.standard_normal((n, G, d)) * np.exp(0.5 * rng.standard_normal((G, d)))).astype(np.float16)


def dev(x, dtype=None):
    return torch.tensor(np.ascontiguousarray(x), dtype=dtype, device=DEV)


def make(rng, lens, *, L=1, H=4, G=2, d=64, T=64, fmt="int8", fp32=True, spare=2, max_seqs=None):
    """A cache whose sequences will have `lens` tokens: random pages, everything that is not stored yet poisoned."""
    S, width = max_seqs or len(lens), max(1, max(-(-n // T) for n in lens)) + 1
    n_pages = sum(-(-n // T) for n in lens) + spare
    c = Cache8(n_layers=L, n_q_heads=H, n_kv_heads=G, head_dim=d, page_tokens=T, n_pages=n_pages, max_seqs=S, max_pages_per_seq=width, format=fmt,
               out_dtype=torch.float32 if fp32 else torch.float16, device=DEV)
    ids, table = list(rng.permutation(n_pages)), np.full((S, width), -1, np.int32)
    for b, n in enumerate(lens):
        for p in range(-(-n // T)):
            table[b, p] = ids.pop()
    c.table.copy_(dev(table))
    c.codes.fill_(0xff)                                      # the E4M3 code of NaN
    c.scales.fill_(float("nan"))
    c.tails.fill_(float("nan"))
    return c


def store(c, parts_k, parts_v, lens, seqs=None):
    starts = np.concatenate([[0], np.cumsum([p.shape[0] for p in parts_k])])
    full = torch.zeros(c.max_seqs, dtype=torch.int32, device=DEV)
    at = np.arange(len(lens)) if seqs is None else np.asarray(seqs)
    full[torch.tensor(at, device=DEV, dtype=torch.long)] = dev(lens, torch.int32)
    k, v = (dev(np.concatenate(p)[None].repeat(c.L, 0)) for p in (parts_k, parts_v))
    c.store(k, v, dev(starts, torch.int32), full, None if seqs is None else dev(seqs, torch.int32))
    return full


def tile_bits(c, lens):
    """The raw bits of everything that the sequences' tiles and tails hold."""
    table, out = c.table.cpu().numpy(), []
    codes, scales, tails = c.codes.cpu().numpy(), c.scales.cpu().numpy().view(np.uint32), c.tails.cpu().numpy().view(np.uint16)
    tpp = c.T // TILE
    for b, n in enumerate(lens):
        for t in range(n // TILE):
            page = table[b, t // tpp]
            out += [codes[:, page, t % tpp], scales[:, page, t % tpp]]
        out.append(tails[:, b, :, :, :n % TILE])
    return out


def equal(a, b):
    return all(np.array_equal(x, y) for x, y in zip(a, b, strict=True))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("d,G,T", [(64, 1, 32), (64, 5, 64), (128, 2, 128), (128, 12, 32)])
def test_store_and_load(fmt, d, G, T):
    rng = np.random.default_rng(d + G)
    lens = [1, 31, 32, 33, 64, 95, 200, 7]
    c = make(rng, lens, L=2, H=G, G=G, d=d, T=T, fmt=fmt)
    k, v = ([rows_of(rng, n, G, d) for n in lens] for _ in range(2))
    after = store(c, k, v, lens)
    starts = dev(np.concatenate([[0], np.cumsum(lens)]), torch.int32)
    out = [torch.full((2, sum(lens), G, d), float("nan"), dtype=torch.float16, device=DEV) for _ in range(2)]
    c.load(out[0], out[1], starts, after)
    for got, rows in zip(out, (k, v)):
        want = np.concatenate([oracle.held(r, fmt, r.shape[0] // TILE * TILE) for r in rows]).astype(np.float16)
        for layer in got.cpu().numpy():
            assert np.array_equal(layer, want)               # (values: a whole number has no -0)
    # the documented layout, byte by byte
    b, t = 6, 3
    page = int(c.table[b, t * TILE // T])
    raw = oracle.unpack(c.codes[1].cpu().numpy(), c.scales[1].cpu().numpy(), G=G, gg=binding.okv_kv_head_group(G, d), d=d, T=T, fmt=fmt, page=page, tile=t % (T // TILE))
    for kv, rows in enumerate((k, v)):
        assert np.array_equal(raw[kv], oracle.held(rows[b], fmt, 192)[t * TILE:(t + 1) * TILE])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_chunks_leave_the_same_bits(fmt):
    """A prompt at once; in chunks that begin and end anywhere, of some of the sequences, in another order; the last rows by decode steps."""
    rng = np.random.default_rng(7)
    lens, G, d, T = [130, 97, 64, 33], 3, 64, 64
    k, v = ([rows_of(rng, n, G, d) for n in lens] for _ in range(2))
    whole = make(np.random.default_rng(1), lens, G=G, H=G, d=d, T=T, fmt=fmt)
    store(whole, k, v, lens)
    want = tile_bits(whole, lens)
    chunks = make(np.random.default_rng(1), lens, G=G, H=G, d=d, T=T, fmt=fmt)
    done = [0, 0, 0, 0]
    for size in (1, 30, 2, 40, 5, 33, 64, 100):
        todo = [b for b in (2, 0, 3, 1) if done[b] < lens[b]]
        if not todo:
            break
        upto = [min(lens[b], done[b] + size) for b in todo]
        store(chunks, [k[b][done[b]:u] for b, u in zip(todo, upto)], [v[b][done[b]:u] for b, u in zip(todo, upto)], upto, seqs=todo)
        for b, u in zip(todo, upto):
            done[b] = u
    assert done == lens and equal(tile_bits(chunks, lens), want)
    steps = make(np.random.default_rng(1), lens, G=G, H=G, d=d, T=T, fmt=fmt)
    back = 35
    store(steps, [x[:max(0, len(x) - back)] for x in k], [x[:max(0, len(x) - back)] for x in v], [max(0, n - back) for n in lens])
    for i in range(back, 0, -1):
        seqs = [b for b in range(4) if lens[b] >= i]
        now = torch.zeros(4, dtype=torch.int32, device=DEV)
        now[seqs] = dev([lens[b] - i + 1 for b in seqs], torch.int32)
        out = torch.empty((1, len(seqs), G, d), device=DEV)
        steps.step(torch.zeros((1, len(seqs), G, d), dtype=torch.float16, device=DEV), dev(np.stack([k[b][lens[b] - i] for b in seqs])[None]),
                   dev(np.stack([v[b][lens[b] - i] for b in seqs])[None]), out, now, dev(seqs, torch.int32))
    assert equal(tile_bits(steps, lens), want)


def test_extreme_numbers():
    """The largest and the smallest fp16 numbers, tiles of zeros, and numbers that are none: those make their tile NaN and no other."""
    rng = np.random.default_rng(5)
    k = rows_of(rng, 192, 2, 64)
    k[0:32, 0] = 65504 * np.sign(k[0:32, 0])
    k[32:64, 0] = (rng.integers(-2, 3, (32, 64)) * 2.0 ** -24).astype(np.float16)
    k[64:96] = 0
    k[100, 1, 3] = np.inf
    k[130, 0, 0] = np.nan
    for fmt in ("int8", "e4m3"):
        c = make(rng, [192], G=2, H=2, d=64, fmt=fmt)
        after = store(c, [k], [k], [192])
        out = [torch.empty((1, 192, 2, 64), dtype=torch.float16, device=DEV) for _ in range(2)]
        c.load(out[0], out[1], dev([0, 192], torch.int32), after)
        with np.errstate(invalid="ignore"):
            want = np.stack([np.concatenate([oracle.held(k[t:t + 32, g:g + 1], fmt, 32) if np.isfinite(k[t:t + 32, g]).all() else np.full((32, 1, 64), np.nan)
                                             for t in range(0, 192, 32)])[:, 0] for g in range(2)], 1).astype(np.float16)
        for x in out:
            np.testing.assert_array_equal(x[0].cpu().numpy(), want)


def check_step(lens, *, H, G, d, T=64, fmt="int8", fp32=True, seed=0, max_seqs=None, seqs=None, strided=False, scale_q=1.0):
    """An appending step and one that appends nothing, against the definition."""
    rng = np.random.default_rng(seed)
    S = max_seqs or len(lens)
    seqs = list(range(len(lens))) if seqs is None else seqs
    by_row = [0] * S
    for s, n in zip(seqs, lens):
        by_row[s] = n
    c = make(rng, by_row, H=H, G=G, d=d, T=T, fmt=fmt, fp32=fp32, max_seqs=S)
    k, v = ([rows_of(rng, max(n, 1), G, d) for n in lens] for _ in range(2))
    store(c, [x[:max(n - 1, 0)] for x, n in zip(k, lens)], [x[:max(n - 1, 0)] for x, n in zip(v, lens)], [max(n - 1, 0) for n in lens], seqs=seqs)
    B = len(lens)
    q = (scale_q * rng.standard_normal((B, H, d))).astype(np.float16)
    kn, vn = (np.stack([x[max(n - 1, 0)] for x, n in zip(p, lens)]) for p in (k, v))
    now = torch.zeros(S, dtype=torch.int32, device=DEV)
    now[torch.tensor(seqs, device=DEV)] = dev(lens, torch.int32)
    ids = dev(seqs, torch.int32)
    out = torch.full((B, H, d), float("nan"), dtype=c.out_dtype, device=DEV)
    if strided:                                              # q, k and v as one product leaves them
        row = torch.full((B, (H + 2 * G) * d + 8), float("nan"), dtype=torch.float16, device=DEV)
        tq, tk, tv = (row[:, a * d:b * d].unflatten(1, (-1, d)) for a, b in ((0, H), (H, H + G), (H + G, H + 2 * G)))
        for t, x in ((tq, q), (tk, kn), (tv, vn)):
            t.copy_(dev(x))
    else:
        tq, tk, tv = dev(q), dev(kn), dev(vn)
    tol = 7e-5 + (0 if fp32 else 2.0 ** -11)
    for appends in (True, False):
        out.fill_(float("nan"))
        c.begin(B, now, ids, appends=appends)
        c.attend(0, tq, tk if appends else None, tv if appends else None, out)
        got = out.double().cpu().numpy()
        for b, n in enumerate(lens):
            want = oracle.attend(q[b], k[b], v[b], n, fmt, appends)
            if n == 0:
                assert (got[b] == 0).all()
                continue
            err = np.linalg.norm(got[b] - want, axis=1) / np.linalg.norm(want, axis=1)
            assert err.max() <= tol, (b, n, appends, err.max())


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("H,G,d", [(4, 4, 64), (1, 1, 128), (16, 1, 64), (15, 5, 128), (32, 2, 128), (20, 10, 64), (12, 12, 128)])
def test_decode_against_the_definition(fmt, H, G, d):
    check_step([1, 2, 31, 32, 33, 63, 64, 65, 200, 449], H=H, G=G, d=d, fmt=fmt, seed=H + d)


@pytest.mark.parametrize("T", [32, 128, 1024])
@pytest.mark.parametrize("fp32", [True, False])
def test_page_sizes_and_output_types(T, fp32):
    check_step([1025, 40, 5, 700], H=8, G=2, d=128, T=T, fp32=fp32, seed=T)


def test_empty_sequences_and_rows_of_the_table():
    check_step([0, 40, 0, 0, 65, 0], H=4, G=2, d=64, seed=3)
    check_step([0, 0], H=4, G=2, d=64, seed=4)
    check_step([70, 0, 33], H=4, G=2, d=64, seed=5, max_seqs=9, seqs=[7, 2, 0])


def test_strided_rows():
    check_step([70, 33, 64], H=6, G=2, d=64, strided=True, seed=6)
    check_step([70, 33, 64], H=5, G=5, d=128, strided=True, seed=7, fp32=False)


def test_scores_far_apart():
    check_step([300, 64, 1000], H=8, G=4, d=128, scale_q=30.0, seed=8)


@pytest.mark.parametrize("B", [65, 300])
def test_many_short_sequences(B):
    rng = np.random.default_rng(B)
    check_step([int(n) for n in rng.integers(0, 90, B)], H=2, G=2, d=64, T=32, seed=B)


@pytest.mark.parametrize("G,n", [(1, 9000), (8, 3000), (40, 800)])
def test_long_sequences_are_cut(G, n):
    check_step([n, 17, n // 2 + 1], H=2 * G, G=G, d=64, T=32, seed=G)


def test_more_pages_than_lanes_and_buffers_beyond_4_gib():
    """Two long sequences in the last pages of buffers of more than 2^32 bytes: page lists of more than 64 entries in 32-token pages."""
    rng = np.random.default_rng(11)
    G, d, T, n_pages = 8, 128, 32, 70000                     # 64 KiB a page: 4.6e9 bytes
    lens = [4500, 2300]
    c = Cache8(n_layers=1, n_q_heads=8, n_kv_heads=G, head_dim=d, page_tokens=T, n_pages=n_pages, max_seqs=2, max_pages_per_seq=150, out_dtype=torch.float32, device=DEV)
    ids, table = list(n_pages - 1 - rng.permutation(300)), np.full((2, 150), -1, np.int32)
    for b, n in enumerate(lens):
        for p in range(-(-n // T)):
            table[b, p] = ids.pop()
    c.table.copy_(dev(table))
    k, v = ([rows_of(rng, n, G, d) for n in lens] for _ in range(2))
    store(c, [x[:-1] for x in k], [x[:-1] for x in v], [n - 1 for n in lens])
    q, out = rng.standard_normal((1, 2, 8, d)).astype(np.float16), torch.empty((1, 2, 8, d), device=DEV)
    c.step(dev(q), dev(np.stack([x[-1] for x in k])[None]), dev(np.stack([x[-1] for x in v])[None]), out, dev(lens, torch.int32))
    for b, n in enumerate(lens):
        want = oracle.attend(q[0, b], k[b], v[b], n, "int8", True)
        err = np.linalg.norm(out[0, b].double().cpu().numpy() - want, axis=1) / np.linalg.norm(want, axis=1)
        assert err.max() <= 7e-5


def test_layers_in_one_call_are_the_layers_one_by_one():
    rng = np.random.default_rng(12)
    L, H, G, d, lens = 3, 8, 2, 128, [200, 64, 1, 95]
    a, b = (make(np.random.default_rng(2), lens, L=L, H=H, G=G, d=d, fp32=False) for _ in range(2))
    k, v = ([rows_of(rng, n - 1, G, d) for n in lens] for _ in range(2))
    for c in (a, b):
        store(c, k, v, [n - 1 for n in lens])
    q, kn, vn = (dev(rng.standard_normal((L, 4, h, d)).astype(np.float16)) for h in (H, G, G))
    now, oa, ob = dev(lens, torch.int32), torch.empty((L, 4, H, d), dtype=torch.float16, device=DEV), torch.empty((L, 4, H, d), dtype=torch.float16, device=DEV)
    a.step(q, kn, vn, oa, now)
    b.begin(4, now)
    for layer in range(L):
        b.attend(layer, q[layer], kn[layer], vn[layer], ob[layer])
    assert torch.equal(oa, ob) and equal(tile_bits(a, lens), tile_bits(b, lens))


def test_a_captured_step_and_another_stream():
    """A graph that raises the lengths and steps, replayed with eager work between, against eager steps on another stream."""
    rng = np.random.default_rng(13)
    H, G, d, lens = 8, 2, 64, [60, 31, 5]
    a, b = (make(np.random.default_rng(2), [n + 12 for n in lens], H=H, G=G, d=d) for _ in range(2))
    k, v = ([rows_of(rng, n, G, d) for n in lens] for _ in range(2))
    q, kn, vn = (dev(rng.standard_normal((1, 3, h, d)).astype(np.float16)) for h in (H, G, G))
    outs, nows = [torch.zeros((1, 3, H, d), device=DEV) for _ in range(2)], [dev(lens, torch.int32) for _ in range(2)]
    for c in (a, b):
        store(c, k, v, lens)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nows[0].add_(1)
        a.step(q, kn, vn, outs[0], nows[0])
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for i in range(6):
        graph.replay()
        torch.randn(1 << 16, device=DEV).sum().item()
        with torch.cuda.stream(other):
            nows[1].add_(1)
            b.step(q, kn, vn, outs[1], nows[1])
        torch.cuda.synchronize()
        assert torch.equal(nows[0], nows[1]) and torch.equal(outs[0], outs[1]), i
    assert equal(tile_bits(a, [n + 6 for n in lens]), tile_bits(b, [n + 6 for n in lens]))


def test_wrong_tensors_are_refused():
    c = make(np.random.default_rng(0), [40], G=2, H=4, d=64, fp32=False)
    q, k = torch.zeros((1, 1, 4, 64), dtype=torch.float16, device=DEV), torch.zeros((1, 1, 2, 64), dtype=torch.float16, device=DEV)
    out, now = torch.zeros_like(q), dev([40], torch.int32)
    for bad in (dict(q=q.float()), dict(q=q[:, :, :3]), dict(k_new=None), dict(k_new=k.cpu()), dict(out=out.float()), dict(lens=now.long()), dict(lens=now[:0]),
                dict(seqs=now.long())):
        args = dict(q=q, k_new=k, v_new=k, out=out, lens=now)
        args.update(bad)
        with pytest.raises(ValueError):
            c.step(**args)
    with pytest.raises(ValueError):
        c.store(k.float(), k, dev([0, 1], torch.int32), now)
    with pytest.raises(ValueError):
        c.store(k, k, dev([0, 1], torch.int64), now)
    with pytest.raises(ValueError):
        c.attend(0, q[0].transpose(0, 1), None, None, out[0])
    with pytest.raises(ValueError):
        Cache8(n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=64, page_tokens=32, n_pages=4, max_seqs=1, max_pages_per_seq=4, format="int4", device=DEV)
    with pytest.raises(binding.OkvError):
        Cache8(n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=80, page_tokens=32, n_pages=4, max_seqs=1, max_pages_per_seq=4, device=DEV)


@pytest.mark.parametrize("lens", [[0, 0, 70, 0, 33, 1, 300, 0], [0], [5], [1000] * 3 + [0] * 4 + [64] * 57, [31] * 64, [32] * 64, [40, 0, 700] * 25], ids=lambda x: f"{len(x)}x{x[0]}")
@pytest.mark.parametrize("H,G,d", [(8, 2, 64), (3, 3, 128)])
def test_steps_of_all_layers(lens, H, G, d):
    """okv8_decode_step: up to 64 sequences share their lengths out in the launch itself, more have them shared out by a launch before; sequences without
    a tile among others; a workspace for one layer only."""
    rng = np.random.default_rng(len(lens))
    L, B = 3, len(lens)
    c = make(rng, lens, L=L, H=H, G=G, d=d, T=32)
    k, v = ([rows_of(rng, max(n, 1), G, d) for n in lens] for _ in range(2))
    store(c, [x[:max(n - 1, 0)] for x, n in zip(k, lens)], [x[:max(n - 1, 0)] for x, n in zip(v, lens)], [max(n - 1, 0) for n in lens])
    q = rng.standard_normal((L, B, H, d)).astype(np.float16)
    kn, vn = (np.stack([x[max(n - 1, 0)] for x, n in zip(p, lens)])[None].repeat(L, 0) for p in (k, v))
    out, now = torch.empty((L, B, H, d), device=DEV), dev(lens, torch.int32)
    for appends, layers_abreast in ((True, L), (False, L), (False, 1)):
        if layers_abreast == 1:
            one = binding.Okv8Cache.from_buffer_copy(c.c)
            one.n_layers = 1
            c._step.workspace_bytes = binding.lib().okv8_workspace_bytes(one, B)
        out.fill_(float("nan"))
        c.step(dev(q), dev(kn) if appends else None, dev(vn) if appends else None, out, now)
        got = out.double().cpu().numpy()
        for b in sorted({0, 1, 2, B // 2, B - 2, B - 1} & set(range(B))):
            for layer in range(L):
                want = oracle.attend(q[layer, b], k[b], v[b], lens[b], "int8", appends)
                err = np.linalg.norm(got[layer, b] - want, axis=1) / np.maximum(np.linalg.norm(want, axis=1), 1e-30) if lens[b] else np.abs(got[layer, b])
                assert err.max() <= 7e-5, (b, layer, appends)
        assert np.isfinite(got).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("H,G,d", [(4, 2, 64), (3, 3, 128)])
@pytest.mark.parametrize("factors", [(0, 1, 0, 1, 0, 1), (1e4, 1e-4, 1, 0, 1e-4, 1e4), (1e-4, 1e4, 0, 1e-4, 1, 1e-4), (0, 0, 0, 0, 0, 0), (2e-6, 2e-6, 0, 2e-6, 0, 2e-6)])
def test_tiles_of_zeros_and_of_magnitudes_far_apart(fmt, H, G, d, factors):
    """A tile's V scale goes through the softmax's exponent and out of the sum again: tiles whose values are all zero count in the sum, and tiles of
    large and of small values add up.  Weights below 2^-14 of the largest scaled one lose at most 2^-24 of it, with each of 203 keys: 203 2^-24 = 1.3e-5
    of a vector on top of the 7e-5."""
    rng = np.random.default_rng(d)
    n = 32 * len(factors) + 11
    k, v = rows_of(rng, n, G, d), rows_of(rng, n, G, d) / 8
    for t, f in enumerate(factors):
        v[32 * t:32 * t + 32] = (v[32 * t:32 * t + 32].astype(np.float64) * f).astype(np.float16)
    if not any(factors):
        v[:] = 0
    assert np.isfinite(v).all()
    c = make(rng, [n], H=H, G=G, d=d, fmt=fmt)
    store(c, [k[:-1]], [v[:-1]], [n - 1])
    q, out = rng.standard_normal((1, 1, H, d)).astype(np.float16), torch.full((1, 1, H, d), float("nan"), device=DEV)
    c.step(dev(q), dev(k[None, -1:]), dev(v[None, -1:]), out, dev([n], torch.int32))
    got, want = out[0, 0].double().cpu().numpy(), oracle.attend(q[0, 0], k, v, n, fmt, True)
    err, size = np.linalg.norm(got - want, axis=1), np.linalg.norm(want, axis=1)
    assert (err <= 8.5e-5 * size).all(), (err / np.maximum(size, 1e-30)).max()


def test_numbers_that_are_none_stay_where_they_are():
    """A NaN in one tile of one KV head makes that sequence's results of that head NaN, though other pieces of it are joined with the one that has it;
    a query head that has one makes its own NaN; nothing else changes by a bit."""
    rng = np.random.default_rng(21)
    lens, H, G, d = [3000, 500, 40], 4, 2, 64
    k, v = ([rows_of(rng, n, G, d) for n in lens] for _ in range(2))
    q = rng.standard_normal((1, 3, H, d)).astype(np.float16)

    def results(k, v, q):
        c = make(np.random.default_rng(1), lens, H=H, G=G, d=d)
        store(c, k, v, lens)
        out = torch.full((1, 3, H, d), 7.0, device=DEV)
        c.step(dev(q), None, None, out, dev(lens, torch.int32))
        return out[0].cpu().numpy()

    plain = results(k, v, q)
    assert np.isfinite(plain).all()
    for what in ("k", "v", "tail", "q nan", "q inf"):
        kk, vv, qq = [x.copy() for x in k], [x.copy() for x in v], q.copy()
        bad = np.zeros((3, H), bool)
        if what == "k":
            kk[0][1000, 1, 5], bad[0, 2:] = np.nan, True
        elif what == "v":
            vv[1][37, 0, 9], bad[1, :2] = np.inf, True
        elif what == "tail":
            kk[2][39, 0, 3], bad[2, :2] = np.nan, True
        else:
            qq[0, 1, 3, 7], bad[1, 3] = np.nan if what == "q nan" else np.inf, True
        got = results(kk, vv, qq)
        assert np.isnan(got[bad]).all(), what
        assert np.array_equal(got[~bad], plain[~bad]), what


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("size", [1.0, 1e-3, 1e-5])
@pytest.mark.parametrize("zeros", [(0,), (0, 2, 4), (3,), (5,), (0, 1, 2, 3, 4)])
def test_small_values_beside_tiles_of_zeros(fmt, size, zeros):
    """Keys of zero values count in the sum and take nothing from the others' accuracy, however small those are; every key in a whole tile, so that no
    fp16 tail is a part of the result.  The weights have their 22 bits: 7e-5 as elsewhere."""
    rng = np.random.default_rng(17)
    n, H, G, d = 192, 4, 2, 64
    k, v = rows_of(rng, n, G, d), (rows_of(rng, n, G, d).astype(np.float64) * size).astype(np.float16)
    for t in zeros:
        v[32 * t:32 * t + 32] = 0
    c = make(rng, [n, n], H=H, G=G, d=d, fmt=fmt)
    store(c, [k, k], [v, v], [n, n])
    q, out = rng.standard_normal((1, 2, H, d)).astype(np.float16), torch.full((1, 2, H, d), float("nan"), device=DEV)
    c.step(dev(q), None, None, out, dev([n, n], torch.int32))
    for b in range(2):
        got, want = out[0, b].double().cpu().numpy(), oracle.attend(q[0, b], k, v, n, fmt, False)
        assert (np.linalg.norm(got - want, axis=1) <= 7e-5 * np.linalg.norm(want, axis=1)).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("B,H,G,d,hi", [(3, 8, 2, 128, 960), (40, 16, 8, 64, 450), (1, 16, 1, 64, 900), (70, 6, 3, 64, 900), (30, 30, 30, 128, 500), (33, 8, 8, 128, 900)])
def test_short_sequences_by_table_width(fmt, B, H, G, d, hi):
    """Tables that hold up to 1024 keys, with few and with many (sequence, KV head) pairs, a layer at a time and two at once; the same sequences under
    a wider table, which are cut.  Both are within the tolerance of the definition, as the head of the file derives it."""
    rng = np.random.default_rng(B + hi)
    lens = [int(x) for x in rng.integers(0, hi + 1, B)]
    lens[0] = hi // 32 * 32
    k, v = ([rows_of(rng, max(n, 1), G, d) for n in lens] for _ in range(2))
    q = rng.standard_normal((2, B, H, d)).astype(np.float16)
    kn, vn = (np.stack([x[max(n - 1, 0)] for x, n in zip(p, lens)])[None].repeat(2, 0) for p in (k, v))
    now = dev(lens, torch.int32)
    picked = sorted({0, 1 % B, B // 2, B - 1})
    want = {(layer, b, appends): oracle.attend(q[layer, b], k[b], v[b], lens[b], fmt, appends) for layer in range(2) for b in picked for appends in (True, False)}
    for width in (None, 2200):
        c = make(np.random.default_rng(3), lens + ([0] if width is None else [width]), L=2, H=H, G=G, d=d, T=32, fmt=fmt)
        store(c, [x[:max(n - 1, 0)] for x, n in zip(k, lens)], [x[:max(n - 1, 0)] for x, n in zip(v, lens)], [max(n - 1, 0) for n in lens], seqs=list(range(B)))
        out = torch.empty((2, B, H, d), device=DEV)
        for appends in (True, False):
            out.fill_(float("nan"))
            c.step(dev(q), dev(kn) if appends else None, dev(vn) if appends else None, out, now)
            got = [out.double().cpu().numpy()]
            if not appends:
                out.fill_(float("nan"))
                c.begin(B, now, appends=False)
                for layer in range(2):
                    c.attend(layer, dev(q[layer]), None, None, out[layer])
                got.append(out.double().cpu().numpy())
            for x in got:
                assert np.isfinite(x).all()
                for layer in range(2):
                    for b in picked:
                        w = want[layer, b, appends]
                        assert (np.linalg.norm(x[layer, b] - w, axis=1) <= 7e-5 * np.linalg.norm(w, axis=1)).all(), (width, layer, b, appends)


def test_the_current_device_by_its_short_name():
    c = Cache8(n_layers=1, n_q_heads=2, n_kv_heads=2, head_dim=64, page_tokens=32, n_pages=3, max_seqs=1, max_pages_per_seq=3, device="cuda")
    assert c.device == c.codes.device == c.table.device
    c.pages.extend(dev([0], torch.int32), dev([40], torch.int32))
    assert c.lens.tolist() == [40]


@pytest.mark.parametrize("layerwise", [False, True])
@pytest.mark.parametrize("width", [4, 60])
def test_a_step_that_lacks_pages_writes_nothing(layerwise, width):
    """Two sequences share a full page and both need another, of which there is one: the call that takes pages changes nothing, and neither does the
    step behind it, in any page, tail or length.  When a page has been freed, the same step goes as if it were the first."""
    rng = np.random.default_rng(8)
    H, G, d, T, L = 4, 2, 64, 32, 2

    def start(n_pages):
        c = Cache8(n_layers=L, n_q_heads=H, n_kv_heads=G, head_dim=d, page_tokens=T, n_pages=n_pages, max_seqs=4, max_pages_per_seq=width, out_dtype=torch.float32, device=DEV)
        c.pages.extend(dev([0, 3], torch.int32), dev([T, 5], torch.int32))
        c.pages.fork(dev([0], torch.int32), dev([1], torch.int32))
        c.codes.copy_(codes[:, :n_pages])
        c.scales.copy_(scales[:, :n_pages])
        c.tails.copy_(tails)
        c.pages.check()
        return c

    codes = dev(rng.integers(1, 255, (L, 6, T // 32, 2 * G * 32 * d)), torch.uint8)
    scales, tails = dev(rng.random((L, 6, T // 32, 2 * G)), torch.float32), dev(rng.standard_normal((L, 4, 2, G, 32, d)).astype(np.float16))
    seqs = dev([0, 1], torch.int32)
    q, kn, vn = (dev(rng.standard_normal((L, 2, h, d)).astype(np.float16)) for h in (H, G, G))

    def step(c):
        out = torch.full((L, 2, H, d), float("nan"), device=DEV)
        c.pages.extend(seqs)
        if layerwise:
            c.begin(2, c.lens, seqs)
            for layer in range(L):
                c.attend(layer, q[layer], kn[layer], vn[layer], out[layer])
        else:
            c.step(q, kn, vn, out, c.lens, seqs)
        return out

    c = start(3)                                             # page 0 shared, page 1 of sequence 3, page 2 free
    before = [x.clone() for x in (c.codes, c.scales, c.tails, c.table, c.lens, c.refs)]
    step(c)
    with pytest.raises(binding.OkvError):
        c.pages.check()
    for x, y in zip(before, (c.codes, c.scales, c.tails, c.table, c.lens, c.refs)):
        assert torch.equal(x, y)
    # a prompt's chunk that finds no room, and is stored all the same
    more = dev(rng.standard_normal((L, 100, G, d)).astype(np.float16))
    c.pages.extend(dev([0], torch.int32), dev([100], torch.int32))
    c.store(more, more, dev([0, 100], torch.int32), c.lens, dev([0], torch.int32))
    with pytest.raises(binding.OkvError):
        c.pages.check()
    for x, y in zip(before, (c.codes, c.scales, c.tails, c.table, c.lens, c.refs)):
        assert torch.equal(x, y)
    c.pages.free(dev([3], torch.int32))
    roomy = start(6)
    assert torch.equal(step(c), step(roomy))
    c.pages.check()
    roomy.pages.check()
    assert c.lens.tolist()[:2] == [T + 1, T + 1] and torch.equal(c.tails[:, :2], roomy.tails[:, :2])
