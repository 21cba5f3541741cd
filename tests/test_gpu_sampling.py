"""Probabilities of logits, verification of drafted tokens and the pages of what was rejected, against 64 bits and plain lists."""
import math

import numpy as np
import pytest
import torch

from oracle import chunk as oracle
from oracle import pages as oracle_pages
from paper_2504_11816_amd import binding
from paper_2504_11816_amd.pages import PageArray, Pages, RowArray
from paper_2504_11816_amd.sampling import Sampler

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
VOCABS = [1, 2, 63, 64, 65, 1000, 2047, 2048, 2049, 4100, 32000, 50001, 131072, 200003]


def ids(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def check_probs(logits, t, got):
    """An exponent x / t log2(e) is off by 3 units of 2^-24 of itself, which is at most S = (largest - smallest that counts) / t; its exponential by 2 units, a sum of n numbers by n 2^-24
    (terms are positive), the quotient by 2: 2^-24 (3 S + 8 + n / 64 + 20) of the result, where a lane adds n / 1024 of them one after the other (n / 64 is more).  What lies below 2^-126 may be 0."""
    x, p = logits.float().cpu().numpy().astype(np.float64), got.cpu().numpy().astype(np.float64)
    for r in range(len(x)):
        temp = 1.0 if t is None else float(t[r])
        want = oracle.probs(x[r], temp)
        if temp == 0 or not np.isfinite(want).all():
            assert np.array_equal(p[r], want, equal_nan=True), r
            continue
        S = 0.0 if x[r].max() == -math.inf else np.where(x[r] == -math.inf, 0, x[r].max() - x[r]) / temp * 1.4427
        tol = 2.0 ** -24 * (3 * S + 3 * min(np.max(S), 40.0) + 28 + len(x[r]) / 64) * want + 2.0 ** -126
        assert (np.abs(p[r] - want) <= tol).all(), (r, temp, float((np.abs(p[r] - want) / tol).max()))


@pytest.mark.parametrize("dtype", (torch.float16, torch.float32), ids=str)
@pytest.mark.parametrize("vocab", VOCABS)
def test_probabilities(vocab, dtype):
    rows = 9 if vocab < 40000 else 4
    g = torch.Generator(device=DEV).manual_seed(vocab)
    for n in (rows, 1):
        x = (torch.randn((n, vocab), generator=g, device=DEV) * 4).to(dtype)
        t = torch.tensor([1.0, 0.7, 0.0, 0.05, 3.0, 0.0, 1.3, 10.0, 0.3][:n], device=DEV)
        out = torch.full((n, vocab), math.nan, device=DEV)
        s = Sampler(max_batch=rows, vocab=vocab, device=DEV)
        s.probs(x, out, t)
        check_probs(x, t, out)
        s.probs(x, out)
        check_probs(x, None, out)


def test_ties_go_to_the_first():
    for vocab in (5, 3000, 140000):
        x = torch.zeros((3, vocab), dtype=torch.float16, device=DEV)
        x[1, vocab // 2:] = 3
        x[2, :] = -2
        out = torch.empty((3, vocab), device=DEV)
        Sampler(max_batch=3, vocab=vocab, device=DEV).probs(x, out, torch.zeros(3, device=DEV))
        assert out.argmax(-1).tolist() == [0, vocab // 2, 0] and torch.equal(out.sum(-1), torch.ones(3, device=DEV))


@pytest.mark.parametrize("vocab", (7, 5000, 140000))
def test_infinities_and_nan_among_logits(vocab):
    for dtype in (torch.float16, torch.float32):
        x = torch.randn((8, vocab), device=DEV).to(dtype)
        x[0, ::2] = -math.inf
        x[1] = -math.inf
        x[2, 3] = math.nan
        x[3, 2] = math.inf
        x[4] = -math.inf
        x[5, 4] = math.inf
        x[6] = -math.inf
        x[6, vocab - 1] = -60000
        t = torch.tensor([0.8, 1, 1, 1, 0, 0, 0.5, -1], device=DEV)
        out = torch.empty((8, vocab), device=DEV)
        Sampler(max_batch=8, vocab=vocab, device=DEV).probs(x, out, t)
        check_probs(x[:1], t[:1], out[:1])
        assert not out[1].any() and out[2].isnan().all() and out[3].isnan().all() and not out[4].any() and out[7].isnan().all()
        assert out[5].nonzero().tolist() == [[4]] and out[6].nonzero().tolist() == [[vocab - 1]] and float(out[6, -1]) == 1


def test_strided_logits():
    x = torch.randn((6, 5003), device=DEV).half()
    out = torch.full((6, 6000), 7.0, device=DEV)
    for at in (0, 1, 2, 3):
        Sampler(max_batch=6, vocab=5000, device=DEV).probs(x[:, at:at + 5000], out[:, 5:5005])
        check_probs(x[:, at:at + 5000], None, out[:, 5:5005])
        assert (out[:, :5] == 7).all() and (out[:, 5005:] == 7).all()


@pytest.mark.parametrize("dtype", (torch.float16, torch.float32), ids=str)
@pytest.mark.parametrize("at, to, columns", [(0, 4, 40004), (1, 5, 40009), (3, 4, 40010), (0, 1, 40004)])
def test_long_rows_that_are_strided(at, to, columns, dtype):
    """Rows whose places are aligned for wide stores, and others."""
    x = torch.randn((5, 40003), device=DEV).to(dtype)
    out = torch.full((5, columns), 7.0, device=DEV)
    Sampler(max_batch=5, vocab=39998, device=DEV).probs(x[:, at:at + 39998], out[:, to:to + 39998])
    check_probs(x[:, at:at + 39998], None, out[:, to:to + 39998])
    assert (out[:, :to] == 7).all() and (out[:, to + 39998:] == 7).all()


def test_more_long_rows_than_a_grid_has():
    rows, vocab = 32770, 32800
    x = torch.randn((rows, vocab), device=DEV, dtype=torch.float16)
    out = torch.empty((rows, vocab), device=DEV)
    t = torch.ones(rows, device=DEV)
    t[32768] = 0.5
    Sampler(max_batch=rows, vocab=vocab, device=DEV).probs(x, out, t)
    some = [0, 1, 20000, 32767, 32768, 32769]
    check_probs(x[some], t[some], out[some])


# ---- verification ---------------------------------------------------------------------------------

def inputs(vocab, n, seed, peaked=1.5, agree=0.7):
    """Distributions of drafts and target that agree more or less; starts as the entry point takes them."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    N, B = sum(n), len(n)
    draft = torch.softmax(peaked * torch.randn((N, vocab), generator=g, device=DEV), -1)
    target = torch.softmax(peaked * torch.randn((N + B, vocab), generator=g, device=DEV), -1)
    row = 0
    for b, k in enumerate(n):
        for i in range(k):
            target[row + b] = agree * draft[row] + (1 - agree) * target[row + b]
            row += 1
    drafts = torch.multinomial(draft, 1, generator=g)[:, 0].int() if N else ids([])
    return target, draft, drafts, torch.rand((N + B,), generator=g, device=DEV)


def check(vocab, n, target, draft, drafts, uniforms, sampler=None):
    N, B = sum(n), len(n)
    tokens, accepted, rejected = (torch.full((k,), -7, dtype=torch.int32, device=DEV) for k in (N + B, B, B))
    starts = ids(np.concatenate([[0], np.cumsum(n)]))
    (sampler or Sampler(max_batch=B, vocab=vocab, device=DEV)).verify(target, drafts, starts, uniforms, tokens, accepted, rejected, draft_probs=draft)
    p, q, x, u = (None if t is None else t.cpu().numpy() for t in (target, draft, drafts, uniforms))
    want, counts, row = [], [], 0
    for b, k in enumerate(n):
        t, a = oracle.verify(p[row + b:row + b + k + 1], None if q is None else q[row:row + k], x[row:row + k], u[row + b:row + b + k + 1])
        want += t
        counts.append(a)
        row += k
    assert accepted.tolist() == counts and rejected.tolist() == [k - a for k, a in zip(n, counts)]
    assert tokens.tolist() == want
    return counts


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("sampled", (True, False))
def test_verification(vocab, sampled):
    n = [3, 0, 1, 8, 5, 2] if vocab < 40000 else [2, 0, 4]
    counts = []
    for seed in range(4):
        target, draft, drafts, u = inputs(vocab, n, seed)
        counts += check(vocab, n, target, draft if sampled else None, target[:sum(n)].argmax(-1).int() if not sampled and seed % 2 else drafts, u)
    assert vocab < 60 or not sampled or len(set(counts)) > 1


def test_certain_drafts_that_are_accepted():
    """Drafts that the target is nearly sure of."""
    n, counts = [6, 3, 0, 7], []
    for seed in range(4):
        target, draft, _, u = inputs(5000, n, seed, peaked=6.0, agree=1.0)
        counts += check(5000, n, target, None, draft.argmax(-1).int(), u)
    assert len(set(counts)) > 2


def test_more_drafts_than_lanes():
    n = [130, 64, 65, 0, 1]
    target, draft, drafts, u = inputs(50, n, 1, agree=1.0)
    u[:131] *= 0.999
    check(50, n, target, draft, drafts, u)
    target[100, int(drafts[100])] = 0
    assert check(50, n, target, draft, drafts, u)[0] <= 100


def test_borders():
    """Random numbers at the borders between tokens, and drafts whose product is the target's probability."""
    V = 4096
    p = torch.full((2, V), 1 / V, device=DEV)                # sums are exact
    for k in (0, 1, 2047, 2048, 4095):
        u = torch.tensor([0.5, k / V], device=DEV)
        drafts = ids([3])
        assert check(V, [1], p, p[:1].clone(), drafts, u) == [1]
        check(V, [0], p[:1], None, ids([]), u[1:])
    q = p.clone()[:1]
    q[0, 3] = 2 / V
    for u0, want in ((0.5, 0), (np.nextafter(np.float32(0.5), np.float32(0)), 1)):
        assert check(V, [1], p, q, ids([3]), torch.tensor([u0, 0.25], device=DEV, dtype=torch.float32)) == [want]


def test_weights_that_do_not_count():
    V = 3000
    target, draft, drafts, u = inputs(V, [1, 1, 1, 1, 2], 5)
    target[0] = 0                                            # nothing to draw from
    target[2, 1000] = math.nan
    target[2, 1001] = math.inf
    target[2, 1002] = -5
    drafts[1] = 1000
    target[4] = draft[2]                                     # nothing above the draft
    drafts[2] = V                                            # no such token
    drafts[3] = -1
    target[8, int(drafts[4])] = 1
    check(V, [1, 1, 1, 1, 2], target, draft, drafts, u)
    check(V, [1, 1, 1, 1, 2], target, None, drafts, u)


def test_strided_tables():
    V, n = 1001, [2, 3]
    target, draft, drafts, u = inputs(V, n, 3)
    wide, wider = torch.empty((7, V + 9), device=DEV), torch.empty((5, V + 3), device=DEV)
    wide[:, 4:4 + V], wider[:, 1:1 + V] = target, draft
    check(V, n, wide[:, 4:4 + V], wider[:, 1:1 + V], drafts, u)


def test_captured_verification():
    V, n = 9000, [3, 2, 4]
    target, draft, drafts, u = inputs(V, n, 8)
    s, starts = Sampler(max_batch=3, vocab=V, device=DEV), ids([0, 3, 5, 9])
    logits, outs = torch.log(target), [torch.empty(k, dtype=torch.int32, device=DEV) for k in (12, 3, 3)]
    probs, wide = torch.empty_like(target), Sampler(max_batch=12, vocab=V, device=DEV)

    def step():
        wide.probs(logits, probs)
        s.verify(probs, drafts, starts, u, *outs, draft_probs=draft)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        u.copy_(torch.rand(12, generator=torch.Generator(device=DEV).manual_seed(i), device=DEV))
        graph.replay()
        torch.randn(1 << 14, device=DEV).sum().item()
        got = [x.tolist() for x in outs]
        step()
        assert got == [x.tolist() for x in outs]
        check(V, n, probs, draft, drafts, u)


def test_wrong_tensors_are_refused():
    V, n = 50, [2, 1]
    target, draft, drafts, u = inputs(V, n, 0)
    s = Sampler(max_batch=2, vocab=V, device=DEV)
    i32 = [torch.empty(k, dtype=torch.int32, device=DEV) for k in (5, 2, 2)]
    good = dict(target=target, drafts=drafts, starts=ids([0, 2, 3]), uniforms=u, tokens=i32[0], accepted=i32[1], rejected=i32[2], draft_probs=draft)
    s.verify(**good)
    s.verify(**{**good, "rejected": None})
    for bad in (dict(target=target[:4]), dict(target=target.half()), dict(target=target.cpu()), dict(target=target[:, ::2]), dict(drafts=drafts.long()), dict(drafts=drafts[:2]), dict(starts=ids([0, 2, 3, 3])),
                dict(starts=ids([])), dict(uniforms=u[:3]), dict(uniforms=u.double()), dict(tokens=i32[0][:4]), dict(accepted=i32[1][:1]), dict(rejected=i32[0]), dict(draft_probs=draft[:2])):
        with pytest.raises(ValueError):
            s.verify(**{**good, **bad})
    x, out = torch.zeros((2, V), device=DEV), torch.empty((2, V), device=DEV)
    for bad in ((x.double(), out), (x, out.half()), (x[:, 1:], out), (x, out[:1]), (x, out, torch.ones(3, device=DEV)), (x, out, torch.ones(2)), (torch.zeros((3, V), device=DEV), torch.empty((3, V), device=DEV))):
        with pytest.raises(ValueError):
            s.probs(*bad)
    with pytest.raises(binding.OkvError):
        Sampler(max_batch=1, vocab=0, device=DEV)


# ---- pages ----------------------------------------------------------------------------------------

class Shrunk:
    def __init__(self, rows=None, S=6, width=9, T=16, n_pages=40):
        self.table = torch.full((S, width), -1, dtype=torch.int32, device=DEV)
        self.lens, self.refs = (torch.zeros(n, dtype=torch.int32, device=DEV) for n in (S, n_pages))
        arrays = [PageArray(torch.zeros((1, n_pages, T), dtype=torch.int32, device=DEV), 1)]
        self.counts = [] if rows is None else [rows]
        tails = [] if rows is None else [RowArray(torch.zeros((1, S, 2, rows, 4), dtype=torch.int32, device=DEV), 2, rows)]
        self.pages = Pages(table=self.table, lens=self.lens, refs=self.refs, page_tokens=T, arrays=arrays, rows=tails)
        self.model = oracle_pages.Model(n_pages, T, S, width)

    def do(self, name, *args):
        getattr(self.pages, name)(*[ids(x) for x in args])
        getattr(self.model, name)(*args, *([self.counts] if name == "shrink" else []))
        assert (self.table.tolist(), self.lens.tolist(), self.refs.tolist(), self.pages.status.tolist()[0]) == (self.model.table, self.model.lens, self.model.refs, self.model.status)

    def refused(self):
        assert self.model.status == binding.OKV_ESTATE
        with pytest.raises(binding.OkvError):
            self.pages.check()
        self.model.status = 0


def test_shortened_sequences():
    p = Shrunk()
    p.do("extend", [0, 1, 2], [100, 16, 33])
    p.do("shrink", [0, 1, 2], [0, 1, 2])
    p.do("shrink", [2, 0], [31, 60])
    p.do("shrink", [99, -1, 0], [5, 5, 1])
    p.do("extend", [3], [140])
    p.do("shrink", [1, 3, 0], [15, 140, 39])
    assert not p.lens.any() and not p.refs.any()
    p.do("shrink", [0], [-4])
    p.do("shrink", [0, 1], [0, 1])                           # more than there is
    p.refused()


def test_shared_pages_are_not_cut():
    p = Shrunk()
    p.do("extend", [0], [40])
    p.do("fork", [0, 0], [1, 2])
    p.do("shrink", [1], [8])                                 # its own last page
    p.do("shrink", [0, 1], [1, 3])
    p.refused()                                              # (all or nothing)
    p.do("shrink", [1], [16])
    p.do("free", [0])
    p.do("shrink", [2], [24])
    p.do("shrink", [1], [3])
    p.refused()
    p.do("free", [2])
    p.do("shrink", [1], [3])
    assert p.lens.tolist()[1] == 13


def test_rows_beside_pages():
    p = Shrunk(rows=8)
    p.do("extend", [0, 1], [43, 40])
    p.do("shrink", [0, 1], [2, 8])
    p.do("shrink", [0], [1])
    p.do("shrink", [0], [1])
    p.refused()
    p.do("shrink", [0], [8])
    p.do("extend", [0], [7])
    p.do("shrink", [0], [3])


def test_nothing_is_taken_back_that_was_refused():
    """A step whose pages could not be taken added nothing: giving its rejected tokens back must not shorten what was there."""
    p = Shrunk(n_pages=4)
    p.do("extend", [0, 1], [20, 30])
    p.do("extend", [0, 1], [5, 5])                           # no page is left for both
    assert p.model.status == binding.OKV_ENOSPC
    p.do("shrink", [0, 1], [4, 2])
    assert p.lens.tolist()[:2] == [20, 30]
    with pytest.raises(binding.OkvError):
        p.pages.check()
    p.model.status, p.model.refused = 0, False
    p.do("shrink", [0, 1], [4, 2])


def test_many_sequences_shrink_at_once():
    rng = np.random.default_rng(0)
    p = Shrunk(S=1500, width=5, n_pages=7000)
    n = [int(x) for x in rng.integers(0, 75, 1500)]
    p.do("extend", list(range(1500)), n)
    p.do("shrink", list(range(1500)), [int(rng.integers(0, k + 1)) for k in n])
    p.do("extend", list(range(1500)), [3] * 1500) if max(p.model.lens) <= 77 else None


def test_captured_shrinking():
    p = Shrunk()
    p.do("extend", [0, 1], [50, 20])
    p.do("shrink", [0, 1], [1, 1])
    more, less, both = ids([5, 5]), ids([4, 2]), ids([0, 1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.pages.extend(both, more)
        p.pages.shrink(both, less)
    for _ in range(5):
        graph.replay()
        torch.randn(1 << 14, device=DEV).sum().item()
        p.model.extend([0, 1], [5, 5])
        p.model.shrink([0, 1], [4, 2])
        assert (p.table.tolist(), p.lens.tolist(), p.refs.tolist()) == (p.model.table, p.model.lens, p.model.refs)
