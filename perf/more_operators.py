"""The operators of a step in which several tokens of a sequence come at once (a prompt in chunks, drafted tokens), as cases that can be timed and checked.

  append   rows of a batch go into the paged fp16 cache, keys rotated by their positions on the way, queries rotated beside them
  chunk    every row of a batch attends over its sequence's cache up to itself: cap, distance bias, window and prefix as the case has them
  probs    rows of logits become probabilities, each row with its temperature
  verify   drafted tokens are held against the target's probabilities with given random numbers, and what was rejected leaves the cache's pages

`own` False: plain tensor operations, in 32 bits (64 for angles, and for sums that a random number is compared with), rounded once at the end.  `own` True: the
library's entry points.

The cache: pages of T tokens, each a row of slabs of 16 St tokens laid out [G / Gg][K, V][St][Gg][16][d]; Gg is the largest divisor of G with Gg d <= 1024, St the
largest power of two with St Gg d <= 1024 that divides T / 16.
"""
import math

import torch

own = False

DEV = "cuda:0"


# ---- cases ----------------------------------------------------------------------------------------

def listed():
    return [
        # four sequences of a small model, a handful of drafted tokens each: launches are all it costs
        dict(name="append_drafts", kind="append", H=8, G=8, d=64, T=32, B=4, lo=1, hi=5, before=300, lens_seed=1, rot=64, interleaved=False),
        # a batch of prompts, grouped heads, at positions where an angle needs more than 32 bits
        dict(name="append_prompts", kind="append", H=32, G=8, d=128, T=64, B=24, lo=100, hi=2000, before=100000, lens_seed=2, rot=128, interleaved=False),
        # the smallest attention: one layer of 8 heads x 64, four sequences of some 300 keys, 1 to 5 tokens each
        dict(name="chunk_small", kind="chunk", H=8, G=8, d=64, T=32, B=4, lo=1, hi=5, before=300, lens_seed=3, cap=0.0, window=0, slopes=False, prefix=0, fp32=False),
        # verification in the middle of a generation: 5 tokens for each of 32 sequences, contexts of up to 4096
        dict(name="chunk_drafts", kind="chunk", H=32, G=8, d=128, T=64, B=32, lo=5, hi=5, before=4096, lens_seed=4, cap=0.0, window=0, slopes=False, prefix=0, fp32=False),
        # a chunk of one long document
        dict(name="chunk_document", kind="chunk", H=32, G=8, d=128, T=128, B=1, lo=512, hi=512, before=100000, lens_seed=5, cap=0.0, window=0, slopes=False, prefix=0, fp32=False),
        # prompts from their beginning, a head of keys for every query head
        dict(name="chunk_prompts", kind="chunk", H=32, G=32, d=128, T=64, B=8, lo=2048, hi=4096, before=0, lens_seed=6, cap=0.0, window=0, slopes=False, prefix=0, fp32=False),
        # a model with capped scores and a window, whose first tokens stay in sight
        dict(name="chunk_capped", kind="chunk", H=16, G=8, d=128, T=64, B=4, lo=700, hi=1024, before=8000, lens_seed=7, cap=50.0, window=4096, slopes=False, prefix=4, fp32=False),
        # heads with a bias by distance, head dimension 64, odd lengths, results in 32 bits
        dict(name="chunk_slopes", kind="chunk", H=40, G=40, d=64, T=16, B=5, lo=33, hi=301, before=1000, lens_seed=8, cap=0.0, window=0, slopes=True, prefix=0, fp32=True),
        # the logits of one sequence's drafts and its next token
        dict(name="probs_few", kind="probs", rows=5, V=32000, fp32=False),
        # ... of a batch, a large vocabulary
        dict(name="probs_batch", kind="probs", rows=320, V=131072, fp32=False),
        # four sequences with up to four drafts each
        dict(name="verify_small", kind="verify", B=4, V=32000, lo=1, hi=4, lens_seed=9, sampled=True, T=32, before=300),
        # a batch with eight drafts each, a large vocabulary
        dict(name="verify_batch", kind="verify", B=64, V=131072, lo=8, hi=8, lens_seed=10, sampled=True, T=64, before=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(8, 8), (32, 32), (40, 40), (32, 8), (64, 8), (32, 4), (12, 12), (16, 2), (20, 5), (16, 1), (24, 2)]


def draw(rng):
    kind = rng.choices(["append", "chunk", "probs", "verify"], weights=[2, 6, 1, 2])[0]
    d, (H, G), T, seed = rng.choice([64, 128, 128]), rng.choice(HEADS), rng.choice([16, 32, 64, 256]), rng.randrange(1 << 30)
    if kind == "append":
        hi = _log_int(rng, 1, 4000)
        B = min(_log_int(rng, 1, 64), max(1, 24 * 2000 * 48 * 128 // 2 // ((H + 2 * G) * d * hi)))
        return dict(kind=kind, H=H, G=G, d=d, T=T, B=B, lo=rng.choice([hi, max(1, hi // 8)]), hi=hi, before=rng.choice([0, 40, 3000, 200000]), lens_seed=seed,
                    rot=rng.choice([d, d, d // 2]), interleaved=rng.random() < 0.3)
    if kind == "chunk":
        hi, before = _log_int(rng, 1, 4096), rng.choice([0, _log_int(rng, 1, 30000), _log_int(rng, 1, 30000)])
        most = 8 * 32 * 4096 * 4096 // 3                                                         # scores, of the largest listed case's
        while H * hi * (hi + before) > most:
            hi, before = max(1, hi // 2), before * 3 // 4
        B = min(_log_int(rng, 1, 64), max(1, most // (H * hi * (hi + before))), max(1, (1 << 20) // (hi + before)))
        # a cap as for scores of some tens; a bias and a window are seldom asked for together
        return dict(kind=kind, H=H, G=G, d=d, T=T, B=B, lo=rng.choice([hi, max(1, hi // 8)]), hi=hi, before=before, lens_seed=seed, cap=rng.choice([0.0, 0.0, 30.0]),
                    window=rng.choice([0, 0, 0, _log_int(rng, 1, 8192)]), slopes=rng.random() < 0.25, prefix=rng.choice([0, 0, 0, 4, hi]), fp32=rng.random() < 0.25)
    V = _log_int(rng, 64, 200000)
    if kind == "probs":
        return dict(kind=kind, rows=min(_log_int(rng, 1, 512), max(1, 320 * 131072 // V)), V=V, fp32=rng.random() < 0.3)
    hi = rng.randint(1, 12)
    return dict(kind=kind, B=min(_log_int(rng, 1, 64), max(1, 64 * 9 * 131072 // (V * (hi + 1)))), V=V, lo=rng.choice([0, 1, hi]), hi=hi, lens_seed=seed,
                sampled=rng.random() < 0.7, T=T, before=rng.choice([1, 50, 1000]))


# ---- inputs ---------------------------------------------------------------------------------------

def _generators(seed):
    g, h = torch.Generator(device=DEV), torch.Generator()
    return g.manual_seed(seed * 7919 + 29), h.manual_seed(seed * 104729 + 31)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float16)


def _layout(c):
    """Slabs of a page, groups of heads, tiles of a slab, heads of a group."""
    gg = max(x for x in range(1, c["G"] + 1) if c["G"] % x == 0 and x * c["d"] <= 1024)
    st = 1
    while 2 * st * gg * c["d"] <= 1024 and c["T"] // 16 % (2 * st) == 0:
        st *= 2
    return c["T"] // 16 // st, c["G"] // gg, st, gg


def _batch(c, h):
    """Sequences in rows of a table of two rows more: (new tokens, tokens with them) of each, its row, its pages.  How long they are is the case's."""
    fixed = torch.Generator().manual_seed(c["lens_seed"])
    B, T = c["B"], c["T"]
    new = torch.randint(c["lo"], c["hi"] + 1, (B,), generator=fixed)
    extra = 1 if c["kind"] == "verify" else 0                                                    # the token after the drafts
    before = torch.randint(c["before"] // 8, c["before"] + 1, (B,), generator=fixed)
    if B > 1:
        before[int(torch.argmin(new))] = c["before"] // 8
    lens = before + new + extra
    seqs = torch.randperm(B + 2, generator=h)[:B]
    pages = (lens + T - 1) // T
    n_pages, width = int(pages.sum()) + 3, int(pages.max()) + 1
    ids = torch.randperm(n_pages, generator=h)
    first, at = torch.cumsum(pages, 0) - pages, torch.arange(width)
    table = torch.full((B + 2, width), -1, dtype=torch.int32)
    table[seqs] = torch.where(at < pages[:, None], ids[(first[:, None] + at).clamp(max=n_pages - 1)], -1).int()
    every = torch.zeros(B + 2, dtype=torch.int32)
    every[seqs] = lens.int()
    starts = torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(new, 0)]).int()
    return dict(table=table.to(DEV), lens=every.to(DEV), seqs=seqs.int().to(DEV), starts=starts.to(DEV), n_pages=n_pages, rows=int(new.sum()))


def _append_inputs(c, seed):
    g, h = _generators(seed)
    s = _batch(c, h)
    G, d, N = c["G"], c["d"], s["rows"]
    slabs, groups, st, gg = _layout(c)
    s["pool"] = _normal(g, 1, s["n_pages"], slabs * groups * 2 * st * gg * 16 * d)
    s["q"], s["k"], s["v"] = _normal(g, N, c["H"], d), _normal(g, N, G, d), _normal(g, N, G, d)
    s["inv_freq"] = 10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device=DEV) / c["rot"])
    return s


def _chunk_inputs(c, seed):
    g, h = _generators(seed)
    s = _batch(c, h)
    slabs, groups, st, gg = _layout(c)
    s["pool"] = _normal(g, 1, s["n_pages"], slabs * groups * 2 * st * gg * 16 * c["d"])
    # queries of different sizes: some rows spread their weight over all keys, some have it on a few (with a cap, scores of tens)
    size = torch.exp(0.7 * torch.randn((s["rows"], c["H"], 1), generator=g, device=DEV)) * (8.0 if c["cap"] else 1.0)
    s["q"] = (_normal(g, s["rows"], c["H"], c["d"]) * size).half()
    s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, c["H"] + 1, device=DEV, dtype=torch.float32) / c["H"]) if c["slopes"] else None
    s["prefix"] = torch.randint(0, c["prefix"] + 1, (c["B"] + 2,), generator=h).int().to(DEV) if c["prefix"] else None
    return s


def _probs_inputs(c, seed):
    g, h = _generators(seed)
    logits = torch.randn((c["rows"], c["V"]), generator=g, device=DEV) * 3
    logits = logits if c["fp32"] else logits.half()
    logits[:, c["V"] // 2] = -math.inf                                                           # a token that is barred
    t = torch.tensor([0.7, 1.0, 0.0, 1.3])[torch.randint(0, 4, (c["rows"],), generator=h)].to(DEV)
    return dict(logits=logits, temperature=t)


def _verify_inputs(c, seed):
    g, h = _generators(seed)
    s = _batch(c, h)
    N, B, V = s["rows"], c["B"], c["V"]
    starts = s["starts"].long()
    draft = 2.5 * torch.randn((N, V), generator=g, device=DEV)
    gumbel = -torch.log(-torch.log(torch.rand((N, V), generator=g, device=DEV).clamp(1e-7, 1 - 1e-7)))
    s["drafts"] = (draft + gumbel if c["sampled"] else draft).argmax(-1).int()
    del gumbel
    # the target agrees with the draft but for some noise; its row after the last draft is by itself
    target = 2.5 * torch.randn((N + B, V), generator=g, device=DEV)
    at = torch.arange(N, device=DEV) + torch.searchsorted(starts[1:], torch.arange(N, device=DEV), right=True)
    target[at] = draft + 0.3 * target[at]
    s["target"] = torch.softmax(target, -1)
    s["draft_probs"] = torch.softmax(draft, -1) if c["sampled"] else None
    s["uniforms"] = torch.rand((N + B,), generator=g, device=DEV)
    lens, T = s["lens"], c["T"]
    table, refs = s["table"], torch.zeros(s["n_pages"], dtype=torch.int32, device=DEV)
    refs[table[table >= 0].long()] = 1
    # tables, lengths and references in one piece, so that a pass can begin with one copy of how they were
    s["book"] = torch.cat([table.reshape(-1), lens, refs])
    s["saved"] = s["book"].clone()
    a, b = table.numel(), table.numel() + lens.numel()
    s["table"], s["lens"], s["refs"] = s["book"][:a].view(table.shape), s["book"][a:b], s["book"][b:]
    return s


def _inputs(case, seed):
    return {"append": _append_inputs, "chunk": _chunk_inputs, "probs": _probs_inputs, "verify": _verify_inputs}[case["kind"]](case, seed)


# ---- state ----------------------------------------------------------------------------------------

def prepare(case, seed):
    """Inputs, and what a program keeps between calls: the cache, the sampler, the output buffers."""
    c, s = case, _inputs(case, seed)
    s["case"] = c
    if c["kind"] == "append":
        s["out"] = torch.empty_like(s["q"])
    elif c["kind"] == "chunk":
        s["out"] = torch.empty_like(s["q"], dtype=torch.float32 if c["fp32"] else torch.float16)
    elif c["kind"] == "probs":
        s["out"] = torch.empty((c["rows"], c["V"]), device=DEV)
    else:
        N, B = s["rows"], c["B"]
        s["out"] = [torch.empty(n, dtype=torch.int32, device=DEV) for n in (N + B, B, B)]
    if own:
        if c["kind"] in ("append", "chunk"):
            from paper_2504_11816_amd.cache16 import Cache16, Rope
            s["cache"] = Cache16(n_layers=1, n_q_heads=c["H"], n_kv_heads=c["G"], head_dim=c["d"], page_tokens=c["T"], n_pages=s["n_pages"], max_seqs=c["B"] + 2,
                                 max_pages_per_seq=s["table"].shape[1], pool=s["pool"], table=s["table"], device=DEV)
            if c["kind"] == "append":
                s["rope"] = Rope(s["inv_freq"], interleaved=c["interleaved"])
        else:
            from paper_2504_11816_amd.sampling import Sampler
            s["sampler"] = Sampler(max_batch=c.get("rows", c.get("B")), vocab=c["V"], device=DEV)
            if c["kind"] == "verify":
                from paper_2504_11816_amd.pages import Pages
                s["pages"] = Pages(table=s["table"], lens=s["lens"], refs=s["refs"], page_tokens=c["T"])
    return s


# ---- the plain forms ------------------------------------------------------------------------------

def _owners(s):
    """Of every row: its sequence, its place among the sequence's rows, its position."""
    starts, row = s["starts"].long(), torch.arange(s["rows"], device=DEV)
    b = torch.searchsorted(starts[1:], row, right=True)
    place = row - starts[b]
    return b, place, s["lens"][s["seqs"].long()].long()[b] - (starts[b + 1] - starts[b]) + place


def _pairs(x, rot, interleaved):
    return (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])


def _plain_rotated(x, cos, sin, c):
    a, b = _pairs(x.float(), c["rot"], c["interleaved"])
    y = x.float().clone()
    u, v = _pairs(y, c["rot"], c["interleaved"])
    u.copy_(a * cos - b * sin)
    v.copy_(a * sin + b * cos)
    return y.half()


def _plain_append(s):
    c, T, G = s["case"], s["case"]["T"], s["case"]["G"]
    slabs, groups, st, gg = _layout(c)
    b, _, pos = _owners(s)
    angle = pos.double()[:, None] * s["inv_freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    s["out"].copy_(_plain_rotated(s["q"], cos, sin, c))
    k = _plain_rotated(s["k"], cos, sin, c)
    page, at = s["table"][s["seqs"].long()[b], pos // T].long(), pos % T
    pool = s["pool"].view(s["n_pages"], slabs, groups, 2, st, gg, 16, c["d"])
    slab, tile, slot = at // (16 * st), at // 16 % st, at % 16
    # (indices that are not side by side come first: [rows][groups][gg][d])
    pool[page, slab, :, 0, tile, :, slot] = k.view(-1, groups, gg, c["d"])
    pool[page, slab, :, 1, tile, :, slot] = s["v"].view(-1, groups, gg, c["d"])
    return [s["out"], s["pool"]]


def _plain_chunk(s):
    """All sequences at once, padded: rows [B][G][H / G * n], keys [B][G][S]."""
    c = s["case"]
    B, H, G, d, T = c["B"], c["H"], c["G"], c["d"], c["T"]
    R = H // G
    slabs, groups, st, gg = _layout(c)
    seqs, starts = s["seqs"].long(), s["starts"].long()
    lens, n = s["lens"][seqs].long(), starts[1:] - starts[:-1]
    most = c["hi"]
    j = torch.arange(most, device=DEV)
    q = s["q"][(starts[:-1, None] + j).clamp(max=s["rows"] - 1)]                                  # [B][n][H][d]
    q = q.float().view(B, most, G, R, d).permute(0, 2, 3, 1, 4).reshape(B, G, R * most, d)
    kv = s["pool"].view(s["n_pages"], slabs, groups, 2, st, gg, 16, d)[s["table"][seqs].clamp(min=0).long()]
    kv = kv.permute(4, 0, 3, 6, 1, 2, 5, 7, 8).reshape(2, B, G, -1, d).float()                      # from [B][P][slabs][groups][2][st][gg][16][d]
    S = kv.shape[3]
    score = torch.matmul(q, kv[0].transpose(-1, -2)).mul_(1 / math.sqrt(d)).view(B, G, R, most, S)
    if c["cap"]:
        score.div_(c["cap"]).tanh_().mul_(c["cap"])
    i = torch.arange(S, device=DEV)
    pos = ((lens - n)[:, None] + j)[:, None, None, :, None]                                       # [B][1][1][n][1]
    if s["slopes"] is not None:
        score.sub_(s["slopes"].view(G, R, 1, 1) * (pos - i).abs())
    seen = i <= pos
    if c["window"]:
        seen &= i > pos - c["window"]
    if s["prefix"] is not None:
        seen |= (i < s["prefix"][seqs][:, None, None, None, None]) & (i < lens[:, None, None, None, None])
    score.masked_fill_(~seen, -math.inf)
    del seen
    score.sub_(score.amax(-1, keepdim=True)).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.view(B, G, R * most, S), kv[1]).view(B, G, R, most, d) / total
    b, place, _ = _owners(s)
    s["out"].copy_(out.permute(0, 3, 1, 2, 4)[b, place].reshape(-1, H, d))
    return s["out"]


def _plain_probs(s):
    x, t, V = s["logits"].float(), s["temperature"][:, None], s["case"]["V"]
    top = x.amax(-1, keepdim=True)
    e = torch.exp((x - top) / torch.where(t > 0, t, 1))
    first = torch.where(x == top, torch.arange(V, device=DEV), V).amin(-1, keepdim=True)
    s["out"].copy_(torch.where(t > 0, e / e.sum(-1, keepdim=True), (torch.arange(V, device=DEV) == first).float()))
    return s["out"]


def _plain_verify(s):
    c, B, V, N = s["case"], s["case"]["B"], s["case"]["V"], s["rows"]
    starts, every, most = s["starts"].long(), torch.arange(s["case"]["B"], device=DEV), s["case"]["hi"]
    n, j = starts[1:] - starts[:-1], torch.arange(most, device=DEV)
    row = (starts[:-1, None] + j).clamp(max=max(0, N - 1))                                        # of a draft; the target's rows have one more in every sequence before
    x = s["drafts"][row].long() if N else torch.zeros((B, most), dtype=torch.int64, device=DEV)
    p = s["target"][row + every[:, None], x]
    chance = s["uniforms"][row + every[:, None]]
    if c["sampled"]:
        chance = chance * (s["draft_probs"][row, x] if N else 0)
    good = (chance < p) & (j < n[:, None])
    count = torch.cumprod(good.int(), -1).sum(-1)
    last = (row.gather(1, count.clamp(max=most - 1)[:, None])[:, 0]).clamp(max=max(0, N - 1))
    w = s["target"][starts[:-1] + every + count].double()
    if c["sampled"]:
        q = s["draft_probs"][last].double() if N else 0
    else:
        q = torch.where(torch.arange(V, device=DEV) == x.gather(1, count.clamp(max=most - 1)[:, None]), math.inf, 0.0)
    rest = torch.where((count < n)[:, None], (w - q).clamp(min=0), w)
    w = torch.where(rest.sum(-1, keepdim=True) > 0, rest, w)
    upto = torch.cumsum(w, -1)
    u = s["uniforms"][starts[1:] + every].double()
    token = (upto <= (u * upto[:, -1])[:, None]).sum(-1).int()
    tokens, accepted, rejected = s["out"]
    tokens.fill_(-1)
    keep = j < count[:, None]
    tokens[(row + every[:, None])[keep]] = x[keep].int()
    tokens[starts[:-1] + every + count] = token
    accepted.copy_(count)
    rejected.copy_(n - count)
    # the cache: sequences without what was rejected, their pages free
    seqs, T = s["seqs"].long(), c["T"]
    lens = s["lens"][seqs] - rejected
    s["lens"][seqs] = lens
    held = s["table"][seqs]
    gone = (torch.arange(held.shape[1], device=DEV) >= ((lens + T - 1) // T)[:, None]) & (held >= 0)
    s["refs"].index_add_(0, held.clamp(min=0).reshape(-1), -gone.int().reshape(-1))
    s["table"][seqs] = torch.where(gone, -1, held)


# ---- one pass -------------------------------------------------------------------------------------

def run(state):
    s, c = state, state["case"]
    if c["kind"] == "append":
        if not own:
            return _plain_append(s)
        s["cache"].append(0, s["k"], s["v"], s["starts"], s["lens"], s["seqs"], q=s["q"], q_out=s["out"], rope=s["rope"])
        return [s["out"], s["pool"]]
    if c["kind"] == "chunk":
        if not own:
            return _plain_chunk(s)
        s["cache"].attend(0, s["q"], s["out"], s["starts"], s["lens"], s["seqs"], cap=c["cap"], window=c["window"], slopes=s["slopes"], prefix=s["prefix"])
        return s["out"]
    if c["kind"] == "probs":
        if not own:
            return _plain_probs(s)
        s["sampler"].probs(s["logits"], s["out"], s["temperature"])
        return s["out"]
    s["book"].copy_(s["saved"])                                                                  # the sequences are as long as before the step's verification
    if own:
        s["sampler"].verify(s["target"], s["drafts"], s["starts"], s["uniforms"], *s["out"], draft_probs=s["draft_probs"])
        s["pages"].shrink(s["seqs"], s["out"][2])
    else:
        _plain_verify(s)
    return [*s["out"], s["table"], s["lens"], s["refs"]]


# ---- what a pass cannot do without ----------------------------------------------------------------

def _seen(c):
    """Over the case's own sequences: rows, keys that a sequence's rows read, (row, key) pairs.  A prefix counts with the mean of its lengths."""
    fixed = torch.Generator().manual_seed(c["lens_seed"])
    new = torch.randint(c["lo"], c["hi"] + 1, (c["B"],), generator=fixed)
    before = torch.randint(c["before"] // 8, c["before"] + 1, (c["B"],), generator=fixed)
    if c["B"] > 1:
        before[int(torch.argmin(new))] = c["before"] // 8
    keys = pairs = 0
    for n, b in zip(new.tolist(), before.tolist()):
        upto = torch.arange(b + 1, b + n + 1, dtype=torch.float64)                               # keys up to the row's own
        recent = torch.clamp(upto, max=c["window"]) if c["window"] else upto
        f = min(c["prefix"] / 2, b + n)
        pairs += float((recent + torch.clamp(upto - recent, max=f) + torch.clamp(f - upto, min=0)).sum())
        keys += min(b + n, c["window"] + n - 1 + f) if c["window"] else b + n
    return int(new.sum()), keys, pairs


def work(case):
    c = case
    if c["kind"] == "append":
        rows = int(torch.randint(c["lo"], c["hi"] + 1, (c["B"],), generator=torch.Generator().manual_seed(c["lens_seed"])).sum())
        return {"bytes": rows * c["d"] * 4 * (c["H"] + 2 * c["G"]), "flops": rows * (c["H"] + c["G"]) * c["rot"] * 3}
    if c["kind"] == "chunk":
        rows, keys, pairs = _seen(c)
        return {"bytes": keys * c["G"] * c["d"] * 4 + rows * c["H"] * c["d"] * (2 + (4 if c["fp32"] else 2)), "flops": 4 * pairs * c["H"] * c["d"]}
    if c["kind"] == "probs":
        n = c["rows"] * c["V"]
        return {"bytes": n * (8 if c["fp32"] else 6), "flops": 4 * n}
    return {"bytes": c["B"] * c["V"] * (8 if c["sampled"] else 4), "flops": 3 * c["B"] * c["V"]}


# ---- the same from the definitions, in 64 bits ----------------------------------------------------

def _place(c, pos, table_row):
    """Element of the pool where the K rows of all heads of tokens `pos` begin: [tokens][G], and how far behind their V rows are."""
    slabs, groups, st, gg = _layout(c)
    head = torch.arange(c["G"], device=DEV)
    page, at = table_row[pos // c["T"]].long(), pos % c["T"]
    unit = 16 * c["d"]
    of_page = slabs * groups * 2 * st * gg * unit
    first = page * of_page + at // (16 * st) * (groups * 2 * st * gg * unit) + at // 16 % st * (gg * unit) + at % 16 * c["d"]
    return first[:, None] + head // gg * (2 * st * gg * unit) + head % gg * unit, st * gg * unit


def _exact_append(c, s):
    out, pool = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV), s["pool"].double().view(-1)
    starts, seqs, lens = s["starts"].tolist(), s["seqs"].tolist(), s["lens"].tolist()
    e = torch.arange(c["d"], device=DEV)
    half = c["rot"] // 2
    for b, row in enumerate(seqs):
        a, z = starts[b], starts[b + 1]
        pos = torch.arange(lens[row] - (z - a), lens[row], device=DEV)
        turn = torch.polar(torch.ones((z - a, half), dtype=torch.float64, device=DEV), pos.double()[:, None] * s["inv_freq"])[:, None]

        def rotated(x):
            x = x.double().clone()
            r = x[..., :c["rot"]]
            z = torch.view_as_complex(r.unflatten(-1, (half, 2)).contiguous()) if c["interleaved"] else torch.complex(r[..., :half], r[..., half:])
            z = z * turn
            x[..., :c["rot"]] = torch.view_as_real(z).flatten(-2) if c["interleaved"] else torch.cat([z.real, z.imag], -1)
            return x

        out[a:z] = rotated(s["q"][a:z])
        at, apart = _place(c, pos, s["table"][row])
        pool[at[..., None] + e] = rotated(s["k"][a:z])
        pool[at[..., None] + apart + e] = s["v"][a:z].double()
    return [out, pool.view(s["pool"].shape)]


def _exact_chunk(c, s):
    H, G, d = c["H"], c["G"], c["d"]
    out, flat = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV), s["pool"].view(-1)
    starts, seqs, lens = s["starts"].tolist(), s["seqs"].tolist(), s["lens"].tolist()
    e = torch.arange(d, device=DEV)
    for b, row in enumerate(seqs):
        a, z, L = starts[b], starts[b + 1], lens[row]
        key = torch.arange(L, device=DEV)
        at, apart = _place(c, key, s["table"][row])
        step = max(1, (1 << 27) // L)                                                            # rows at a time: 1 GiB of scores
        for g in range(G):
            k, v = flat[at[:, g, None] + e].double(), flat[at[:, g, None] + apart + e].double()
            for h in range(g * (H // G), (g + 1) * (H // G)):
                for r in range(a, z, step):
                    n = min(step, z - r)
                    pos = torch.arange(L - (z - r), L - (z - r) + n, device=DEV)[:, None]
                    x = s["q"][r:r + n, h].double() @ k.T / d ** 0.5
                    if c["cap"]:
                        x = c["cap"] * torch.tanh(x / c["cap"])
                    if s["slopes"] is not None:
                        x -= s["slopes"][h].double() * (pos - key).abs()
                    hidden = key > pos
                    if c["window"]:
                        hidden |= pos - key >= c["window"]
                    if s["prefix"] is not None:
                        hidden &= key >= s["prefix"][row]
                    out[r:r + n, h] = torch.softmax(x.masked_fill(hidden, -math.inf), -1) @ v
    return out


def exact(case, seed):
    if case["kind"] == "verify":
        return None                                                                              # whole numbers throughout
    c, s = case, _inputs(case, seed)
    if c["kind"] == "append":
        return _exact_append(c, s)
    if c["kind"] == "chunk":
        return _exact_chunk(c, s)
    out = torch.zeros((c["rows"], c["V"]), dtype=torch.float64, device=DEV)
    for r, t in enumerate(s["temperature"].double().tolist()):
        x = s["logits"][r].double()
        if t > 0:
            out[r] = torch.softmax(x / t, -1)
        else:
            out[r, int((x == x.max()).nonzero()[0])] = 1
    return out
