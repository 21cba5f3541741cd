"""Speculative decoding over the fp16 paged cache, with 4-bit weights, on one GPU:

  the prompts go through the layers in chunks; then, step by step, a draft (the model's first layers, with a cache of its own) proposes a few tokens for every
  sequence, the model takes all of them in one chunk, the drafts are held against its probabilities, and what was rejected leaves both caches.

Weights, embeddings and prompts are random.

    python examples/serve_speculative.py --prompts 4 --drafts 4 --steps 12
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2504_11816_amd.cache16 import Cache16, Rope  # noqa: E402
from paper_2504_11816_amd.compressed import CompressedLayer, Scratch, decoder_chunk  # noqa: E402
from paper_2504_11816_amd.harness import LayerWeights  # noqa: E402
from paper_2504_11816_amd.linear4 import Linear4  # noqa: E402
from paper_2504_11816_amd.sampling import Sampler  # noqa: E402


def serve(*, prompts=4, drafts=4, steps=12, layers=4, draft_layers=2, heads=16, kv_heads=4, d=64, h2=4096, vocab=2048, page_tokens=64, longest=300, chunk=128, temperature=0.8,
          window=0, seed=1, device="cuda:0"):
    rng = np.random.default_rng(seed)
    torch.manual_seed(seed)
    h1, kv, B, k = heads * d, kv_heads * d, prompts, drafts
    model = [CompressedLayer(LayerWeights(h1, h2, seed, l, device, kv_cols=kv)) for l in range(layers)]
    embed = torch.randn((vocab, h1), device=device).half()
    head = Linear4.quantize((torch.randn((vocab, h1), device=device) / h1 ** 0.5).half())
    rope = Rope.of(d, device=device)
    lens = rng.integers(longest // 3, longest + 1, B)
    tokens = [torch.tensor(rng.integers(0, vocab, n), dtype=torch.int64, device=device) for n in lens]
    per_seq = -(-(longest + (steps + 1) * (k + 1)) // page_tokens)

    def cache(n_layers):
        return Cache16(n_layers=n_layers, n_q_heads=heads, n_kv_heads=kv_heads, head_dim=d, page_tokens=page_tokens, n_pages=B * per_seq, max_seqs=B, max_pages_per_seq=per_seq, device=device)

    def ids(x):
        return torch.tensor(np.asarray(x), dtype=torch.int32, device=device)

    target, draft = cache(layers), cache(draft_layers)
    scratch = Scratch(max(B * chunk, B * (k + 1)), h1, h2, kv, device)
    seqs, sampler = ids(range(B)), Sampler(max_batch=B * (k + 1), vocab=vocab, device=device)
    temperatures = torch.full((B * (k + 1),), temperature, device=device)

    # the prompts but for their last tokens, a chunk of every sequence at a time
    for first in range(0, int(lens.max()) - 1, chunk):
        n = np.clip(lens - 1 - first, 0, chunk)
        rows = torch.cat([t[first:first + m] for t, m in zip(tokens, n)])
        starts, new = ids(np.concatenate([[0], np.cumsum(n)])), ids(n)
        for c in (target, draft):
            x = embed[rows]
            decoder_chunk(c, model[:c.L], scratch, x, starts, seqs, new, rope=rope, window=window)
    last = torch.stack([t[-1] for t in tokens])

    ones, one_each = ids([1] * B), ids(range(B + 1))
    empty, none = ids([]), ids([0] * (B + 1))
    several, starts_several, starts_drafts = ids([k + 1] * B), ids(np.arange(B + 1) * (k + 1)), ids(np.arange(B + 1) * k)
    q, p = torch.empty((B, k, vocab), device=device), torch.empty((B * (k + 1), vocab), device=device)
    logits, few = torch.empty((B * (k + 1), vocab), dtype=torch.float16, device=device), torch.empty((B, vocab), dtype=torch.float16, device=device)
    drawn, counts = torch.empty(B, dtype=torch.int32, device=device), [torch.empty(B, dtype=torch.int32, device=device) for _ in range(2)]
    out, accepted_all = torch.empty(B * (k + 1), dtype=torch.int32, device=device), 0
    answers = [[] for _ in range(B)]
    for _ in range(steps):
        proposed = [last]
        for i in range(k + 1):                               # (the last one is stored, too: its draft may be accepted)
            x = embed[proposed[-1]]
            decoder_chunk(draft, model[:draft_layers], scratch, x, one_each, seqs, ones, rope=rope, window=window)
            if i == k:
                break
            head(x, few)
            sampler.probs(few, q[:, i], temperatures[:B])
            sampler.verify(q[:, i], empty, none, torch.rand(B, device=device), drawn, counts[0])      # (no drafts: a token is drawn)
            proposed.append(drawn.long())
        x = embed[torch.stack(proposed, 1).view(-1)]
        decoder_chunk(target, model, scratch, x, starts_several, seqs, several, rope=rope, window=window)
        head(x, logits)
        sampler.probs(logits, p, temperatures)
        guesses = torch.stack(proposed[1:], 1).view(-1).int().contiguous()
        sampler.verify(p, guesses, starts_drafts, torch.rand(B * (k + 1), device=device), out, *counts, draft_probs=q.view(B * k, vocab))
        for c in (target, draft):
            c.pages.shrink(seqs, counts[1])
        last = out.view(B, k + 1).gather(1, counts[0].long()[:, None])[:, 0].long()
        for b, (row, n) in enumerate(zip(out.view(B, k + 1).tolist(), counts[0].tolist())):
            answers[b] += row[:n + 1]
            accepted_all += n
    for c in (target, draft):
        c.pages.check()
    return dict(target=target, draft=draft, model=model, embed=embed, rope=rope, prompts=[t.tolist() for t in tokens], answers=answers, accepted=accepted_all, proposed=B * k * steps)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("prompts", 4), ("drafts", 4), ("steps", 12), ("layers", 4), ("draft-layers", 2), ("window", 0)):
        ap.add_argument("--" + name, type=int, default=default)
    r = serve(**vars(ap.parse_args()))
    print(f"lengths {r['target'].lens.tolist()}, pages {int((r['target'].refs > 0).sum())} and {int((r['draft'].refs > 0).sum())}")
    print(f"drafts accepted {r['accepted']} of {r['proposed']}; tokens {[len(a) for a in r['answers']]}")


if __name__ == "__main__":
    main()
