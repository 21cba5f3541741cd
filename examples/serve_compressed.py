"""Several answers to each of a few prompts, with 4-bit weights and an 8-bit paged KV cache, on one GPU:

  the prompts' keys and values go into the cache (quantised), every prompt is forked once per answer more (full pages are shared), all answers are
  decoded together, those that end give their pages back, the pages left move together and are gathered for one copy to the host.

Weights are random, and so are the prompts' keys and values, as a prefill would leave them.

    python examples/serve_compressed.py --prompts 4 --answers 3 --steps 40
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2504_11816_amd.cache8 import Cache8  # noqa: E402
from paper_2504_11816_amd.compressed import CompressedLayer, Scratch, decoder_step  # noqa: E402
from paper_2504_11816_amd.harness import LayerWeights  # noqa: E402
from paper_2504_11816_amd.pages import PageArray  # noqa: E402


def serve(*, prompts=4, answers=3, steps=40, layers=4, heads=16, kv_heads=4, d=64, h2=4096, page_tokens=64, longest=300, format="int8", seed=1, device="cuda:0"):
    rng = np.random.default_rng(seed)
    h1, kv, n = heads * d, kv_heads * d, prompts * answers
    weights = [LayerWeights(h1, h2, seed, l, device, kv_cols=kv) for l in range(layers)]
    compressed = [CompressedLayer(w) for w in weights]
    lens = rng.integers(longest // 3, longest + 1, prompts)
    per_seq = -(-(longest + steps) // page_tokens)
    cache = Cache8(n_layers=layers, n_q_heads=heads, n_kv_heads=kv_heads, head_dim=d, page_tokens=page_tokens, n_pages=n * per_seq, max_seqs=n,
                   max_pages_per_seq=per_seq, format=format, device=device)

    def ids(x):
        return torch.tensor(np.asarray(x), dtype=torch.int32, device=device)

    # the prompts
    first = ids(range(prompts))
    cache.pages.extend(first, ids(lens))
    k, v = (torch.randn((layers, int(lens.sum()), kv_heads, d), device=device).half() for _ in range(2))
    cache.store(k, v, ids(np.concatenate([[0], np.cumsum(lens)])), cache.lens, first)
    # the other answers to them
    rest = ids(range(prompts, n))
    if n > prompts:
        cache.pages.fork(first.repeat(answers - 1), rest)
    used, unshared = int((cache.refs > 0).sum()), int(sum(-(-int(x) // page_tokens) for x in lens)) * answers
    # decoding; every prompt's first answer ends half way
    live, x = torch.cat([first, rest]), torch.randn((n, h1), device=device).half()
    scratch = Scratch(n, h1, h2, kv, device)
    for step in range(steps):
        if step == steps // 2 and n > prompts:
            cache.pages.free(first)
            live, x = rest, x[prompts:].contiguous()
        decoder_step(cache, compressed, scratch, x, live)
    cache.pages.check()
    # what is left, in one piece for the host
    cache.pages.compact()
    left = int(cache.pages.status[1])
    staging = [torch.empty_like(t[:, :left]) for t in (cache.codes, cache.scales)]
    cache.pages.copy(ids(range(left)), ids(range(left)), to=[PageArray(t) for t in staging])
    on_host = [torch.empty(t.shape, dtype=t.dtype, pin_memory=True).copy_(t, non_blocking=True) for t in staging]
    torch.cuda.synchronize()
    return dict(out=x, cache=cache, weights=weights, live=live, pages_after_fork=used, pages_unshared=unshared, pages_left=left, on_host=on_host,
                weight_bytes=sum(w.packed_bytes() for w in compressed), weight_bytes_fp16=sum(w.bytes_read_per_step() for w in weights))


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("prompts", 4), ("answers", 3), ("steps", 40), ("layers", 4)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--format", choices=("int8", "e4m3"), default="int8")
    r = serve(**vars(ap.parse_args()))
    print(f"lengths {r['cache'].lens.tolist()}")
    print(f"pages after forking {r['pages_after_fork']} ({r['pages_unshared']} without sharing), at the end {r['pages_left']}")
    print(f"weights {r['weight_bytes'] / 1e6:.1f} MB ({r['weight_bytes_fp16'] / 1e6:.1f} in fp16), on the host {sum(t.numel() * t.element_size() for t in r['on_host']) / 1e6:.1f} MB of cache")
    print(f"output finite: {bool(torch.isfinite(r['out']).all())}")


if __name__ == "__main__":
    main()
