"""What the speculative example leaves in its caches, token by token."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import kv_layout
from paper_2504_11816_amd.cache16 import Cache16
from paper_2504_11816_amd.compressed import Scratch, decoder_chunk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def ids(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("window", (0, 64))
def test_what_the_example_leaves_in_every_page(window):
    """Both caches hold, for every token up to a sequence's last one, what the tokens by themselves give in one chunk of a fresh cache: the last, partly filled page, where drafts were rejected and others came in
    their place, among them.  Tolerance of whole layers (1.5e-2 + 1.5e-2 of the largest), which four fp16 stores of a layer before may each take."""
    spec = importlib.util.spec_from_file_location("serve_speculative", os.path.join(ROOT, "examples", "serve_speculative.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.serve(prompts=3, drafts=3, steps=6, layers=2, draft_layers=1, longest=150, window=window)
    assert r["accepted"] < r["proposed"]
    partly_filled = 0
    for c in (r["target"], r["draft"]):
        table = c.table.cpu().numpy()
        for b in range(3):
            tokens = torch.tensor([*r["prompts"][b], *r["answers"][b]][:-1], device=DEV)
            n = len(tokens)
            fresh = Cache16(n_layers=c.L, n_q_heads=c.H, n_kv_heads=c.G, head_dim=c.d, page_tokens=c.T, n_pages=8, max_seqs=1, max_pages_per_seq=8, device=DEV)
            x = r["embed"][tokens]
            decoder_chunk(fresh, r["model"][:c.L], Scratch(n, x.shape[1], 4096, c.G * c.d, DEV), x, ids([0, n]), ids([0]), ids([n]), rope=r["rope"], window=window)
            partly_filled += n % c.T > 0
            for l in range(c.L):
                a, z = c.pool[l].cpu().numpy().reshape(-1), fresh.pool[l].cpu().numpy().reshape(-1)
                for kv in range(2):
                    for g in range(c.G):
                        u = kv_layout.gather_rows(a, dict(kind="paged", G=c.G, d=c.d, T=c.T, block_table=table), b, kv, g, n).astype(np.float64)
                        w = kv_layout.gather_rows(z, dict(kind="paged", G=c.G, d=c.d, T=c.T, block_table=fresh.table.cpu().numpy()), 0, kv, g, n).astype(np.float64)
                        off, tol = np.abs(u - w).max(-1), 1.5e-2 * 4 + 1.5e-2 * np.abs(w).max()
                        assert np.median(np.abs(w[1:] - w[:-1]).max(-1)) > 4 * tol      # (another token's row would be seen)
                        assert (off <= tol).all(), f"layer {l} kv {kv} head {g} sequence {b} of {n} tokens: token {int(off.argmax())} is off by {off.max()}"
    assert partly_filled
