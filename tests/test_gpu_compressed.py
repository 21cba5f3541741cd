"""Whole decoder layers with 4-bit weights over the 8-bit cache, and the example that serves with them.

Tolerance of whole layers as for the fp16 ones (a different rounding decision at one fp16 store moves a value by 2^-11 relative, and four products and
two norms follow one another): 1.5e-2 + 1.5e-2 |oracle| against the oracle that rounds to fp16 where the GPU stores fp16."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import cache8 as oracle8
from oracle import decode_layer as dl
from oracle import linear4 as oracle4
from paper_2504_11816_amd.cache8 import Cache8
from paper_2504_11816_amd.compressed import CompressedLayer, Scratch, decoder_step
from paper_2504_11816_amd.harness import LayerWeights

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def ids(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("group,zeros,fmt", [(128, False, "int8"), (32, True, "e4m3"), (64, True, "int8")])
def test_decoder_layers_against_the_definition(group, zeros, fmt):
    rng = np.random.default_rng(group)
    H, G, d, h2, lens, L = 8, 2, 64, 1024, [31, 70, 0], 1
    h1, kv, B = H * d, G * d, 3
    weights = [LayerWeights(h1, h2, 5, l, DEV, kv_cols=kv) for l in range(L)]
    layers = [CompressedLayer(w, group, zeros) for w in weights]
    cache = Cache8(n_layers=L, n_q_heads=H, n_kv_heads=G, head_dim=d, page_tokens=32, n_pages=20, max_seqs=4, max_pages_per_seq=5, format=fmt, device=DEV)
    seqs = ids([2, 0, 3])
    cache.pages.extend(seqs, ids(lens))
    k, v = (torch.randn((L, sum(lens), G, d), device=DEV).half() for _ in range(2))
    cache.store(k, v, ids(np.concatenate([[0], np.cumsum(lens)])), cache.lens, seqs)
    ends = np.cumsum(lens)
    rows = [[[x[l, a:b].double().cpu().numpy() for a, b in zip(ends - lens, ends)] for x in (k, v)] for l in range(L)]
    scratch, x = Scratch(4, h1, h2, kv, DEV), torch.zeros((B, h1), dtype=torch.float16, device=DEV)
    for step in range(3):
        first = rng.standard_normal((B, h1)).astype(np.float16)
        x.copy_(torch.tensor(first))
        decoder_step(cache, layers, scratch, x, seqs)
        want = first.astype(np.float64)
        for l, w in enumerate(weights):
            p = w.numpy()
            stacked = oracle4.quantise(w.wqkv.cpu().numpy(), group, zeros)
            p.update(wq=stacked[:h1], wk=stacked[h1:h1 + kv], wv=stacked[h1 + kv:])
            p.update({n: oracle4.quantise(w.t[n].cpu().numpy(), group, zeros) for n in ("wo", "w1", "w2")})
            q, kn, vn = dl.qkv(want, p, fp16_between=True)
            t = np.empty((B, h1))
            for b in range(B):
                for i, new in enumerate((kn, vn)):
                    rows[l][i][b] = np.concatenate([rows[l][i][b], new[b].reshape(1, G, d)])
                n = len(rows[l][0][b])
                t[b] = oracle8.attend(q[b].reshape(H, d), rows[l][0][b], rows[l][1][b], n, fmt, True).reshape(-1)
            want = dl.after_attention(want, dl.round16(t), p, fp16_between=True)
        got = x.double().cpu().numpy()
        assert np.isfinite(got).all() and (np.abs(got - want) <= 1.5e-2 + 1.5e-2 * np.abs(want)).all(), step
    cache.pages.check()
    assert cache.lens.tolist() == [73, 0, 34, 3]


def test_the_example():
    spec = importlib.util.spec_from_file_location("serve_compressed", os.path.join(ROOT, "examples", "serve_compressed.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    r = m.serve(prompts=2, answers=3, steps=10, layers=2)
    cache = r["cache"]
    assert torch.isfinite(r["out"]).all() and r["pages_after_fork"] < r["pages_unshared"]
    assert r["weight_bytes"] < 0.3 * r["weight_bytes_fp16"]
    live = cache.table[r["live"].long()]
    assert live[live >= 0].max() == r["pages_left"] - 1 and int((cache.refs > 0).sum()) == r["pages_left"]
    for host, dev in zip(r["on_host"], (cache.codes, cache.scales)):
        assert torch.equal(host, dev[:, :r["pages_left"]].cpu())
    with pytest.raises(ValueError):
        decoder_step(cache, [], Scratch(1, 1024, 4096, 256, DEV), r["out"], r["live"])
