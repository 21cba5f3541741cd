"""Steps of whole layers that do not fit, refused before lengths grow."""
import math
import types

import numpy as np
import pytest
import torch

from paper_2504_11816_amd.cache16 import Cache16, Rope
from paper_2504_11816_amd.cache8 import Cache8
from paper_2504_11816_amd.compressed import CompressedLayer, Scratch, decoder_chunk, decoder_step
from paper_2504_11816_amd.harness import LayerWeights

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
H, G, D, H2 = 8, 2, 64, 1024
H1, KV = H * D, G * D


def ids(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def between(rows):
    """[rows][h1] contiguous, two bytes past an address that loads of 16 bytes can take."""
    return torch.zeros(rows * H1 + 8, dtype=torch.float16, device=DEV)[1:1 + rows * H1].view(rows, H1)


def refuses(step, cache, buffers, bad):
    before = [t.clone() for t in buffers]
    for kw in bad:
        with pytest.raises(ValueError):
            step(**kw)
        assert all(torch.equal(a, b) for a, b in zip(before, buffers)), kw
    cache.pages.check()


def test_chunks_that_a_later_call_would_refuse():
    c = Cache16(n_layers=1, n_q_heads=H, n_kv_heads=G, head_dim=D, page_tokens=32, n_pages=40, max_seqs=4, max_pages_per_seq=8, device=DEV)
    layers, scratch = [CompressedLayer(LayerWeights(H1, H2, 5, 0, DEV, kv_cols=KV))], Scratch(16, H1, H2, KV, DEV)
    c.pages.extend(ids([0, 1]), ids([10, 20]))
    good = dict(cache=c, layers=layers, scratch=scratch, x=torch.randn((6, H1), device=DEV).half(), starts=ids([0, 2, 6]), seqs=ids([1, 0]), n_new=ids([2, 4]), rope=Rope.of(D, device=DEV))
    bad = [dict(x=between(6)), dict(eps=-1.0), dict(eps=math.nan), dict(window=2.5), dict(window=math.nan), dict(window=torch.tensor(2.5)), dict(cap="1")]
    refuses(lambda **kw: decoder_chunk(**{**good, **kw}), c, (c.pool, c.table, c.lens, c.refs), bad)
    decoder_chunk(**good, window=np.int64(7), eps=0)
    assert c.lens.tolist()[:2] == [14, 22]


def test_steps_that_a_later_call_would_refuse():
    c = Cache8(n_layers=1, n_q_heads=H, n_kv_heads=G, head_dim=D, page_tokens=32, n_pages=40, max_seqs=4, max_pages_per_seq=8, device=DEV)
    layers, scratch = [CompressedLayer(LayerWeights(H1, H2, 5, 0, DEV, kv_cols=KV))], Scratch(16, H1, H2, KV, DEV)
    c.pages.extend(ids([0, 1]), ids([10, 20]))
    good = dict(cache=c, layers=layers, scratch=scratch, x=torch.randn((2, H1), device=DEV).half(), seqs=ids([1, 0]))
    refuses(lambda **kw: decoder_step(**{**good, **kw}), c, (c.codes, c.scales, c.tails, c.table, c.lens, c.refs), [dict(x=between(2)), dict(eps=-1.0), dict(eps=math.nan)])
    decoder_step(**good)
    assert c.lens.tolist()[:2] == [11, 21]


def test_layers_that_are_wider_than_a_norm():
    """(The weights are never reached.)"""
    heads, kv_heads = 272, 17
    h1, kv = heads * D, kv_heads * D
    layers, scratch, x = [types.SimpleNamespace(h1=h1, kv_cols=kv, h2=64)], Scratch(2, h1, 64, kv, DEV), torch.zeros((2, h1), dtype=torch.float16, device=DEV)
    how = dict(n_layers=1, n_q_heads=heads, n_kv_heads=kv_heads, head_dim=D, page_tokens=32, n_pages=2, max_seqs=2, max_pages_per_seq=1, device=DEV)
    c, c8 = Cache16(**how), Cache8(**how)
    refuses(lambda: decoder_chunk(c, layers, scratch, x, ids([0, 2]), ids([0]), ids([2])), c, (c.table, c.lens, c.refs), [dict()])
    refuses(lambda: decoder_step(c8, layers, scratch, x, ids([0, 1])), c8, (c8.table, c8.lens, c8.refs), [dict()])
