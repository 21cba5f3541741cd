"""A step of whole compressed layers that is refused leaves the cache as it was: lengths, pages, tails."""
import numpy as np
import pytest
import torch

from paper_2504_11816_amd.cache8 import Cache8
from paper_2504_11816_amd.compressed import CompressedLayer, Scratch, decoder_step
from paper_2504_11816_amd.harness import LayerWeights

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
H, G, D, H2, L, B = 4, 2, 64, 512, 2, 3
H1, KV = H * D, G * D


def ids(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


@pytest.fixture(scope="module")
def layers():
    return [CompressedLayer(LayerWeights(H1, H2, 5, layer, DEV, kv_cols=KV)) for layer in range(L)]


def cache(**kw):
    c = Cache8(**{**dict(n_layers=L, n_q_heads=H, n_kv_heads=G, head_dim=D, page_tokens=32, n_pages=20, max_seqs=4, max_pages_per_seq=5, device=DEV), **kw})
    c.pages.extend(ids(range(4)), ids([31, 7, 0, 40]))
    c.tails.normal_(generator=torch.Generator(device=DEV).manual_seed(1))
    return c


def refused(c, layers, scratch, x, seqs):
    state = (c.codes, c.scales, c.tails, c.table, c.lens, c.refs)
    before = [t.clone() for t in state]
    with pytest.raises(ValueError):
        decoder_step(c, layers, scratch, x, seqs)
    assert all(torch.equal(a, b) for a, b in zip(before, state))


def test_rows_of_another_number(layers):
    c, scratch, x = cache(), Scratch(4, H1, H2, KV, DEV), torch.randn((B, H1), device=DEV).half()
    refused(c, layers, scratch, x, ids([0, 1]))
    refused(c, layers, scratch, x, ids(range(4)))
    refused(c, layers, scratch, x, ids([0, 1, 2]).long())
    refused(c, layers, scratch, x.float(), ids([0, 1, 3]))
    decoder_step(c, layers, scratch, x, ids([0, 1, 3]))
    c.pages.check()
    assert c.lens.tolist() == [32, 8, 0, 41] and torch.isfinite(x).all()


def test_widths_that_do_not_fit(layers):
    """Refused before a kernel reads a norm's vectors, or writes activations, at another width."""
    c, scratch, x, seqs = cache(), Scratch(4, H1, H2, KV, DEV), torch.randn((B, H1), device=DEV).half(), ids([0, 1, 3])
    wide = torch.randn((B, 2 * H1), device=DEV).half()
    for bad in (wide, wide[:, :H1], x[:, :128].contiguous(), x.cpu(), x.view(B, H, D)):
        refused(c, layers, scratch, bad, seqs)
    refused(c, layers, scratch, x, seqs.cpu())
    for bad in (layers[:1], [*layers, layers[0]], []):
        refused(c, bad, scratch, x, seqs)
    for bad in (Scratch(4, 2 * H1, H2, KV, DEV), Scratch(4, 128, H2, KV, DEV), Scratch(4, H1, 2 * H2, KV, DEV), Scratch(4, H1, H2, 64, DEV), Scratch(2, H1, H2, KV, DEV),
                Scratch(4, H1, H2, KV, "cpu")):
        refused(c, layers, bad, x, seqs)
    refused(cache(out_dtype=torch.float32), layers, scratch, x, seqs)
    refused(cache(n_q_heads=8), layers, scratch, x, seqs)
    refused(cache(n_kv_heads=4), layers, scratch, x, seqs)


def test_weights_that_do_not_fit():
    good = LayerWeights(H1, H2, 5, 0, DEV, kv_cols=KV)
    for name, change in (("ln1_g", lambda t: t[:-1]), ("ln2_b", lambda t: t.float()), ("wq", lambda t: t[:-16]), ("wv", lambda t: t[:-16]), ("w2", lambda t: t[:, :-32])):
        class Weights:
            t = {**good.t, name: change(good.t[name])}
        with pytest.raises(ValueError):
            CompressedLayer(Weights)
