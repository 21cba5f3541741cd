"""Steps over the 8-bit cache whose layers come one by one: what begin() is given, the calls between it and the layers, the streams that they come on, and
what attend() refuses."""
import numpy as np
import pytest
import torch

from paper_2504_11816_amd.cache8 import Cache8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
L, H, G, D, T = 2, 4, 2, 64, 32


def ids(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def filled(lens, width=40, seed=1):
    """A cache with these sequences, one token of room in each; width: of the page table, above 32 sequences are cut among wavefronts."""
    rng = np.random.default_rng(seed)
    c = Cache8(n_layers=L, n_q_heads=H, n_kv_heads=G, head_dim=D, page_tokens=T, n_pages=sum(n // T + 1 for n in lens), max_seqs=len(lens), max_pages_per_seq=width,
               out_dtype=torch.float32, device=DEV)
    every = ids(range(len(lens)))
    c.pages.extend(every, ids(lens))
    k, v = (torch.tensor(rng.standard_normal((L, sum(lens), G, D)), dtype=torch.float16, device=DEV) for _ in range(2))
    c.store(k, v, ids(np.concatenate([[0], np.cumsum(lens)])), c.lens)
    c.pages.extend(every)
    c.pages.check()
    return c


def inputs(B, seed=2):
    rng = np.random.default_rng(seed)
    return [torch.tensor(rng.standard_normal((L, B, h, D)), dtype=torch.float16, device=DEV) for h in (H, G, G)]


def layers(c, q, k, v, out):
    for layer in range(L):
        c.attend(layer, q[layer], k[layer], v[layer], out[layer])


@pytest.mark.parametrize("width", [32, 40])
def test_lengths_and_rows_that_nobody_else_keeps(width):
    """begin() with temporaries: what is allocated and filled after it is not what the layers read."""
    lens = [40, 100, 7, 64]
    a, b = filled(lens, width), filled(lens, width)
    q, k, v = inputs(3)
    outs = [torch.empty((L, 3, H, D), device=DEV) for _ in range(2)]
    seqs, now = ids([2, 0, 3]), a.lens.clone()
    a.begin(3, now, seqs)
    layers(a, q, k, v, outs[0])
    b.begin(3, b.lens + 0, ids([2, 0, 3]))
    others = [torch.ones(n, dtype=torch.int32, device=DEV) for n in (3, 4) for _ in range(50)]
    layers(b, q, k, v, outs[1])
    assert torch.equal(*outs) and torch.equal(a.tails, b.tails) and torch.equal(a.codes, b.codes)
    assert all((x == 1).all() for x in others)


@pytest.mark.parametrize("width", [32, 40])
def test_a_step_of_all_layers_ends_a_layerwise_one(width):
    """A step() between two layers has lengths, rows and a plan of its own: the other layers are refused, and change nothing."""
    c = filled([40, 100, 7], width)
    q, k, v = inputs(3)
    out = torch.empty((L, 3, H, D), device=DEV)
    c.begin(3, c.lens)
    c.attend(0, q[0], k[0], v[0], out[0])
    c.step(q[:, :2].contiguous(), None, None, torch.empty((L, 2, H, D), device=DEV), c.lens, ids([1, 2]))
    before = [x.clone() for x in (c.codes, c.scales, c.tails, out)]
    for n in (2, 3):
        with pytest.raises(ValueError):
            c.attend(1, q[1, :n], k[1, :n], v[1, :n], out[1, :n])
    with pytest.raises(ValueError):
        c.attend(1, q[1, :2], None, None, out[1, :2])
    assert all(torch.equal(x, y) for x, y in zip(before, (c.codes, c.scales, c.tails, out)))
    c.begin(3, c.lens)                                       # again, from its first layer
    layers(c, q, k, v, out)
    other, want = filled([40, 100, 7], width), torch.empty_like(out)
    other.begin(3, other.lens)
    layers(other, q, k, v, want)
    assert torch.equal(out, want) and torch.equal(c.tails, other.tails)


def test_a_layer_without_a_step():
    c = filled([40, 7])
    q, k, v = inputs(2)
    out = torch.empty((2, H, D), device=DEV)
    with pytest.raises(ValueError):
        c.attend(0, q[0], k[0], v[0], out)
    c.begin(2, c.lens)
    with pytest.raises(ValueError):
        c.begin(2, c.lens.long())                            # refused: there is no step any more
    with pytest.raises(ValueError):
        c.attend(0, q[0], k[0], v[0], out)


def test_layers_run_on_the_current_stream():
    """A layer's call on another stream than begin()'s comes after what that stream had to do before: here a long product, then q, k and v."""
    c, other_c = filled([40, 100, 7]), filled([40, 100, 7])
    q, k, v = inputs(3)
    want, out = (torch.empty((L, 3, H, D), device=DEV) for _ in range(2))
    other_c.begin(3, other_c.lens)
    layers(other_c, q, k, v, want)
    late = [torch.zeros_like(x) for x in (q, k, v)]
    a = torch.randn((8192, 8192), device=DEV)
    torch.cuda.synchronize()
    c.begin(3, c.lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(4):
            a = a @ a
            a = a / a.abs().max()
        for to, x in zip(late, (q, k, v)):
            to.copy_(x)
        layers(c, *late, out)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(c.tails, other_c.tails)


def test_captured_layers():
    """begin() and the layers in a graph, replayed with eager work in between, against eager steps."""
    c, other = filled([40, 31, 7]), filled([40, 31, 7])
    q, k, v = inputs(3)
    out, want = (torch.empty((L, 3, H, D), device=DEV) for _ in range(2))
    every, lens, n = ids(range(3)), c.lens.clone(), other.lens.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.begin(3, lens, every)
        layers(c, q, k, v, out)
        lens.add_(1)
    for i in range(5):
        for x in (q, k, v):
            x.normal_()
        graph.replay()
        torch.randn(1 << 14, device=DEV).sum().item()
        other.begin(3, n, every)
        layers(other, q, k, v, want)
        n.add_(1)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(c.tails, other.tails), i


def test_wrong_tensors_are_refused():
    """On the host, before anything is launched."""
    c = filled([40, 100, 7])
    q, k, v = (x[0] for x in inputs(3))
    out = torch.empty((3, H, D), device=DEV)
    before = [x.clone() for x in (c.codes, c.scales, c.tails)]
    good = dict(q=q, k_new=k, v_new=v, out=out)
    c.begin(3, c.lens)
    for bad in (dict(q=q.cpu()), dict(k_new=k.cpu()), dict(v_new=v.cpu()), dict(out=out.cpu()), dict(k_new=None), dict(v_new=None), dict(k_new=None, v_new=None),
                dict(q=q.float()), dict(q=q[:2]), dict(k_new=k[:, :1]), dict(v_new=v.float()), dict(v_new=v.transpose(0, 1)), dict(out=out.half()), dict(out=out[:2])):
        with pytest.raises(ValueError):
            c.attend(0, **{**good, **bad})
    c.begin(3, c.lens, appends=False)
    for bad in (dict(), dict(k_new=None), dict(v_new=None)):
        with pytest.raises(ValueError):
            c.attend(0, **{**good, **bad})
    assert all(torch.equal(x, y) for x, y in zip(before, (c.codes, c.scales, c.tails)))
