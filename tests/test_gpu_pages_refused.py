"""What follows an extension that lacked pages: nothing grows and nothing is written until the caller has seen it, whatever the sequences of later calls."""
import numpy as np
import pytest
import torch

from oracle import pages as oracle
from paper_2504_11816_amd import binding
from paper_2504_11816_amd.cache8 import Cache8
from paper_2504_11816_amd.pages import Pages

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ids(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def test_an_accepted_extension_does_not_hide_a_refused_one():
    """Sequences 0 and 1 share a full page and find no others; sequence 3 has room in its own.  A step over all three must not write the first two's rows, which
    would go where their last tokens are, and into the page that they share."""
    rng = np.random.default_rng(1)
    H, G, d, T, L = 4, 2, 64, 32, 2
    c = Cache8(n_layers=L, n_q_heads=H, n_kv_heads=G, head_dim=d, page_tokens=T, n_pages=3, max_seqs=4, max_pages_per_seq=4, out_dtype=torch.float32, device=DEV)
    c.pages.extend(ids([0, 3]), ids([T, 5]))
    c.pages.fork(ids([0]), ids([1]))
    c.codes.copy_(torch.tensor(rng.integers(1, 255, c.codes.shape), dtype=torch.uint8))
    c.scales.copy_(torch.tensor(rng.random(c.scales.shape)))
    c.tails.copy_(torch.tensor(rng.standard_normal(c.tails.shape)))
    c.pages.check()
    state = (c.codes, c.scales, c.tails, c.table, c.lens, c.refs)
    before = [x.clone() for x in state]
    q, k, v = (torch.tensor(rng.standard_normal((L, 3, h, d)), dtype=torch.float16, device=DEV) for h in (H, G, G))
    out = torch.empty((L, 3, H, d), device=DEV)
    for layerwise in (False, True):
        c.pages.extend(ids([0, 1]))                          # two pages, one is free
        c.pages.extend(ids([3]))                             # room in its own page
        seqs = ids([0, 1, 3])
        if layerwise:
            c.begin(3, c.lens, seqs)
            for layer in range(L):
                c.attend(layer, q[layer], k[layer], v[layer], out[layer])
        else:
            c.step(q, k, v, out, c.lens, seqs)
        for x, y in zip(before, state):
            assert torch.equal(x, y)
        with pytest.raises(binding.OkvError) as e:
            c.pages.check()
        assert e.value.code == binding.OKV_ENOSPC
    # seen: the cache is as before the refused call, and what there is room for goes on
    c.pages.extend(ids([3]))
    c.step(q[:, :1].contiguous(), k[:, :1].contiguous(), v[:, :1].contiguous(), out[:, :1].contiguous(), c.lens, ids([3]))
    c.pages.check()
    assert c.lens.tolist() == [T, T, 0, 6]
    assert torch.equal(c.tails[:, 3, 0, :, 5], k[:, 0]) and torch.equal(c.tails[:, 3, 1, :, 5], v[:, 0])
    assert torch.equal(c.tails[:, :3], before[2][:, :3]) and torch.equal(c.codes, before[0])


def test_later_extensions_wait_until_the_status_is_cleared():
    T, S, width, n_pages = 4, 3, 3, 4
    table, lens, refs = torch.full((S, width), -1, dtype=torch.int32, device=DEV), ids([0] * S), ids([0] * n_pages)
    p, m = Pages(table=table, lens=lens, refs=refs, page_tokens=T), oracle.Model(n_pages, T, S, width)

    def do(name, *args):
        getattr(p, name)(*[ids(x) for x in args])
        getattr(m, name)(*args)
        assert (table.tolist(), lens.tolist(), refs.tolist(), p.status.tolist()[0]) == (m.table, m.lens, m.refs, m.status)

    do("extend", [0, 1], [6, 4])
    do("extend", [2, 0], [3, 5])                             # three pages, one is free
    assert m.status == binding.OKV_ENOSPC and p.status.tolist()[3] == binding.OKV_ENOSPC
    do("extend", [2], [1])                                   # there is a page, but nobody has looked
    do("free", [1])                                          # these go on
    do("fork", [0], [1])
    do("extend", [1], [1])
    assert lens.tolist() == [6, 6, 0]
    p.status[0] = 0                                          # a caller that clears the first word alone
    m.status = 0
    do("extend", [2], [1])
    assert lens.tolist() == [6, 6, 1] and p.status.tolist()[3] == 0
    do("extend", [0], [9])                                   # no room in the row of the table
    do("extend", [0], [1])
    with pytest.raises(binding.OkvError):
        p.check()
    m.status = 0
    do("extend", [0], [1])
    assert lens.tolist() == [7, 6, 1]


@pytest.mark.parametrize("rows,width", [(2, 1 << 30), (8, 1 << 28), (3, 1 << 30)])
def test_more_pages_than_are_counted_in_32_bits(rows, width):
    """A call whose sequences lack 2^31 pages and more together, each of them less: refused like any other that lacks some."""
    table = torch.full((rows, width), -1, dtype=torch.int32, device=DEV)
    lens, refs = torch.zeros(rows, dtype=torch.int32, device=DEV), torch.zeros(100, dtype=torch.int32, device=DEV)
    p = Pages(table=table, lens=lens, refs=refs, page_tokens=1)
    p.extend(ids(range(rows)), ids([width] * rows))
    assert p.status.tolist()[::3] == [binding.OKV_ENOSPC] * 2 and not lens.any() and not refs.any()
    p.status.zero_()
    p.extend(ids(range(rows)), ids(range(rows)))
    assert p.status.tolist()[0] == 0 and lens.tolist() == list(range(rows)) and int(refs.sum()) == sum(range(rows))
    assert [int(table[r, i]) for r in range(rows) for i in range(r + 1)] == [x for r in range(rows) for x in [*range(r * (r - 1) // 2, r * (r + 1) // 2), -1]]
