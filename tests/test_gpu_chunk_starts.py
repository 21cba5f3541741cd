"""Starts that do not ascend, in calls whose keys may be cut among workgroups: no access outside the buffers, the launch's own workspace included."""
import math

import numpy as np
import pytest
import torch

from paper_2504_11816_amd.cache16 import Cache16

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ids(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("B", (64, 130))
def test_more_items_than_workgroups(B):
    """Every second sequence takes all rows, so that there are some thirty times the tiles that n_rows rows make, and the last one is long enough to be cut: its pieces have no workgroup.  The workspace is full of
    descriptions of cut tiles that all name row 0 and results that are 0 (in range, should they be read): row 0 must not have them."""
    N, T, long = 4096, 256, 60000
    width = -(-(long + N) // T)
    c = Cache16(n_layers=1, n_q_heads=1, n_kv_heads=1, head_dim=64, page_tokens=T, n_pages=width, max_seqs=B, max_pages_per_seq=width, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    c.pool.copy_(torch.randn(c.pool.shape, generator=g, device=DEV, dtype=torch.float16))
    c.table.copy_(torch.arange(width, device=DEV).int().expand(B, width))
    c.lens.fill_(N)
    last = (B - 1) // 2 * 2
    c.lens[last] = long + N
    starts = ids([0 if b % 2 == 0 else N for b in range(B + 1)])
    q = torch.randn((N, 1, 64), generator=g, device=DEV, dtype=torch.float16)
    cut = ids([0, 1, 0, 0, 0, 0, 0, 1])                      # first row, rows, tile, head, slots of results, pieces
    for dtype in (torch.float16, torch.float32):
        c.workspace.zero_()
        at, n = 2048 + 16, 1024
        c.workspace[at:at + 32 * n] = cut.view(torch.uint8).repeat(n)
        around = torch.full((N + 2, 1, 64), math.nan, dtype=dtype, device=DEV)
        out = around[1:-1]
        c.attend(0, q, out, starts, c.lens)
        assert torch.isfinite(out).all() and out[0].any()
        assert around[0].isnan().all() and around[-1].isnan().all()


def test_ascending_starts_are_cut_as_before():
    """The long sequence of the same batch by itself beside empty ones: its keys are cut, and the results are those of a call with it alone."""
    N, T, long, B = 300, 256, 20000, 70
    width = -(-(long + N) // T)
    c = Cache16(n_layers=1, n_q_heads=2, n_kv_heads=2, head_dim=64, page_tokens=T, n_pages=width, max_seqs=B, max_pages_per_seq=width, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(2)
    c.pool.copy_(torch.randn(c.pool.shape, generator=g, device=DEV, dtype=torch.float16))
    c.table.copy_(torch.arange(width, device=DEV).int().expand(B, width))
    c.lens.fill_(long + N)
    rows = 32 * B + N                                        # (those behind the last sequence count where the form is chosen)
    q = torch.randn((rows, 2, 64), generator=g, device=DEV, dtype=torch.float16)
    out, alone = (torch.full((rows, 2, 64), math.nan, device=DEV) for _ in range(2))
    for o, starts, seqs in ((out, [0] * B + [N], range(B)), (alone, [0, N], [B - 1])):
        c.attend(0, q, o, ids(starts), c.lens, ids(seqs))
        assert int(c.workspace[2048:2052].view(torch.int32)[0]) > 0      # tiles that are cut
        assert o[N:].isnan().all()
    torch.testing.assert_close(out[:N], alone[:N], rtol=0, atol=2.0 ** -19)      # (weights of 22 bits, sums in another order; values of up to 4)
