"""Evictions from rows that several workgroups share, against the plain form."""
import pytest
import torch

from paper_2510_06175_amd import binding as vb
from test_gpu_evict import evict, weights
from test_gpu_paged import Cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,made,runs", [(40000, 7, (4, 5, 6, 7)), (65536, 3, (1, 2, 3)), (100003, 3, (2,))])
def test_a_workspace_of_more_sequences(N, made, runs):
    """One workspace, made for the largest batch and longest rows, for smaller ones after each other: the same as with their own."""
    c = Cache(made, 8, 64, 256, N, fill=False)
    w = weights(c, N).cuda()
    table, keep = c.table.cuda(), 1500
    big = vb.new_evict_workspace(c.pages, made, N, 2048)
    for B in runs:
        for n in (N, 33000, 5000):
            got = []
            for ws in (big, vb.new_evict_workspace(c.pages, B, n, keep)):
                dst = vb.Pages(*(torch.zeros(6 * B, 8, 256, 64, dtype=c.dtype, device="cuda") for _ in range(2)))
                dtable = torch.arange(6 * B, dtype=torch.int32, device="cuda").reshape(B, 6)
                lens, kept = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, 8, keep, dtype=torch.int32, device="cuda")
                vb.vecinfer_paged_evict(c.pages, w[:B], table[:B], dst, dtable, lens, ws, keep, first=4, recent=100, N=n, kept=kept)
                torch.cuda.synchronize()
                got.append((lens, kept))
            assert all(torch.equal(a, b) for a, b in zip(*got))
            assert (got[0][0] == keep).all()


@pytest.mark.parametrize("N,lens", [(40000, [40000, 20000, 33000]), (70000, [70000, 69999, 4097]), (300000, [300000, 1, 0])])
@pytest.mark.parametrize("how", ["spread", "ties"])
def test_everything_stays(N, lens, how):
    """Rows of as many tokens as may stay, or fewer, over several workgroups: each lists behind what those before it have."""
    c = Cache(len(lens), 1, 64, 1024, N, seed=N)
    evict(c, weights(c, N, how), N, 10, 200, lens=lens, dP=512)
    evict(c, weights(c, N, how), N + 500, 0, 0, lens=lens, dP=1024)


@pytest.mark.parametrize("holes", ["start", "end", "every other", "most", "all"])
@pytest.mark.parametrize("how", ["spread", "ties", "zero"])
@pytest.mark.parametrize("keep,first,recent", [(20500, 3000, 4000), (15000, 0, 0), (100, 20, 50)])
def test_holes(holes, how, keep, first, recent):
    """Holes in rows that workgroups share, so many that more may stay than are there, and fewer, which end among equal weights."""
    N, P = 40000, 64
    c = Cache(2, 2, 64, P, N, seed=keep)
    cols = c.table.shape[1]
    where = {"start": slice(0, cols // 3), "end": slice(cols // 2, cols), "every other": slice(1, cols, 2), "most": slice(5, cols - 3), "all": slice(0, cols)}[holes]
    c.table[0, where] = -1
    c.table[1, where] = c.k.shape[0] + 7
    evict(c, weights(c, N, how), keep, first, recent, lens=[N, N - 4321])
