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
