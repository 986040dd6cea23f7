"""More tokens in one call than a grid has workgroups along an axis."""
import torch

import paged_reference as ref
import pytest
from paper_2510_06175_amd import binding as vb

pytestmark = pytest.mark.gpu


def test_rotary():
    T = 2 ** 26 + 5
    rot = vb.Rotary(64, 64)
    x = torch.empty(1, 1, T, 64, dtype=torch.float16, device="cuda")
    x.view(-1, 64).copy_(torch.randn(1, 64, generator=torch.Generator().manual_seed(1)).half().cuda().expand(T, 64))
    at = torch.tensor([0, 1, 2 ** 24 - 1, 2 ** 24, 2 ** 25 + 3, 2 ** 26 - 1, 2 ** 26, 2 ** 26 + 3, T - 1])
    before = x[:, :, at.cuda()].cpu()
    vb.vecinfer_rotary(rot, vb.new_rotary_table(rot), x, x)
    want, loose = ref.rotary(rot, before, at[None])
    # (the reference's own angle, a product in 64 bits below 2^26, is off by 2^-27 at most, below 2^-21 of the pair)
    ref.close(x[:, :, at.cuda()], want, 1.02 * loose + ref.half_step(want.abs() + loose, x.dtype), "rows")


def test_append():
    T, P = 2 ** 26 + 5, 1024
    k, v = (torch.zeros(2, 1, P, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.full((1, -(-T // P)), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[0, -1] = 0, 1
    row = torch.randn(2, 64, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    vb.vecinfer_paged_append(vb.Pages(k, v), row[0].expand(1, 1, T, 64), row[1].expand(1, 1, T, 64), table,
                             torch.tensor([T], dtype=torch.int32, device="cuda"))
    n = T % P
    assert torch.equal(k[0, 0], row[0].expand(P, 64)) and torch.equal(v[0, 0], row[1].expand(P, 64))
    assert torch.equal(k[1, 0, :n], row[0].expand(n, 64)) and torch.equal(v[1, 0, :n], row[1].expand(n, 64))
    assert (k[1, 0, n:] == 0).all() and (v[1, 0, n:] == 0).all()


def test_evict():
    N, P = 2 ** 28 + 100, 1024
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn(3, 1, P, 128, generator=g, dtype=torch.float16, device="cuda") for _ in range(2))
    dk, dv = torch.zeros_like(k), torch.zeros_like(v)
    cols = -(-N // P)
    table = (torch.arange(cols, dtype=torch.int32, device="cuda") % 3)[None].contiguous()
    dtable = torch.full((1, cols), -1, dtype=torch.int32, device="cuda")
    dtable[0, 0], dtable[0, cols - 2], dtable[0, cols - 1] = 0, 1, 2
    pages = vb.Pages(k, v)
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    vb.vecinfer_paged_evict(pages, torch.zeros(1, 1, N, device="cuda"), table, vb.Pages(dk, dv), dtable, lens, vb.new_evict_workspace(pages, 1, N, N), N)
    torch.cuda.synchronize()
    assert int(lens[0]) == N
    for dst, src in ((dk, k), (dv, v)):
        assert torch.equal(dst[0], src[0]) and torch.equal(dst[1], src[(cols - 2) % 3])
        n = N % P
        assert torch.equal(dst[2, :, :n], src[(cols - 1) % 3, :, :n]) and (dst[2, :, n:] == 0).all()
