"""Paged append and paged decode attention on the GPU against plain 64-bit forms."""
import math

import pytest
import torch

import paged_reference as ref
from paper_2510_06175_amd import binding as vb

pytestmark = pytest.mark.gpu


class Cache:
    """A pool with some free pages and a table of the sequences' pages, in no order."""

    def __init__(self, B, Hkv, D, P, N, dtype="fp16", token_major=False, seed=0, fill=True, spare=3):
        g = torch.Generator().manual_seed(seed)
        self.g, self.dtype, self.P, self.N, self.B = g, ref.DTYPES[dtype], P, N, B
        cols = -(-N // P)
        n = B * cols + spare
        self.table = torch.randperm(n, generator=g)[: B * cols].reshape(B, cols).to(torch.int32)
        shape = (n, P, Hkv, D) if token_major else (n, Hkv, P, D)
        make = lambda: (torch.randn(shape, generator=g) if fill else torch.zeros(shape)).to(self.dtype).cuda()  # noqa: E731
        k, v = make(), make()
        self.k, self.v = (k.transpose(1, 2), v.transpose(1, 2)) if token_major else (k, v)
        self.pages = vb.Pages(self.k, self.v)
        self.D, self.Hkv = D, Hkv

    def queries(self, Hq, scale=1.0):
        return (scale * torch.randn(self.B, Hq, self.D, generator=self.g)).to(self.dtype).cuda()


def attend(c, q, lens=None, N=None, splits=0, weights=None, scale=None, ws=None, w_in=None, check=True, table=None):
    """One call, checked against the reference; returns out, lse, weights."""
    B, Hq, D = q.shape
    N = c.N if N is None else N
    table = c.table if table is None else table
    out = torch.full((B, Hq, D), float("nan"), dtype=c.dtype, device="cuda")
    lse = torch.full((B, Hq), float("nan"), device="cuda")
    ws = vb.new_paged_workspace(c.pages, Hq, B, N, splits, weights=weights is not None) if ws is None else ws
    before = None if weights is None else weights.cpu().double()
    start = None if w_in is None else w_in.cpu().double()
    vb.vecinfer_paged_attention(c.pages, q, table.cuda(), ws, out, lse=lse, N=N, num_splits=splits, scale=scale,
                                seq_lens=None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                weights_in=w_in, weights_out=weights)
    torch.cuda.synchronize()
    if check:
        clamped = [N] * B if lens is None else [min(max(n, 0), N) for n in lens]
        want = ref.attention(q.cpu(), c.k.cpu(), c.v.cpu(), table, clamped, D ** -0.5 if scale is None else scale)
        ref.close(out, want["out"], want["tol_out"] + ref.half_step(want["out"].abs() + want["tol_out"], c.dtype), "out")
        ref.close(lse, want["lse"], want["tol_lse"], "lse")
        if weights is not None:
            for b, n in enumerate(clamped):
                w = want["weights"][b] + (0 if start is None else start[b, :, :n])
                ref.close(weights[b, :, :n], w, want["tol_w"][b] + (Hq // c.Hkv + 1) * 2.0 ** -23 * w.abs() + 2.0 ** -126, "weights")
                assert torch.equal(weights[b, :, n:].cpu().double(), before[b, :, n:])      # rows behind the end
    return out, lse, weights


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2), (14, 2), (5, 1), (16, 1), (12, 3)])
@pytest.mark.parametrize("P,N,splits", [(16, 100, 0), (8, 333, 3), (64, 1000, 0), (256, 700, 7), (1024, 1500, 2)])
def test_attention(dtype, D, Hq, Hkv, P, N, splits):
    c = Cache(3, Hkv, D, P, N, dtype, token_major=P == 16, seed=N)
    attend(c, c.queries(Hq, 2.0), [N, N // 3 + 1, N - 1], splits=splits)


@pytest.mark.parametrize("lens", [[0], [1], [2], [7], [8], [9], [31], [32], [33], [255], [256], [257], [0, 0], [0, 1, 300, 5], [-3, 1000]])
@pytest.mark.parametrize("splits", [0, 1, 5])
@pytest.mark.parametrize("weights", [False, True])
def test_lengths(lens, splits, weights):
    c = Cache(len(lens), 2, 128, 16, 300, seed=len(lens))
    w = torch.rand(len(lens), 2, 310, generator=c.g).cuda() if weights else None
    attend(c, c.queries(8), lens, splits=splits, weights=w)


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("splits", [1, 3])
def test_masked_rows_are_of_no_account(dtype, splits):
    """Infinities and NaN behind the end of a sequence, in free pages and in holes' neighbours."""
    c = Cache(3, 2, 128, 16, 150, dtype)
    lens = [70, 101, 0]
    q = c.queries(8)
    clean = attend(c, q, lens, splits=splits)
    free = sorted(set(range(c.k.shape[0])) - set(c.table.flatten().tolist()))
    for x, bad in ((c.k, float("nan")), (c.v, float("inf"))):
        x[free] = bad
        for b, n in enumerate(lens):
            for col in range(c.table.shape[1]):
                page = int(c.table[b, col])
                x[page, :, max(0, n - 16 * col):] = bad
    out, lse, _ = attend(c, q, lens, splits=splits, check=False)
    assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1])


@pytest.mark.parametrize("P", [8, 16, 64])
@pytest.mark.parametrize("splits", [0, 1, 4])
def test_holes(P, splits):
    c = Cache(4, 2, 64, P, 500, seed=P)
    c.table[0, ::2] = -1
    c.table[1, 1:] = c.k.shape[0]                           # one behind the last page
    c.table[2, :] = -(2 ** 31)                              # nothing left
    c.table[3, -1] = 2 ** 31 - 1
    w = torch.rand(4, 2, 500, generator=c.g).cuda()
    out, lse, _ = attend(c, c.queries(6), [500, 499, 500, 500], splits=splits, weights=w, w_in=torch.rand(4, 2, 500, device="cuda"))
    assert (out[2] == 0).all() and torch.isinf(lse[2]).all()


def test_scores_far_apart():
    """A token far above all others, and scores of the order of 10^4."""
    c = Cache(2, 2, 128, 16, 400)
    c.k[int(c.table[0, 20]), :, 3] *= 30
    attend(c, c.queries(8, 8.0))
    attend(c, c.queries(8, 100.0), scale=1.0)
    attend(c, c.queries(8), scale=-0.2)
    out, lse, _ = attend(c, c.queries(8), scale=0.0)
    assert (lse - math.log(400)).abs().max() < 1e-5


@pytest.mark.parametrize("dtype", ref.DTYPES)
def test_many_small_weights(dtype):
    """Ten thousand tokens of a weight far below the first one's, which together outweigh it."""
    c = Cache(1, 1, 64, 64, 10000, dtype, fill=False)
    q = torch.zeros(1, 1, 64, dtype=c.dtype, device="cuda")
    q[..., 0] = 1
    c.k[..., 0] = -6.0
    c.v[...] = 1.0
    first = int(c.table[0, 0])
    c.k[first, 0, 0, 0] = 0.0
    c.v[first, 0, 0] = -1.0
    attend(c, q, scale=1.0)


def test_scores_that_are_no_numbers():
    """A NaN or an infinite key among the attended tokens goes into its own heads' outputs, and no others'."""
    c = Cache(2, 2, 64, 16, 200)
    c.k[int(c.table[0, 3]), 0, 2, 5] = float("nan")
    c.k[int(c.table[0, 4]), 1, 2, 5] = float("inf")
    for splits in (1, 4):
        out, lse, _ = attend(c, c.queries(4), splits=splits, check=False)
        assert torch.isnan(out[0, :2]).all() and torch.isnan(lse[0, :2]).all()
        assert torch.isfinite(out[1]).all() and torch.isfinite(lse[1]).all()
    # keys of -inf alone: nothing to attend to
    c.k[...] = 0
    c.k[..., 0] = float("-inf")
    q = torch.ones(2, 4, 64, dtype=c.dtype, device="cuda")
    for splits in (1, 4):
        out, lse, _ = attend(c, q, splits=splits, check=False)
        assert (out == 0).all() and (lse == float("-inf")).all()


def test_splits_agree_and_repeat():
    c = Cache(2, 2, 128, 16, 4000, "bf16")
    q = c.queries(8)
    for s in (1, 2, 31, 32, 64, 65, 200, 256):
        a = attend(c, q, [4000, 37], splits=s)
        b = attend(c, q, [4000, 37], splits=s, check=False)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_strided_queries_and_wide_tables():
    c = Cache(2, 2, 128, 16, 200)
    big = torch.randn(2, 3, 8, 160, generator=c.g).to(c.dtype).cuda()
    q = big[:, 1, :, 8:136]
    a = attend(c, q)
    b = attend(c, q.contiguous())
    assert torch.equal(a[0], b[0])
    table = torch.full((2, 40), -1, dtype=torch.int32)       # a table for longer sequences
    table[:, : c.table.shape[1]] = c.table
    d = attend(c, q, table=table)
    assert torch.equal(a[0], d[0])


def test_shared_pages_and_the_same_page_twice():
    """Sequences that share pages keep sums of their own; a page that is named twice counts twice."""
    c = Cache(3, 2, 64, 16, 96)
    c.table[1, :4] = c.table[0, :4]
    c.table[2, 1] = c.table[2, 0]
    w = torch.zeros(3, 2, 96, device="cuda")
    attend(c, c.queries(4), weights=w)


def test_weights_in_place_and_without_a_start():
    c = Cache(2, 2, 128, 16, 130, "bf16")
    q = c.queries(8)
    w = torch.rand(2, 2, 140, generator=c.g).cuda()
    w0 = w.clone()
    _, _, apart = attend(c, q, [130, 9], weights=torch.zeros_like(w), w_in=w0)
    attend(c, q, [130, 9], weights=w, w_in=w)
    for b, n in ((0, 130), (1, 9)):
        assert torch.equal(w[b, :, :n], apart[b, :, :n]) and torch.equal(w[b, :, n:], w0[b, :, n:])
    _, _, own = attend(c, q, weights=torch.full_like(w, 7.0))
    assert (own[:, :, :130].sum(-1) - 4).abs().max() < 1e-4          # four heads' weights


def test_any_workspace():
    """A workspace of one split is enough, whatever it holds, and one too small is refused."""
    c = Cache(2, 2, 128, 16, 3000)
    q = c.queries(8)
    for w in (None, torch.zeros(2, 2, 3000, device="cuda")):
        least = vb.vecinfer_paged_workspace_bytes(c.pages, 8, 2, 3000, 1, w is not None)
        for fill in (0, 255, 1):
            for more in (0, 100000):
                attend(c, q, ws=torch.full((least + more,), fill, dtype=torch.uint8, device="cuda"), weights=w)
        with pytest.raises(vb.VecInferError) as e:
            attend(c, q, ws=torch.empty(least - 256, dtype=torch.uint8, device="cuda"), weights=w)
        assert e.value.code == vb.EWORKSPACE


def test_offsets_past_32_bits():
    """Pages behind 4 GiB of the pool."""
    n, P, D = 1 << 19, 64, 128                              # 8 GiB each
    k = torch.empty(n, 1, P, D, dtype=torch.float16, device="cuda")
    v = torch.empty_like(k)
    c = Cache(1, 1, D, P, 200)
    rows = torch.randn(4, 1, P, D, generator=c.g).half().cuda()
    at = torch.tensor([n - 1, 1 << 18, (1 << 18) - 1, 5], device="cuda")
    k[at], v[at] = rows, rows.flip(0)
    big = vb.Pages(k, v)
    q = c.queries(8)
    small = vb.Pages(rows.clone(), rows.flip(0).contiguous())
    outs = []
    for pages, table in ((big, at.int()[None]), (small, torch.arange(4, dtype=torch.int32, device="cuda")[None])):
        out = torch.empty(1, 8, D, dtype=torch.float16, device="cuda")
        vb.vecinfer_paged_attention(pages, q, table.contiguous(), vb.new_paged_workspace(pages, 8, 1, 200), out, N=200)
        outs.append(out)
    assert torch.equal(*outs)
    kn = torch.randn(1, 1, 130, D, generator=c.g).half().cuda()
    for pages, table in ((big, at.int()[None]), (small, torch.arange(4, dtype=torch.int32, device="cuda")[None])):
        vb.vecinfer_paged_append(pages, kn, kn, table.contiguous(), torch.tensor([256], dtype=torch.int32, device="cuda"))
    assert torch.equal(big.k[at], small.k) and torch.equal(big.v[at], small.v)


def test_streams_and_graphs():
    """Two captured calls that share a workspace, replayed with eager calls in between."""
    c = Cache(2, 2, 128, 16, 2000)
    qs = [c.queries(8) for _ in range(2)]
    ws = vb.new_paged_workspace(c.pages, 8, 2, 2000, weights=1)
    table = c.table.cuda()
    outs = [torch.empty(2, 8, 128, dtype=torch.float16, device="cuda") for _ in range(2)]
    sums = [torch.zeros(2, 2, 2000, device="cuda") for _ in range(2)]
    call = lambda i, out, w, **k: vb.vecinfer_paged_attention(c.pages, qs[i], table, ws, out, weights_out=w, N=2000, **k)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(0, outs[0], sums[0], stream=side)
    side.synchronize()
    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            call(i, outs[i], sums[i])
    for turn in range(3):
        for q in qs:
            q.copy_(torch.randn(q.shape, generator=c.g))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            out, w = torch.empty_like(outs[i]), torch.zeros_like(sums[i])
            call(i, out, w)
            torch.cuda.synchronize()
            assert torch.equal(out, outs[i]) and torch.equal(w, sums[i])


# ---- append


def append_reference(c, k_new, v_new, lens, new, rot, positions, q, q_out, before):
    """Every slot's and query's value in 64 bits with its bound, from the state `before` (k, v)."""
    k, v = before[0].double(), before[1].double()
    tk = torch.zeros_like(k)
    B, _, T, _ = k_new.shape
    qo = None if q is None else q_out.double().clone()
    tq = None if q is None else torch.zeros_like(qo)
    written = torch.zeros(k.shape[:3], dtype=torch.bool)
    for b in range(B):
        n = min(max(new[b], 0), T)
        at = torch.arange(n) + lens[b] - n
        pos = at if positions is None else positions[b, :n].long()
        if n == 0:
            continue
        rows, loose = (k_new[b:b + 1, :, :n].double(), torch.zeros(1, 1, 1, 1).expand(1, k.shape[1], n, 1)) if rot is None else \
            ref.rotary(rot, k_new[b:b + 1, :, :n], pos[None])
        if q is not None:
            qo[b, :, :n], tq[b, :, :n] = (x[0] for x in ref.rotary(rot, q[b:b + 1, :, :n], pos[None]))
        for t in range(n):
            a = int(at[t])
            if a < 0 or a // c.P >= c.table.shape[1]:
                continue
            page = int(c.table[b, a // c.P])
            if not 0 <= page < k.shape[0]:
                continue
            k[page, :, a % c.P], tk[page, :, a % c.P], v[page, :, a % c.P] = rows[0, :, t], loose[0, :, t], v_new[b, :, t].double()
            written[page, :, a % c.P] = True
    return k, tk, v, qo, tq, written


def append(c, T, lens, new=None, rot=None, positions=None, Hq=0, weights=None):
    B, Hkv, D = c.B, c.Hkv, c.D
    k_new, v_new = (torch.randn(B, T, Hkv, D, generator=c.g).to(c.dtype).transpose(1, 2) for _ in range(2))
    q = torch.randn(B, T, Hq, D, generator=c.g).to(c.dtype).transpose(1, 2) if Hq else None
    q_out = torch.full((B, Hq, T, D), 3.0, dtype=c.dtype) if Hq else None
    before = (c.k.cpu(), c.v.cpu())
    gpu = lambda x: None if x is None else torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda").copy_(x)  # noqa: E731
    ints = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    qo = gpu(q_out)
    vb.vecinfer_paged_append(c.pages, gpu(k_new), gpu(v_new), c.table.cuda(), ints(lens), new_lens=ints(new), rot=rot,
                             table=None if rot is None else vb.new_rotary_table(rot), q=gpu(q), q_out=qo,
                             positions=None if positions is None else positions.int().cuda(), weights=weights)
    torch.cuda.synchronize()
    k, tk, v, want_q, tq, written = append_reference(c, k_new, v_new, lens, [T] * B if new is None else new, rot, positions, q, q_out, before)
    got_k, got_v = c.k.cpu(), c.v.cpu()
    assert torch.equal(got_v.double(), v)
    assert torch.equal(got_k[~written], before[0][~written])
    ref.close(got_k, k, 1.01 * tk + torch.where(tk > 0, ref.half_step(k.abs() + tk, c.dtype), 0.0), "keys")
    if q is not None:
        ref.close(qo, want_q, 1.01 * tq + torch.where(tq > 0, ref.half_step(want_q.abs() + tq, c.dtype), 0.0), "queries")
    return written


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("D,R,interleaved", [(128, 128, 0), (128, 64, 1), (64, 64, 0), (64, 16, 1)])
@pytest.mark.parametrize("P,T", [(16, 1), (8, 9), (64, 130), (1024, 3)])
def test_append(dtype, D, R, interleaved, P, T):
    c = Cache(3, 2, D, P, 300, dtype, token_major=P == 16, seed=T)
    append(c, T, [T, T + 5, 299], rot=vb.Rotary(D, R, interleaved, base=10000.0), Hq=6)


@pytest.mark.parametrize("T,new", [(1, [1, 0, 1, 1]), (40, [40, 0, 13, 39]), (40, [50, -2, 1, 40]), (300, [300, 7, 299, 64])])
def test_append_a_padded_batch(T, new):
    c = Cache(4, 2, 128, 16, 320)
    append(c, T, [310, 50, 301, 64], new, rot=vb.Rotary(128, 128), Hq=8)


def test_append_where_nothing_is():
    """Holes, places behind the table and before the start: nothing is written, queries are turned all the same."""
    c = Cache(4, 2, 64, 16, 100, fill=True)
    c.table[0, 1] = -1
    c.table[1, 2] = c.k.shape[0]
    written = append(c, 60, [60, 130, 20, 2 ** 31 - 1], rot=vb.Rotary(64, 64), Hq=2)
    assert written.any()


def test_append_positions_and_no_rotation():
    c = Cache(2, 3, 128, 16, 64)
    append(c, 20, [20, 50])
    positions = torch.randint(0, 100000, (2, 20), generator=c.g)
    append(c, 20, [64, 33], rot=vb.Rotary(128, 128, base=500000.0), positions=positions, Hq=3)


@pytest.mark.parametrize("B,T", [(1, 2000), (300, 5)])
def test_append_many(B, T):
    c = Cache(B, 2, 64, 16, T, "bf16", fill=False)
    append(c, T, [T] * B, rot=vb.Rotary(64, 32), Hq=4)


@pytest.mark.parametrize("dtype", ref.DTYPES)
def test_append_more_than_the_caches_hold(dtype):
    c = Cache(2, 8, 128, 32, 1800, dtype, fill=False)
    append(c, 1750, [1800, 1400], [1750, 650], rot=vb.Rotary(128, 128), Hq=24)


def test_append_clears_weights():
    c = Cache(2, 2, 64, 16, 96)
    w = torch.rand(2, 2, 90, generator=c.g).cuda() + 1
    before = w.clone()
    append(c, 8, [40, 94], [8, 8], weights=w)
    want = before.clone()
    want[0, :, 32:40] = 0
    want[1, :, 86:90] = 0                                   # (tokens from 90 on have no sum)
    assert torch.equal(w, want)


def test_what_is_refused():
    c = Cache(2, 2, 64, 16, 96)
    table, q = c.table.cuda(), c.queries(4)
    ws, out = vb.new_paged_workspace(c.pages, 4, 2, 96), torch.empty(2, 4, 64, dtype=c.dtype, device="cuda")
    call = lambda **k: vb.vecinfer_paged_attention(**{**dict(pages=c.pages, q=q, block_table=table, workspace=ws, out=out), **k})  # noqa: E731
    call()
    for bad in (dict(q=q.bfloat16()), dict(q=q[:1]), dict(block_table=table.long()), dict(block_table=table[:, ::2]), dict(out=out[:, :2]),
                dict(lse=torch.empty(2, 4, device="cuda").half()), dict(seq_lens=torch.zeros(3, dtype=torch.int32, device="cuda")),
                dict(weights_out=torch.zeros(2, 3, 96, device="cuda"))):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(pages=c.k), dict(q=q.cpu()), dict(workspace=ws.cpu())):
        with pytest.raises(TypeError):
            call(**bad)
    for bad in (dict(N=97), dict(N=0), dict(num_splits=257), dict(weights_out=torch.zeros(2, 2, 95, device="cuda")),
                dict(weights_in=torch.zeros(2, 2, 0, device="cuda"))):
        with pytest.raises(vb.VecInferError):
            call(**bad)
    for k, v in ((c.k, c.v[:1]), (c.k, c.v.bfloat16()), (c.k.float(), c.v.float()), (c.k[0], c.v[0]), (c.k[:1].expand_as(c.k), c.v)):
        with pytest.raises(ValueError):
            vb.Pages(k, v)


@pytest.mark.parametrize("B,Hq,Hkv,D,N", [(2, 4, 4, 64, 4000), (5, 8, 2, 64, 5003), (9, 4, 1, 64, 4500), (20, 7, 1, 128, 4100), (64, 2, 2, 64, 4001),
                                          (65, 2, 1, 64, 4001)])
@pytest.mark.parametrize("how", ["spread", "one", "short", "none"])
def test_batches_dealt_by_length(B, Hq, Hkv, D, N, how):
    """Long batches with lengths of their own: sequences in proportion, one that has nearly all tokens, all but empty ones."""
    c = Cache(B, Hkv, D, 64, N, "bf16", seed=B)
    g = torch.Generator().manual_seed(B)
    lens = {"spread": torch.randint(0, N + 1, (B,), generator=g), "one": torch.where(torch.arange(B) == B // 2, N, 3), "short": torch.arange(B) % 3,
            "none": torch.zeros(B)}[how].int().tolist()
    w = torch.rand(B, Hkv, N, generator=g).cuda() if B < 20 else None
    attend(c, c.queries(Hq), lens, weights=w)


def test_dealt_batches_in_any_workspace():
    c = Cache(3, 2, 64, 64, 5000)
    q, lens = c.queries(8), [5000, 17, 1234]
    least, most = (vb.vecinfer_paged_workspace_bytes(c.pages, 8, 3, 5000, s) for s in (1, 0))
    for size in (least, (least + most) // 2 // 256 * 256, most):
        attend(c, q, lens, ws=torch.full((size,), 255, dtype=torch.uint8, device="cuda"))


def test_dealt_batches_in_a_graph():
    """Lengths that change between the replays."""
    c = Cache(4, 2, 64, 64, 4500)
    q, table, ws = c.queries(8), c.table.cuda(), vb.new_paged_workspace(c.pages, 8, 4, 4500, weights=1)
    lens = torch.tensor([4500, 3, 900, 0], dtype=torch.int32, device="cuda")
    out, w = torch.empty(4, 8, 64, dtype=c.dtype, device="cuda"), torch.zeros(4, 2, 4500, device="cuda")
    call = lambda o, s: vb.vecinfer_paged_attention(c.pages, q, table, ws, o, seq_lens=lens, N=4500, weights_out=s)  # noqa: E731
    call(out, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, w)
    for new in ([4500, 3, 900, 0], [1, 4500, 4500, 4500], [0, 0, 0, 0], [700, 4000, 2, 4499]):
        lens.copy_(torch.tensor(new, dtype=torch.int32))
        w.zero_()
        graph.replay()
        torch.cuda.synchronize()
        eager, sums = torch.empty_like(out), torch.zeros_like(w)
        call(eager, sums)
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(w, sums)
        want = ref.attention(q.cpu(), c.k.cpu(), c.v.cpu(), c.table, new, 0.125)
        ref.close(out, want["out"], want["tol_out"] + ref.half_step(want["out"].abs() + want["tol_out"], c.dtype), "out")


def test_two_streams_at_once():
    """Two calls with workspaces of their own, at the same time."""
    cs = [Cache(2, 2, 128, 16, 3000, seed=i) for i in range(2)]
    qs = [c.queries(8) for c in cs]
    want = [attend(c, q)[0] for c, q in zip(cs, qs)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(want[0]) for _ in range(20)] for _ in range(2)]
    wss, tables = [vb.new_paged_workspace(c.pages, 8, 2, 3000) for c in cs], [c.table.cuda() for c in cs]
    torch.cuda.synchronize()
    for turn in range(20):
        for i in range(2):
            vb.vecinfer_paged_attention(cs[i].pages, qs[i], tables[i], wss[i], outs[i][turn], N=3000, stream=streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in range(2) for o in outs[i])


def test_both_ways_into_the_library(monkeypatch):
    """The native argument checks and the interpreter's make the same calls."""
    c = Cache(2, 2, 64, 16, 200, "bf16")
    q = torch.randn(2, 9, 4, 64, generator=c.g).to(c.dtype).cuda()[:, 3]
    table, lens = c.table.cuda(), torch.tensor([200, 77], dtype=torch.int32, device="cuda")
    rot = vb.Rotary(64, 32, 1)
    rt = vb.new_rotary_table(rot)
    kn = torch.randn(2, 3, 2, 64, generator=c.g).to(c.dtype).cuda().transpose(1, 2)

    def everything():
        pages = vb.Pages(c.k.clone(), c.v.clone())
        out, lse, w = torch.empty(2, 4, 64, dtype=c.dtype, device="cuda"), torch.empty(2, 4, device="cuda"), torch.ones(2, 2, 200, device="cuda")
        qo = torch.zeros(2, 2, 3, 64, dtype=c.dtype, device="cuda")
        vb.vecinfer_paged_append(pages, kn, kn, table, lens, rot=rot, table=rt, q=kn, q_out=qo, weights=w)
        vb.vecinfer_paged_attention(pages, q, table, vb.new_paged_workspace(pages, 4, 2, 200, weights=1), out, lse=lse, seq_lens=lens, N=200,
                                    scale=0.3, weights_in=w, weights_out=w)
        dst, dl = vb.Pages(torch.zeros_like(c.k), torch.zeros_like(c.v)), torch.zeros(2, dtype=torch.int32, device="cuda")
        dw, kept = torch.zeros(2, 2, 50, device="cuda"), torch.zeros(2, 2, 50, dtype=torch.int32, device="cuda")
        vb.vecinfer_paged_evict(pages, w, table, dst, table, dl, vb.new_evict_workspace(pages, 2, 200, 50), 50, first=1, recent=5, seq_lens=lens,
                                N=200, dst_weights=dw, kept=kept)
        back = torch.empty_like(qo)
        vb.vecinfer_rotary(rot, rt, qo, back, pos0=4, inverse=True)
        torch.cuda.synchronize()
        return pages.k, pages.v, out, lse, w, qo, dst.k, dst.v, dl, dw, kept, back

    native = everything()
    assert vb._fast is not None
    monkeypatch.setattr(vb, "_fast", None)
    assert all(torch.equal(a, b) for a, b in zip(native, everything()))


@pytest.mark.parametrize("native", [True, False])
def test_another_device_is_refused(monkeypatch, native):
    """Tensors that are not on the current device: an error, and nothing is enqueued."""
    c = Cache(1, 2, 64, 16, 64)
    q, table, out = c.queries(4), c.table.cuda(), torch.full((1, 4, 64), 7.0, dtype=c.dtype, device="cuda")
    ws, rot = vb.new_paged_workspace(c.pages, 4, 1, 64), vb.Rotary(64, 64)
    rt, x = vb.new_rotary_table(rot), torch.ones(1, 2, 3, 64, dtype=c.dtype, device="cuda")
    lens = torch.tensor([3], dtype=torch.int32, device="cuda")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    if native:
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
        vb._bind_fast(vb.lib())
    else:
        monkeypatch.setattr(vb, "_fast", None)
    for call in (lambda: vb.vecinfer_paged_attention(c.pages, q, table, ws, out), lambda: vb.vecinfer_rotary(rot, rt, x, x),
                 lambda: vb.vecinfer_paged_append(c.pages, x, x, table, lens)):
        with pytest.raises(ValueError):
            call()
    monkeypatch.undo()
    vb._bind_fast(vb.lib())
    torch.cuda.synchronize()
    assert (out == 7).all() and (x == 1).all()
