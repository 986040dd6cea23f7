"""Eviction from a paged cache on the GPU against a plain form: what stays is decided by comparisons alone, so everything
is equal; and a life of a cache, from prompt to eviction and on, against dense attention in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paged_reference as ref
from paper_2510_06175_amd import binding as vb
from test_gpu_paged import Cache

pytestmark = pytest.mark.gpu


def evict(c, w, keep, first=0, recent=0, lens=None, N=None, dP=None, same_pool=False, with_kept=True, with_weights=True, holes=()):
    B, Hkv, D = c.B, c.Hkv, c.D
    N = min(c.N, w.shape[-1]) if N is None else N
    dP = c.P if dP is None else dP
    cols = -(-keep // dP)
    if same_pool:
        used = set(c.table.flatten().tolist())
        free = [i for i in range(c.k.shape[0]) if i not in used]
        dst, dk, dv = c.pages, c.k, c.v
        dtable = torch.tensor(free[: B * cols], dtype=torch.int32).reshape(B, cols)
    else:
        dk, dv = (torch.full((B * cols + 1, Hkv, dP, D), 5.0, dtype=c.dtype, device="cuda") for _ in range(2))
        dst = vb.Pages(dk, dv)
        dtable = torch.randperm(B * cols + 1, generator=c.g)[: B * cols].reshape(B, cols).to(torch.int32)
    for b, col, page in holes:
        dtable[b, col] = page
    before = (dk.cpu(), dv.cpu())
    dlens = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    dw = torch.full((B, Hkv, keep + 3), 9.0, device="cuda") if with_weights else None
    kept = torch.full((B, Hkv, keep), -9, dtype=torch.int32, device="cuda") if with_kept else None
    vb.vecinfer_paged_evict(c.pages, w.cuda(), c.table.cuda(), dst, dtable.cuda(), dlens, vb.new_evict_workspace(c.pages, B, N, keep), keep,
                            first=first, recent=recent, seq_lens=None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda"),
                            N=N, dst_weights=dw, kept=kept)
    torch.cuda.synchronize()
    clamped = [N] * B if lens is None else [min(max(n, 0), N) for n in lens]
    k, v = (x.clone() for x in before)
    want_w, want_kept = torch.full((B, Hkv, keep + 3), 9.0), torch.full((B, Hkv, keep), -9, dtype=torch.int32)
    src_k, src_v = c.k.cpu(), c.v.cpu()
    if same_pool:
        src_k, src_v = before
    for b, n in enumerate(clamped):
        ids = ref.evict(w[b, :, :n].cpu(), c.table[b], c.k.shape[0], c.P, n, keep, first, recent)
        assert len({len(i) for i in ids}) == 1
        m = len(ids[0])
        assert int(dlens[b]) == m
        for h in range(Hkv):
            i = torch.from_numpy(ids[h])
            want_kept[b, h, :m], want_w[b, h, :m] = i.int(), w[b, h, i].float().cpu()
            page = c.table[b, i // c.P].long()
            to = torch.arange(m)
            dpage = dtable[b, to // dP].long()
            ok = (dpage >= 0) & (dpage < dk.shape[0])
            for d, s in ((k, src_k), (v, src_v)):
                d[dpage[ok], h, (to % dP)[ok]] = s[page, h, i % c.P][ok]
    if with_kept:
        assert torch.equal(kept.cpu(), want_kept)
    if with_weights:
        assert torch.equal(dw.cpu().view(torch.int32), want_w.view(torch.int32))
    bits = lambda x: x.cpu().contiguous().view(torch.int16)  # noqa: E731
    assert torch.equal(bits(dk), bits(k)) and torch.equal(bits(dv), bits(v))
    return dlens, kept


def weights(c, N, how="spread"):
    w = torch.rand(c.B, c.Hkv, N, generator=c.g)
    if how == "ties":
        return torch.floor(w * 3) / 8
    if how == "zero":
        return torch.zeros_like(w)
    if how == "bits":                            # every kind of number
        return torch.randint(-2 ** 31, 2 ** 31, w.shape, generator=c.g).int().view(torch.float32)
    if how == "close":                           # one value's neighbours
        return (torch.randint(0, 5, w.shape, generator=c.g).int() + 0x3f800000).view(torch.float32)
    return torch.exp(6 * w)


@pytest.mark.parametrize("how", ["spread", "ties", "zero", "bits", "close"])
@pytest.mark.parametrize("D,P,dP,dtype", [(128, 16, 16, "fp16"), (64, 8, 64, "bf16"), (128, 256, 32, "bf16")])
@pytest.mark.parametrize("N,keep,first,recent", [(1000, 300, 4, 50), (1025, 1024, 0, 0), (2500, 1, 0, 0), (700, 64, 64, 0), (900, 77, 0, 77),
                                                (333, 100, 50, 50)])
def test_evict(how, D, P, dP, dtype, N, keep, first, recent):
    c = Cache(2, 3, D, P, N, dtype, token_major=P == 16, seed=keep)
    evict(c, weights(c, N, how), keep, first, recent, dP=dP)


@pytest.mark.parametrize("lens", [[0], [1], [5], [63], [64], [65], [128], [400], [0, 1, 64, 500, -2, 33]])
@pytest.mark.parametrize("keep,first,recent", [(64, 0, 0), (64, 4, 32), (1, 0, 1), (450, 0, 10)])
def test_lengths(lens, keep, first, recent):
    c = Cache(len(lens), 2, 64, 16, 400, seed=len(lens))
    evict(c, weights(c, 410, "ties"), keep, first, recent, lens=lens)


@pytest.mark.parametrize("N", [1023, 1024, 1025, 20000, 70001])
@pytest.mark.parametrize("how", ["spread", "ties"])
def test_long(N, how):
    c = Cache(1, 2, 64, 64, N, seed=N)
    evict(c, weights(c, N, how), N // 3, 10, N // 6)


@pytest.mark.parametrize("N,lens", [(16385, [16385, 16384, 1]), (32768, [32768, 16383, 1]), (32769, [32769, 0, 300]),
                                    (40000, [40000, 39999, 8191, 8193, 16384, 5])])
@pytest.mark.parametrize("how", ["zero", "bits", "close"])
def test_rows_of_one_or_more_workgroups(N, lens, how):
    c = Cache(len(lens), 1, 64, 1024, N, seed=N)
    evict(c, weights(c, N, how), 5000, 100, 1000, lens=lens)


def test_very_long():
    """More tokens than the registers of all workgroups of a row hold."""
    c = Cache(1, 1, 64, 256, 1100003, fill=False)
    evict(c, weights(c, 1100003), 1000, 3, 400)


def test_many_long_rows():
    c = Cache(24, 8, 64, 64, 20000, fill=False)
    evict(c, weights(c, 20000, "ties"), 300, 3, 40, lens=[20000 - 700 * i for i in range(24)])


@pytest.mark.parametrize("D,B,keep", [(128, 4, 2103), (64, 8, 2103)])
def test_more_than_the_caches_hold(D, B, keep):
    c = Cache(B, 8, D, 32, 4003, token_major=D == 64, seed=D)
    evict(c, weights(c, 4003), keep, 4, 100, lens=[4003 - 300 * i for i in range(B)], dP=64)


def test_special_weights():
    """-0 equals 0, infinities are ordered, what is no number comes below them, and ties go to the lowest index."""
    c = Cache(1, 1, 64, 8, 12)
    inf, nan = float("inf"), float("nan")
    w = torch.tensor([[[0.0, -0.0, nan, -inf, inf, 1.0, -1.0, -0.0, 0.0, nan, inf, -inf]]])
    order = [4, 10, 5, 0, 1, 7, 8, 6, 3, 11, 2, 9]
    for keep in range(1, 13):
        _, kept = evict(c, w, keep)
        assert kept[0, 0].tolist() == sorted(order[:keep])


def test_holes():
    c = Cache(3, 2, 64, 16, 200)
    c.table[0, 3] = -1
    c.table[1, 1:] = c.k.shape[0] + 5
    c.table[2, :] = -1
    w = weights(c, 200)
    evict(c, w, 60, 20, 20)
    evict(c, w, 200, 0, 0)
    evict(c, w, 60, 20, 20, holes=[(0, 0, -1), (1, 0, 10 ** 6)])


def test_options():
    c = Cache(2, 2, 128, 16, 300, spare=40)
    w = weights(c, 300)
    evict(c, w, 100, 3, 20, with_kept=False)
    evict(c, w, 100, 3, 20, with_weights=False)
    evict(c, w, 100, 3, 20, N=250)
    evict(c, w, 100, 3, 20, same_pool=True)


def test_a_batch_of_many():
    c = Cache(40, 8, 64, 16, 128, seed=3)
    evict(c, weights(c, 128, "ties"), 50, 2, 10, lens=[int(x) for x in torch.randint(0, 129, (40,), generator=c.g)])


def test_stream_and_graph():
    c = Cache(2, 2, 64, 16, 500)
    w = weights(c, 500).cuda()
    dk, dv = (torch.zeros(14, 2, 16, 64, dtype=c.dtype, device="cuda") for _ in range(2))
    dst, dtable = vb.Pages(dk, dv), torch.arange(14, dtype=torch.int32, device="cuda").reshape(2, 7)
    ws, table = vb.new_evict_workspace(c.pages, 2, 500, 100), c.table.cuda()
    dl, dw, kept = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 2, 100, device="cuda"), torch.zeros(2, 2, 100, dtype=torch.int32, device="cuda")
    call = lambda **k: vb.vecinfer_paged_evict(c.pages, w, table, dst, dtable, dl, ws, 100, first=2, recent=9, dst_weights=dw, kept=kept, **k)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        w.copy_(weights(c, 500))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (dk, dv, dl, dw, kept)]
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (dk, dv, dl, dw, kept)))


def test_what_is_refused():
    c = Cache(2, 2, 64, 16, 96)
    w = weights(c, 96).cuda()
    table, dl = c.table.cuda(), torch.zeros(2, dtype=torch.int32, device="cuda")
    dst = vb.Pages(*(torch.zeros(4, 2, 16, 64, dtype=c.dtype, device="cuda") for _ in range(2)))
    dtable, ws = torch.arange(4, dtype=torch.int32, device="cuda").reshape(2, 2), vb.new_evict_workspace(c.pages, 2, 96, 32)
    call = lambda **k: vb.vecinfer_paged_evict(**{**dict(pages=c.pages, weights=w, block_table=table, dst_pages=dst, dst_table=dtable,  # noqa: E731
                                                         dst_lens=dl, workspace=ws, keep=32), **k})
    call()
    other = vb.Pages(*(torch.zeros(4, 2, 16, 128, dtype=c.dtype, device="cuda") for _ in range(2)))
    for bad in (dict(keep=33), dict(keep=0), dict(first=20, recent=20), dict(dst_pages=other), dict(N=97), dict(seq_lens=dl),
                dict(dst_weights=torch.zeros(2, 2, 31, device="cuda")), dict(workspace=ws[:0])):
        with pytest.raises(vb.VecInferError):
            call(**bad)
    for bad in (dict(weights=w.half()), dict(weights=w[:1]), dict(kept=torch.zeros(2, 2, 31, dtype=torch.int32, device="cuda")),
                dict(dst_lens=dl[:1]), dict(dst_table=dtable.long())):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(TypeError):
        call(dst_pages=c.k)


@pytest.mark.parametrize("dtype", ref.DTYPES)
def test_a_life_of_a_cache(dtype):
    """Prompts of a padded batch, decode steps that sum their weights, an eviction into other pages, and more steps with
    the text's positions: every output against dense attention over the rows that are left, kept here in 64 bits."""
    B, Hq, Hkv, D, P, cap, keep = 2, 8, 2, 64, 16, 160, 48
    G, dt = Hq // Hkv, ref.DTYPES[dtype]
    g = torch.Generator().manual_seed(11)
    rot = vb.Rotary(D, D, base=10000.0, scaling=vb.ROTARY_PARTS, factor=4.0, orig_len=128, low_turns=1.0, high_turns=4.0)
    table_r = vb.new_rotary_table(rot)
    cols = cap // P
    k, v = (torch.zeros(3 * B * cols, Hkv, P, D, dtype=dt, device="cuda") for _ in range(2))
    pages = vb.Pages(k, v)
    order = torch.randperm(3 * B * cols, generator=g).to(torch.int32)
    tables = [order[i * B * cols:(i + 1) * B * cols].reshape(B, cols).cuda() for i in range(2)]
    table, free = tables
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    sums = torch.full((B, Hkv, cap), 99.0, device="cuda")
    ws = vb.new_paged_workspace(pages, Hq, B, cap, weights=1)
    # the rows as they were stored, and the weights: [b][h] -> [n, D] in 64 bits
    K, V = [[torch.zeros(0, D, dtype=torch.float64)] * Hkv for _ in range(B)], [[torch.zeros(0, D, dtype=torch.float64)] * Hkv for _ in range(B)]
    W = [[torch.zeros(0, dtype=torch.float64)] * Hkv for _ in range(B)]
    text, length = [70, 41], [70, 41]

    def put(T, new):
        kn, vn, q = (torch.randn(B, H, T, D, generator=g).to(dt) for H in (Hkv, Hkv, Hq))
        q_out = torch.zeros(B, Hq, T, D, dtype=dt, device="cuda")
        pos = torch.stack([torch.arange(T) + text[b] - new[b] for b in range(B)]).int()
        vb.vecinfer_paged_append(pages, kn.cuda(), vn.cuda(), table, ints(length), new_lens=ints(new), rot=rot, table=table_r, positions=pos.cuda(),
                                 q=q.cuda(), q_out=q_out, weights=sums)
        for b in range(B):
            want, loose = ref.rotary(rot, kn[b:b + 1, :, :new[b]], pos[b:b + 1, :new[b]])
            at = torch.arange(length[b] - new[b], length[b])
            stored = k[table[b].cpu().long()[at // P], :, at % P].cpu().double().transpose(0, 1)
            ref.close(stored, want[0], 1.01 * loose[0] + ref.half_step(want[0].abs() + loose[0], dt), "stored keys")
            for h in range(Hkv):
                K[b][h] = torch.cat([K[b][h], stored[h]])
                V[b][h] = torch.cat([V[b][h], vn[b, h, :new[b]].double()])
                W[b][h] = torch.cat([W[b][h], torch.zeros(new[b], dtype=torch.float64)])
        return q_out

    def step():
        for b in range(B):
            text[b] += 1
            length[b] += 1
        q = put(1, [1] * B)[:, :, 0]
        out, lse = torch.empty(B, Hq, D, dtype=dt, device="cuda"), torch.empty(B, Hq, device="cuda")
        vb.vecinfer_paged_attention(pages, q, table, ws, out, lse=lse, seq_lens=ints(length), N=cap, weights_in=sums, weights_out=sums)
        torch.cuda.synchronize()
        for b in range(B):
            for h in range(Hq):
                kk, vv, qq = K[b][h // G], V[b][h // G], q[b, h].double().cpu()
                s = kk @ qq / math.sqrt(D)
                p = torch.softmax(s, 0)
                # (as in paged_reference.attention; |s| stays below 16 here, a row's |k| |q| below 2^9)
                d = (D + 8) * 2.0 ** -23 * float((kk.abs() @ qq.abs()).max()) / math.sqrt(D) + 2.0 ** -18
                tol = (p @ vv.abs()) * (2 * d + 300 * 2.0 ** -23 + 2.0 ** -16)
                ref.close(out[b, h], p @ vv, tol + ref.half_step((p @ vv).abs() + tol, dt), "step")
                W[b][h // G] = W[b][h // G] + p
        for b in range(B):
            for h in range(Hkv):
                assert (sums[b, h, :length[b]].cpu().double() - W[b][h]).abs().max() < 1e-3      # (only the order of evictions hangs on it)

    put(70, [70, 41])
    for _ in range(6):
        step()
    for _ in range(2):
        new_lens, new_sums, kept = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full_like(sums, 99.0), torch.zeros(B, Hkv, keep, dtype=torch.int32, device="cuda")
        vb.vecinfer_paged_evict(pages, sums, table, pages, free, new_lens, vb.new_evict_workspace(pages, B, cap, keep), keep, first=2, recent=8,
                                seq_lens=ints(length), N=cap, dst_weights=new_sums, kept=kept)
        torch.cuda.synchronize()
        for b in range(B):
            n = min(keep, length[b])
            assert int(new_lens[b]) == n
            ids = ref.evict(sums[b, :, :length[b]].cpu(), table[b].cpu(), k.shape[0], P, length[b], keep, 2, 8)
            for h in range(Hkv):
                assert np.array_equal(kept[b, h, :n].cpu().numpy(), ids[h])
                i = torch.from_numpy(ids[h])
                K[b][h], V[b][h], W[b][h] = K[b][h][i], V[b][h][i], W[b][h][i]
            length[b] = n
        table, free, sums = free, table, new_sums
        for _ in range(5):
            step()


def test_turned_keys_go_into_the_quantized_cache(oracle):
    """vecinfer_rotary's output is what vecinfer_encode_keys takes: codes of turned keys."""
    rot = vb.Rotary(128, 128)
    g = torch.Generator().manual_seed(2)
    k = torch.randn(1, 40, 2, 128, generator=g).half().cuda().transpose(1, 2)
    turned = torch.empty(1, 2, 40, 128, dtype=torch.float16, device="cuda")
    vb.vecinfer_rotary(rot, vb.new_rotary_table(rot), k, turned, pos0=1000)
    cfg = vb.Config(128, 8, 2, 4, 4)
    lam, cb = torch.ones(2, 128, device="cuda"), torch.randn(cfg.cb_shape(True), generator=g).half().cuda()
    idx = torch.zeros(1, 2, 40, 32, dtype=torch.uint8, device="cuda")
    vb.vecinfer_encode_keys(cfg, turned, lam, cb, idx)
    want, gap = oracle.encode_keys(turned.cpu().numpy(), lam.cpu().numpy(), cb.cpu().numpy(), want_gap=True)
    differ = idx.cpu().numpy() != want
    assert not (differ & (gap >= 1e-6)).any()
