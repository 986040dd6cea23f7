"""The operators around a full-precision paged cache, as timed cases: rotary positions, the append to the cache's
pages, the attention of one new token over them (with and without the sums of attention weight that an eviction goes
by), and the eviction.

    listed()            named cases over the range of sizes, types and layouts in use
    draw(rng)           one more case of the same ranges
    prepare(case, seed) what a program holds before the call, on the GPU
    run(state)          one pass and its outputs: plain torch operations, or with `own` the library's entry points
    exact(case, seed)   the same outputs from the definitions, in 64 bits
    work(case)          bytes and operations of one pass that nothing can save

Kinds of case (`kind`):
    rotary  one tensor of queries or keys turned by its positions (or, `inverse`, its gradient turned back)
    append  T new tokens per sequence: queries and keys turned, keys and values written to their pages
    attend  one new token per sequence attends to its pages
    weigh   the same, and every cached token's weight is added to its sum
    evict   the tokens of most weight, the first and the most recent ones move to pages of their own
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _case(kind, dtype, B, Hq, Hkv, D, N, **more):
    return dict({"kind": kind, "dtype": dtype, "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "N": N}, **more)


def listed():
    c = lambda name, *a, **k: dict(_case(*a, **k), name=name)  # noqa: E731
    return [
        # the queries of one token far into a text: launch latency is what it costs
        c("rotary-1", "rotary", "fp16", 1, 32, 8, 128, 1, rot=128, pos0=100003),
        # the queries of a prompt, positions stretched for a long context
        c("rotary-8k", "rotary", "bf16", 1, 32, 8, 128, 8192, rot=128, scaling="parts", factor=8.0, pos0=0),
        # gradients of the keys of a training batch: adjacent pairs, half of the head
        c("rotary-grad", "rotary", "fp16", 3, 8, 8, 128, 4099, rot=64, interleaved=1, scaling="base", factor=4.0, pos0=0, inverse=1),
        # decode-time append of a batch of different lengths
        c("append-32", "append", "fp16", 32, 32, 8, 128, 1, rot=128, past=500, page=16, ragged=1),
        # prompts of a padded batch
        c("append-prompts", "append", "bf16", 4, 32, 8, 128, 2048, rot=128, scaling="parts", factor=8.0, past=0, page=16, ragged=1),
        # a chat turn's first tokens: one sequence, a short cache
        c("attend-1000", "attend", "fp16", 1, 32, 8, 128, 1000, page=16),
        # a serving batch: 32 sequences of different lengths, up to 8192 tokens
        c("attend-batch32", "attend", "bf16", 32, 32, 8, 128, 8192, page=16, ragged=1),
        # the longest context the layer is benchmarked on
        c("attend-196k", "attend", "fp16", 1, 32, 8, 128, 196608, page=64),
        # head dim 64, seven query heads per KV head, pages with a token's heads side by side
        c("attend-d64", "attend", "bf16", 4, 28, 4, 64, 30001, page=32, token_major=1),
        # a long document whose cache is to be cut later: weights are summed
        c("weigh-32k", "weigh", "fp16", 2, 32, 8, 128, 32768, page=16, ragged=1),
        # a serving batch cut to a quarter
        c("evict-batch8", "evict", "bf16", 8, 32, 8, 128, 8192, page=16, keep=2048, first=4, recent=512, ragged=1),
        # one long document cut to a third
        c("evict-100k", "evict", "fp16", 1, 32, 8, 128, 100003, page=64, keep=32768, first=16, recent=4096),
    ]


def _log(rng, lo, hi):
    """An integer from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    kind = rng.choices(["rotary", "append", "attend", "weigh", "evict"], [3, 3, 6, 2, 3])[0]
    dtype = rng.choice(["fp16", "bf16"])
    D = rng.choices([128, 64], [3, 1])[0]
    Hq, Hkv = rng.choices([(32, 8), (28, 4), (64, 8), (16, 8), (8, 8), (40, 8)], [5, 1, 1, 1, 1, 1])[0]
    more = {}
    if kind in ("rotary", "append"):
        more["rot"] = rng.choice([D, D, D // 2, 16])
        if rng.random() < 0.4:
            more["interleaved"] = 1
        if rng.random() < 0.6:
            more["scaling"], more["factor"] = rng.choice(["linear", "base", "parts"]), rng.choice([2.0, 8.0, 32.0])
    else:
        more["page"] = rng.choice([8, 16, 16, 32, 64, 256])
        if rng.random() < 0.3:
            more["token_major"] = 1
    B = rng.choice([1, 1, 2, 3, 4, 8, 16, 32])
    if kind == "rotary":
        if rng.random() < 0.4:
            more["inverse"] = 1
        return _case(kind, dtype, B, Hq, Hkv, D, _log(rng, 1, 48000000 // (B * Hq * D)), pos0=rng.choice([0, rng.randint(1, 1000000)]), **more)
    if B > 1 and rng.random() < 0.7:
        more["ragged"] = 1
    if kind == "append":
        T = rng.choice([1, 1, 1, _log(rng, 2, 24000000 // (B * (Hq + 2 * Hkv) * D))])
        return _case(kind, dtype, B, Hq, Hkv, D, T, past=rng.choice([0, rng.randint(1, 600)]), page=rng.choice([8, 16, 16, 32, 64, 256]), **more)
    most = min(196608, int((6.0e8 if kind != "evict" else 2.0e8) / (B * Hkv * D * 4)))      # no more than the largest listed cache
    N = _log(rng, 300 if kind != "attend" else 20, most)
    if kind == "evict":
        more["keep"] = max(24, int(N * rng.choice([0.1, 0.25, 0.5, 0.9])))
        more["first"], more["recent"] = rng.choice([0, 1, 4]), rng.choice([0, more["keep"] // 4, more["keep"] // 2])
    return _case(kind, dtype, B, Hq, Hkv, D, N, **more)


def _lengths(case):
    """Tokens attended per sequence; lengths of a ragged batch are spread evenly from an eighth of N to N."""
    B, N = case["B"], case["N"]
    if not case.get("ragged"):
        return [N] * B
    return [max(1, N // 8 + (N - N // 8) * (i + 1) // B) for i in range(B)]


def _past(case):
    """Tokens that a sequence holds before an append."""
    return [case["past"] * (i + 1) // case["B"] if case.get("ragged") else case["past"] for i in range(case["B"])]


def _frequencies(case):
    """Angle per position of every pair, in 64 bits."""
    R, base, s = case["rot"], 500000.0, case.get("factor", 1.0)
    i = np.arange(R // 2, dtype=np.float64)
    how = case.get("scaling")
    if how == "base":
        base = base * s ** (R / (R - 2.0))
    f = base ** (-2.0 * i / R)
    if how == "linear":
        f = f / s
    if how == "parts":                  # by the turns that a pair makes in the original context
        g = np.clip((8192 * f / (2 * math.pi) - 1.0) / (4.0 - 1.0), 0.0, 1.0)
        f = (1 - g) * f / s + g * f
    return f


class _Draws:
    """Seeded tensors on the GPU."""

    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))
        self.dtype = dtype

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=self.dtype)

    def order(self, n):
        return torch.randperm(n, generator=self.g, device="cuda")


def _pool(r, n, Hkv, P, D, token_major, fill):
    shape = (n, P, Hkv, D) if token_major else (n, Hkv, P, D)
    x = r.normal(*shape) if fill else torch.zeros(shape, dtype=r.dtype, device="cuda")
    return x.transpose(1, 2) if token_major else x


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    r = _Draws(seed, TYPES[case["dtype"]])
    kind, B, Hq, Hkv, D, N = (case[k] for k in ("kind", "B", "Hq", "Hkv", "D", "N"))
    s = {"case": case}
    if own:
        from paper_2510_06175_amd import binding as vb
    if kind in ("rotary", "append"):
        if own:
            how = {None: vb.ROTARY_PLAIN, "linear": vb.ROTARY_LINEAR, "base": vb.ROTARY_BASE, "parts": vb.ROTARY_PARTS}[case.get("scaling")]
            s["rot"] = vb.Rotary(D, case["rot"], interleaved=case.get("interleaved", 0), base=500000.0, scaling=how,
                                 factor=case.get("factor", 1.0), orig_len=8192, low_turns=1.0, high_turns=4.0)
            s["table"] = vb.new_rotary_table(s["rot"])
        else:
            s["freqs"] = torch.from_numpy(_frequencies(case)).cuda()
    if kind == "rotary":
        # (queries as a projection leaves them: tokens, then heads)
        s["x"] = r.normal(B, N, Hq, D).transpose(1, 2)
        s["positions"] = None
        if case.get("pos0"):
            s["positions"] = (_ints([[case["pos0"]]]) + torch.arange(N, dtype=torch.int32, device="cuda")).expand(B, N).contiguous()
        s["out"] = torch.empty(B, Hq, N, D, dtype=r.dtype, device="cuda")
        return s
    P = case["page"]
    if kind == "append":
        past, lens = _past(case), _lengths(case)
        total = [a + b for a, b in zip(past, lens)]
        pages = -(-max(total) // P)
        s["k"], s["v"] = r.normal(B, N, Hkv, D).transpose(1, 2), r.normal(B, N, Hkv, D).transpose(1, 2)
        s["q"] = r.normal(B, N, Hq, D).transpose(1, 2)
        s["q_out"] = torch.zeros(B, Hq, N, D, dtype=r.dtype, device="cuda")
        s["table_b"] = r.order(B * pages).reshape(B, pages).to(torch.int32).contiguous()
        s["pk"], s["pv"] = (_pool(r, B * pages, Hkv, P, D, False, False) for _ in range(2))
        s["seq_lens"], s["new_lens"] = _ints(total), _ints(lens)
        if own:
            s["pages"] = vb.Pages(s["pk"], s["pv"])
        return s
    # a pool with a few free pages, the sequences' pages in no order
    pages = -(-N // P)
    s["seq_lens"] = _ints(_lengths(case))[r.order(B)].contiguous()
    s["table_b"] = r.order(B * pages + 3)[: B * pages].reshape(B, pages).to(torch.int32).contiguous()
    s["pk"], s["pv"] = (_pool(r, B * pages + 3, Hkv, P, D, case.get("token_major"), True) for _ in range(2))
    if own:
        s["pages"] = vb.Pages(s["pk"], s["pv"])
    if kind in ("weigh", "evict"):
        # sums of many steps' weights: a few tokens have most, and many of the least are alike
        w = torch.exp(2.0 * torch.randn(B, Hkv, N, generator=r.g, device="cuda"))
        s["w"] = torch.round(w * 256) / 256
    if kind != "evict":
        s["q"] = r.normal(B, Hq, D) * 2                 # scores of a few units: some tokens stand out
        s["out"] = torch.empty(B, Hq, D, dtype=r.dtype, device="cuda")
        s["lse"] = torch.empty(B, Hq, dtype=torch.float32, device="cuda")
        s["w_out"] = torch.zeros(B, Hkv, N, device="cuda") if kind == "weigh" else None
        if own:
            s["ws"] = vb.new_paged_workspace(s["pages"], Hq, B, N, weights=kind == "weigh")
        return s
    keep = case["keep"]
    dpages = -(-keep // P)
    s["dk"], s["dv"] = (_pool(r, B * dpages, Hkv, P, D, case.get("token_major"), False) for _ in range(2))
    s["dtable"] = r.order(B * dpages).reshape(B, dpages).to(torch.int32).contiguous()
    s["dlens"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    s["dw"] = torch.zeros(B, Hkv, keep, device="cuda")
    s["kept"] = torch.zeros(B, Hkv, keep, dtype=torch.int32, device="cuda")
    if own:
        s["dst"] = vb.Pages(s["dk"], s["dv"])
        s["ws"] = vb.new_evict_workspace(s["pages"], B, N, keep)
    return s


# ---- plain forms


def _turned(x, case, freqs, positions):
    """x [B, H, T, D] turned by positions [B, T]: angles in 64 bits, the rest in 32."""
    R = case["rot"]
    angle = positions.double()[:, None, :, None] * freqs
    c, s = torch.cos(angle).float(), torch.sin(angle).float()
    if case.get("inverse"):
        s = -s
    y = x.float()
    a, b = (y[..., 0:R:2], y[..., 1:R:2]) if case.get("interleaved") else (y[..., : R // 2], y[..., R // 2: R])
    u, v = a * c - b * s, a * s + b * c
    head = torch.stack([u, v], -1).flatten(-2) if case.get("interleaved") else torch.cat([u, v], -1)
    return torch.cat([head, y[..., R:]], -1).to(x.dtype)


def _plain_rotary(s):
    c, x = s["case"], s["x"]
    pos = s["positions"]
    if pos is None:
        pos = torch.arange(x.shape[2], device=x.device).expand(x.shape[0], -1)
    return _turned(x, c, s["freqs"], pos)


def _plain_append(s):
    c, k, P = s["case"], s["k"], s["case"]["page"]
    T = k.shape[2]
    t = torch.arange(T, device=k.device)
    live = t < s["new_lens"][:, None]                                   # [B, T]
    pos = (s["seq_lens"] - s["new_lens"])[:, None] + t
    q, kk = _turned(s["q"], c, s["freqs"], pos), _turned(k, c, s["freqs"], pos)
    b, i = torch.nonzero(live, as_tuple=True)
    at = pos[b, i].long()
    page, slot = s["table_b"][b, at // P].long(), at % P
    s["pk"][page, :, slot] = kk[b, :, i]
    s["pv"][page, :, slot] = s["v"][b, :, i]
    s["q_out"].copy_(torch.where(live[:, None, :, None], q, s["q_out"]))
    return {"q": s["q_out"], "k": s["pk"], "v": s["pv"]}


def _rows(pool, table, N):
    """Rows 0 .. N-1 of every sequence, [B, Hkv, N, D] in 32 bits."""
    x = pool[table.long()]                                              # [B, pages, Hkv, P, D]
    B, n, H, P, D = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(B, H, n * P, D)[:, :, :N].float()


def _plain_attend(s):
    q, c = s["q"], s["case"]
    B, Hq, D = q.shape
    Hkv, N = c["Hkv"], c["N"]
    k = _rows(s["pk"], s["table_b"], N)
    score = torch.matmul(q.float().reshape(B, Hkv, Hq // Hkv, D), k.transpose(2, 3)) / math.sqrt(D)
    del k
    live = torch.arange(N, device=q.device) < s["seq_lens"][:, None]
    score = torch.where(live[:, None, None], score, float("-inf"))
    m = score.amax(-1, keepdim=True)
    p = torch.exp(score - m)
    den = p.sum(-1, keepdim=True)
    p = p / den
    v = _rows(s["pv"], s["table_b"], N)
    out = torch.matmul(p, v).reshape(B, Hq, D).to(q.dtype)
    r = {"out": out, "lse": (m + torch.log(den)).reshape(B, Hq)}
    if c["kind"] == "weigh":
        s["w_out"].copy_(torch.where(live[:, None], s["w"] + p.sum(2), s["w_out"]))
        r["w"] = s["w_out"]
    return r


def _plain_evict(s):
    c, w, P = s["case"], s["w"], s["case"]["page"]
    B, Hkv, N = w.shape
    keep = c["keep"]
    lens = s["seq_lens"].long()[:, None, None]
    t = torch.arange(N, device=w.device)
    always = (t < c["first"]) | (t >= lens - c["recent"])
    key = torch.where(t < lens, torch.where(always, float("inf"), w), float("-inf"))
    kept = torch.sort(key, dim=-1, descending=True, stable=True)[1][..., :keep]
    n = torch.minimum(lens, torch.full_like(lens, keep))                # [B, 1, 1]
    rank = torch.arange(kept.shape[-1], device=w.device)
    kept = torch.sort(torch.where(rank < n, kept, N), dim=-1)[0]        # in order, unused places at the end
    live = rank < n
    src = torch.where(live, kept, 0)
    b = torch.arange(B, device=w.device)[:, None, None]
    h = torch.arange(Hkv, device=w.device)[None, :, None]
    page, slot = s["table_b"][b, src // P].long(), src % P
    dpage, dslot = s["dtable"][b, rank // P].long(), rank % P
    for a, d in ((s["pk"], s["dk"]), (s["pv"], s["dv"])):
        d[dpage, h, dslot] = torch.where(live[..., None], a[page, h, slot], d[dpage, h, dslot])
    m = kept.shape[-1]                                                  # (a cache shorter than what may be kept)
    s["dw"][..., :m] = torch.where(live, torch.gather(w, 2, src), s["dw"][..., :m])
    s["kept"][..., :m] = torch.where(live, kept.int(), s["kept"][..., :m])
    s["dlens"].copy_(n[:, 0, 0])
    return {"k": s["dk"], "v": s["dv"], "w": s["dw"], "kept": s["kept"], "lens": s["dlens"]}


def run(s):
    c = s["case"]
    kind = c["kind"]
    if not own:
        return {"rotary": _plain_rotary, "append": _plain_append, "attend": _plain_attend, "weigh": _plain_attend, "evict": _plain_evict}[kind](s)
    from paper_2510_06175_amd import binding as vb
    if kind == "rotary":
        vb.vecinfer_rotary(s["rot"], s["table"], s["x"], s["out"], positions=s["positions"], inverse=c.get("inverse", 0))
        return s["out"]
    if kind == "append":
        vb.vecinfer_paged_append(s["pages"], s["k"], s["v"], s["table_b"], s["seq_lens"], new_lens=s["new_lens"], rot=s["rot"],
                                 table=s["table"], q=s["q"], q_out=s["q_out"])
        return {"q": s["q_out"], "k": s["pk"], "v": s["pv"]}
    if kind == "evict":
        vb.vecinfer_paged_evict(s["pages"], s["w"], s["table_b"], s["dst"], s["dtable"], s["dlens"], s["ws"], c["keep"],
                                first=c["first"], recent=c["recent"], seq_lens=s["seq_lens"], dst_weights=s["dw"], kept=s["kept"])
        return {"k": s["dk"], "v": s["dv"], "w": s["dw"], "kept": s["kept"], "lens": s["dlens"]}
    vb.vecinfer_paged_attention(s["pages"], s["q"], s["table_b"], s["ws"], s["out"], lse=s["lse"], seq_lens=s["seq_lens"], N=c["N"],
                                weights_in=s.get("w"), weights_out=s["w_out"])
    r = {"out": s["out"], "lse": s["lse"]}
    if kind == "weigh":
        r["w"] = s["w_out"]
    return r


# ---- the definitions in 64 bits


def _spun(x, case, positions):
    """x [.., T, D] by positions [T], as products of complex numbers."""
    R = case["rot"]
    angle = positions.double()[:, None] * torch.from_numpy(_frequencies(case)).to(x.device)
    turn = torch.polar(torch.ones_like(angle), -angle if case.get("inverse") else angle)
    y = x.double().clone()
    if case.get("interleaved"):
        z = torch.view_as_complex(y[..., :R].reshape(*y.shape[:-1], R // 2, 2).contiguous()) * turn
        y[..., :R] = torch.view_as_real(z).reshape(*y.shape[:-1], R)
    else:
        z = torch.complex(y[..., : R // 2].contiguous(), y[..., R // 2: R].contiguous()) * turn
        y[..., : R // 2], y[..., R // 2: R] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    kind, B, Hq, Hkv, D, N = (case[k] for k in ("kind", "B", "Hq", "Hkv", "D", "N"))
    if kind == "rotary":
        return torch.stack([_spun(s["x"][b], case, torch.arange(N, device="cuda") + case.get("pos0", 0)) for b in range(B)])
    P = case["page"]
    if kind == "append":
        q, k, v = s["q_out"].double(), s["pk"].double(), s["pv"].double()
        for b, (past, n) in enumerate(zip(_past(case), _lengths(case))):
            at = torch.arange(past, past + n, device="cuda")
            q[b, :, :n] = _spun(s["q"][b, :, :n], case, at)
            rows = _spun(s["k"][b, :, :n], case, at)
            page = s["table_b"][b].long()[at // P]
            k[page, :, at % P] = rows.transpose(0, 1)
            v[page, :, at % P] = s["v"][b, :, :n].double().transpose(0, 1)
        return {"q": q, "k": k, "v": v}
    lens = [int(n) for n in s["seq_lens"].tolist()]
    if kind == "evict":
        keep, first, recent = case["keep"], case["first"], case["recent"]
        w, table = s["w"].cpu().numpy(), s["table_b"].long()
        k, v, dw, kept = s["dk"].double(), s["dv"].double(), s["dw"].double(), s["kept"].clone()
        for b, n in enumerate(lens):
            tail = max(first, n - recent)
            for h in range(Hkv):
                if n <= keep:
                    ids = np.arange(n)
                else:
                    middle = np.arange(min(first, n), tail)
                    room = keep - min(first, n) - (n - tail)
                    best = middle[np.lexsort((middle, -w[b, h, middle].astype(np.float64)))[:room]]
                    ids = np.concatenate([np.arange(min(first, n)), np.sort(best), np.arange(tail, n)])
                at = torch.from_numpy(ids).cuda()
                to = torch.arange(len(ids), device="cuda")
                dp = s["dtable"][b].long()[to // P]
                k[dp, h, to % P] = s["pk"][table[b][at // P], h, at % P].double()
                v[dp, h, to % P] = s["pv"][table[b][at // P], h, at % P].double()
                dw[b, h, : len(ids)] = s["w"][b, h, at].double()
                kept[b, h, : len(ids)] = at.int()
        return {"k": k, "v": v, "w": dw, "kept": kept, "lens": torch.tensor([min(n, keep) for n in lens], dtype=torch.int32)}
    out, lse = torch.zeros(B, Hq, D, dtype=torch.float64), torch.zeros(B, Hq, dtype=torch.float64)
    w = s["w_out"].double().cpu() if kind == "weigh" else None
    G = Hq // Hkv
    for b, n in enumerate(lens):
        at = torch.arange(n, device="cuda")
        page = s["table_b"][b].long()[at // P]
        for h in range(Hkv):
            k, v = s["pk"][page, h, at % P].double(), s["pv"][page, h, at % P].double()
            score = (k @ s["q"][b, h * G: (h + 1) * G].double().t().contiguous()) / math.sqrt(D)          # [n, G]
            top = torch.logsumexp(score, 0)
            p = torch.exp(score - top)
            out[b, h * G: (h + 1) * G] = (p.t().contiguous() @ v).cpu()
            lse[b, h * G: (h + 1) * G] = top.cpu()
            if w is not None:
                w[b, h, :n] = (s["w"][b, h, :n].double() + p.sum(1)).cpu()
    r = {"out": out, "lse": lse}
    if w is not None:
        r["w"] = w
    return r


def work(case):
    kind, B, Hq, Hkv, D, N = (case[k] for k in ("kind", "B", "Hq", "Hkv", "D", "N"))
    if kind == "rotary":
        return {"bytes": 4 * B * Hq * N * D + (4 * B * N if case.get("pos0") else 0), "flops": 3 * B * Hq * N * case["rot"]}
    tokens = sum(_lengths(case))
    tables = 4 * (-(-tokens // case["page"]) + B)
    if kind == "append":
        return {"bytes": 4 * tokens * (Hq + 2 * Hkv) * D + tables + 4 * B, "flops": 3 * tokens * (Hq + Hkv) * case["rot"]}
    if kind == "evict":
        kept = sum(min(n, case["keep"]) for n in _lengths(case))
        return {"bytes": 4 * tokens * Hkv + kept * Hkv * (8 * D + 12) + tables, "flops": tokens * Hkv}
    extra = 8 * Hkv * tokens if kind == "weigh" else 0
    return {"bytes": 4 * Hkv * D * tokens + 4 * B * Hq * D + 4 * B * Hq + tables + extra, "flops": 4 * Hq * D * tokens}
