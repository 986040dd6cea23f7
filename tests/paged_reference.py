"""Plain 64-bit forms of rotary positions, paged append, paged attention and eviction, on the CPU, and the bounds of what
fp32 arithmetic may lose against them."""
import math

import numpy as np
import torch

from paper_2510_06175_amd import binding as vb

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def half_step(y, dtype):
    """Half a step of `dtype` at the values y, half the smallest step near 0."""
    fi = torch.finfo(dtype)
    return torch.clamp(y.abs() * (fi.eps / 2), min=fi.tiny * fi.eps / 2)


def frequencies(rot):
    R, i = rot.rot_dim, np.arange(rot.rot_dim // 2, dtype=np.float64)
    base = rot.base * rot.factor ** (R / (R - 2.0)) if rot.scaling == vb.ROTARY_BASE else rot.base
    f = base ** (-2.0 * i / R)
    if rot.scaling == vb.ROTARY_LINEAR:
        return f / rot.factor
    if rot.scaling == vb.ROTARY_PARTS:
        g = np.clip((rot.orig_len * f / (2 * math.pi) - rot.low_turns) / (rot.high_turns - rot.low_turns), 0, 1)
        return g * f + (1 - g) * f / rot.factor
    return f


def rotary(rot, x, positions, inverse=0, freqs=None):
    """x [B, H, T, D], positions [B, T] -> the turned rows in 64 bits, and how far fp32 may be off them before their
    last rounding."""
    R = rot.rot_dim
    f = torch.from_numpy(frequencies(rot) if freqs is None else np.asarray(freqs, np.float64))
    a = positions.double()[:, None, :, None] * f
    c, s = torch.cos(a) * rot.magnitude, torch.sin(a) * rot.magnitude * (-1 if inverse else 1)
    x = x.double()
    one, two = (x[..., 0:R:2], x[..., 1:R:2]) if rot.interleaved else (x[..., :R // 2], x[..., R // 2:R])
    u, v, size = one * c - two * s, one * s + two * c, one.abs() + two.abs()
    join = (lambda p, q: torch.stack([p, q], -1).flatten(-2)) if rot.interleaved else (lambda p, q: torch.cat([p, q], -1))
    # angle as a 24-bit number of half turns (pi 2^-25), sine and cosine (2^-23), times the magnitude (2^-24, twice where it
    # is rounded itself), a product and a sum (2^-24 each): below 2^-21 of both parts
    loose = abs(rot.magnitude) * 2.0 ** -21 * join(size, size)
    return torch.cat([join(u, v), x[..., R:]], -1), torch.cat([loose, torch.zeros_like(x[..., R:])], -1)


def gather(pool, table, n, page_size):
    """Rows 0 .. n - 1 of one sequence, [Hkv, n, D] in 64 bits, and which of them exist."""
    t = torch.arange(n)
    page = table[t // page_size].long()
    there = (page >= 0) & (page < pool.shape[0])
    rows = pool[torch.where(there, page, 0), :, t % page_size].double().transpose(0, 1)
    return rows, there


def attention(q, k_pool, v_pool, table, lens, scale):
    """q [B, Hq, D], pools [pages, Hkv, P, D], table [B, .], lens [B] -> dict of out, lse, weights (list of [Hkv, n]) with
    their bounds (tol_*) in fp32 arithmetic, the output's without its rounding."""
    B, Hq, D = q.shape
    Hkv, P = k_pool.shape[1:3]
    G, bf16 = Hq // Hkv, q.dtype is torch.bfloat16
    out, lse = torch.zeros(B, Hq, D, dtype=torch.float64), torch.full((B, Hq), -math.inf, dtype=torch.float64)
    tol_out, tol_lse, weights, tol_w = torch.zeros_like(out), torch.zeros_like(lse), [], []
    for b, n in enumerate(lens):
        k, there = gather(k_pool, table[b], n, P)
        v, _ = gather(v_pool, table[b], n, P)
        w, tw = torch.zeros(Hkv, n, dtype=torch.float64), torch.zeros(Hkv, n, dtype=torch.float64)
        for h in range(Hq):
            g = h // G
            if not bool(there.any()):
                continue
            kk, vv, qq = k[g][there], v[g][there], q[b, h].double()
            s = (kk @ qq) * scale
            # D products summed in any order, every addition off by a whole unit, then the scale (to log2 units)
            ds = (D + 8) * 2.0 ** -23 * abs(scale) * (kk.abs() @ qq.abs()) + 2.0 ** -22 * s.abs()
            top = torch.logsumexp(s, 0)
            p = torch.exp(s - top)
            d = float(ds.max())
            # as many additions as tokens, every one off by a unit; exp2; probabilities in two parts of 8 (bf16) or 11
            # bits and their signs, 2^-17 or 2^-22
            rest = (len(s) + 64) * 2.0 ** -23 + 2.0 ** -20 + (2.0 ** -17 if bf16 else 2.0 ** -22)
            out[b, h] = p @ vv
            tol_out[b, h] = (p @ vv.abs()) * (2 * d + rest)
            lse[b, h] = top
            tol_lse[b, h] = d + rest + 2.0 ** -21 * abs(float(top))
            w[g, there] += p
            tw[g, there] += p * (2 * d + rest + 2.0 ** -21 * (s.abs() + abs(float(top)) + 1))
        weights.append(w)
        tol_w.append(tw)
    return {"out": out, "lse": lse, "weights": weights, "tol_out": tol_out, "tol_lse": tol_lse, "tol_w": tol_w}


def evict(w, table, num_pages, page_size, n, keep, first, recent):
    """w [Hkv, n] -> the kept indices of every KV head, in order."""
    t = np.arange(n)
    page = table[:(n + page_size - 1) // page_size].numpy()[t // page_size] if n else t
    there = (page >= 0) & (page < num_pages)
    kept = []
    for row in w.double().numpy():
        row = np.where(np.isnan(row), -np.inf, row)
        nan = np.isnan(w.double().numpy()[len(kept)])
        always = (t < first) | (t >= n - recent)
        # always kept, then by weight, what is no number behind -inf, then by index
        order = sorted(t[there], key=lambda i: (not always[i], 0 if always[i] else bool(nan[i]), 0 if always[i] else -row[i], i))
        kept.append(np.sort(np.array(order[:keep], dtype=np.int64)))
    return kept


def close(got, ref, tol, what=""):
    """got within tol of ref, infinities equal."""
    got, ref, tol = got.double().cpu(), ref.double(), tol.double()
    same = got == ref
    bad = ~(same | ((got - ref).abs() <= tol))
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} off, the worst by "
                                 f"{float(((got - ref).abs() / tol)[bad].max()):.3g} of what is allowed, first at {bad.nonzero()[0].tolist()}")
