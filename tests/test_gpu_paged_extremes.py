"""Paged decode attention on the GPU where scores are very large and values infinite, against the formula in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paged_reference as ref
from paper_2510_06175_amd import binding as vb
from test_gpu_paged import Cache, attend

pytestmark = pytest.mark.gpu


def unit_scale():
    """A softmax scale that is one in the units of the scores' powers of two: scale * log2(e) = 1 in fp32."""
    x = np.float32(math.log(2))
    for s in (x, np.nextafter(x, np.float32(0)), np.nextafter(x, np.float32(1))):
        if s * np.float32(math.log2(math.e)) == 1:
            return float(s)
    raise AssertionError("no such scale")


def far_scores(j, sign, dtype, lens, N=300):
    """A cache and queries (64 channels, two query heads per KV head) whose scores are sign 2^j + step n in powers of two, n = 0 .. 3
    by the token and step the spacing of fp32 numbers there, or 1.  All products and sums of a score are exact in fp32, so the
    probabilities 2^(score - largest) are known.  Returns the cache, the queries and, per sequence, the probabilities [Hkv, n] and the
    logarithm of the sum."""
    c = Cache(len(lens), 2, 64, 16, N, dtype, seed=j)
    step = max(1.0, 2.0 ** (j - 23))
    q = torch.zeros(len(lens), 4, 64)
    q[..., 0], q[..., 1] = 2.0 ** 15, sign * step
    n = torch.randint(0, 4, c.k.shape[:3], generator=c.g)
    k = torch.zeros(c.k.shape)
    k[..., 0], k[..., 1] = sign * 2.0 ** (j - 15), n.float()
    c.k.copy_(k)
    want = []
    for b, m in enumerate(lens):
        rows, _ = ref.gather(k, c.table[b], m, 16)
        d = (rows * q[b, 0].double()).sum(-1)
        top = d.amax(-1, keepdim=True)
        e = torch.exp2(d - top)
        want.append((e / e.sum(-1, keepdim=True), (top[:, 0] + torch.log2(e.sum(-1))) * math.log(2)))
    return c, q.to(c.dtype).cuda(), want


# of the probabilities and their sums, relative: as in paged_reference.attention
def rest(n, dtype):
    return (n + 64) * 2.0 ** -23 + 2.0 ** -20 + (2.0 ** -17 if dtype == "bf16" else 2.0 ** -22)


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("j", [10, 20, 22, 23, 24, 25, 26, 27, 28, 29, 30])
@pytest.mark.parametrize("splits", [1, 3])
def test_scores_of_every_size(dtype, sign, j, splits):
    """Probabilities do not depend on how large the scores are, as long as fp32 has their differences."""
    lens = [300, 37]
    c, q, want = far_scores(j, sign, dtype, lens)
    out, lse, _ = attend(c, q, lens, splits=splits, scale=unit_scale(), check=False)
    for b, n in enumerate(lens):
        p, total = want[b]
        v, _ = ref.gather(c.v.cpu(), c.table[b], n, 16)
        for h in range(4):
            o, tol = p[h // 2] @ v[h // 2], (p[h // 2] @ v[h // 2].abs()) * rest(n, dtype)
            ref.close(out[b, h], o, tol + ref.half_step(o.abs() + tol, c.dtype), f"head {h}")
            ref.close(lse[b, h], total[h // 2], rest(n, dtype) + 2.0 ** -21 * total[h // 2].abs(), "lse")


@pytest.mark.parametrize("splits", [0, 1, 4])
def test_rows_of_a_thousand(splits):
    """Finite rows whose scores pass 2^24 at the usual scale: the tokens alike share the weight, their opposites have none."""
    c = Cache(1, 1, 128, 16, 400, "fp16")
    c.k[...] = 1100.0
    last = c.table[0, -4:].long()
    c.k[last.cuda()] = -1100.0
    q = torch.full((1, 4, 128), 1100.0, dtype=c.dtype, device="cuda")
    for sign, tokens in ((1.0, slice(0, 336)), (-1.0, slice(336, 400))):
        out, _, _ = attend(c, sign * q, splits=splits, check=False)
        v = ref.gather(c.v.cpu(), c.table[0], 400, 16)[0][0, tokens]
        tol = v.abs().mean(0) * rest(400, "fp16")
        for h in range(4):
            ref.close(out[0, h], v.mean(0), tol + ref.half_step(v.mean(0).abs() + tol, c.dtype), f"sign {sign} head {h}")


def whole_number_of(x):
    """0 finite, 1 infinity, -1 its opposite, 2 not a number."""
    return torch.where(torch.isnan(x), 2, torch.where(torch.isinf(x), torch.sign(x), 0)).int()


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,N,splits", [(1, 20, 1), (2, 500, 1), (2, 500, 3), (1, 700, 7), (1, 3000, 0), (3, 4100, 0)])
@pytest.mark.parametrize("far", [False, True])
def test_infinite_values(dtype, D, B, N, splits, far):
    """An infinity among the attended values goes into its channel of its heads' outputs, however small its weight is, as in
    the sum of the formula; two of opposite signs, or what is no number, give what is no number; other channels do not notice."""
    c = Cache(B, 2, D, 16, N, dtype, seed=N)
    lens = [N - 7 * b for b in range(B)]
    q = c.queries(6, 2.0)
    if far:                                       # (weights of 2^-400 and less for one half of the tokens, in channels of no other use)
        c.k[..., 0] = torch.where(torch.arange(16, device="cuda") % 2 == 1, -30.0, 0.0).to(c.dtype)
        q[..., 0] = 16.0
    special = {3: (float("inf"),), 5: (float("-inf"),), 7: (float("inf"), float("-inf")), 11: (float("nan"),), 13: (float("inf"), float("inf"))}
    clean = attend(c, q, lens, splits=splits, scale=1.0 if far else None)
    want = {3: 1, 5: -1, 7: 2, 11: 2, 13: 1}
    for at in (1, 9, 12, N // 2 + 1, N - 7 * B - (N - 7 * B) % 2):      # also among the last split's
        if at < 0 or at >= min(lens):
            continue
        for b in range(B):
            was = c.v.clone()
            for ch, values in special.items():
                for i, x in enumerate(values):
                    t = max(0, at - 2 * i)
                    c.v[int(c.table[b, t // 16]), 1, t % 16, ch] = x
            out, lse, _ = attend(c, q, lens, splits=splits, scale=1.0 if far else None, check=False)
            kind = torch.zeros(out.shape, dtype=torch.int32)
            for ch in special:
                kind[b, 3:, ch] = want[ch]
            assert torch.equal(whole_number_of(out.cpu()), kind), (at, b)
            assert torch.equal(lse, clean[1])
            assert torch.equal(out.cpu()[kind == 0], clean[0].cpu()[kind == 0]), (at, b)
            c.v.copy_(was)


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("j", [4, 10, 16, 22, 24, 27, 30])
@pytest.mark.parametrize("splits", [1, 3])
def test_weights_of_scores_of_every_size(dtype, sign, j, splits):
    """The weights of a head add up to one however large its scores are."""
    lens = [300, 37]
    c, q, want = far_scores(j, sign, dtype, lens)
    start = torch.rand(2, 2, 300, generator=c.g).cuda()
    for w_in in (None, start):
        w = torch.zeros(2, 2, 300, device="cuda")
        attend(c, q, lens, splits=splits, scale=unit_scale(), weights=w, w_in=w_in, check=False)
        for b, n in enumerate(lens):
            p = 2 * want[b][0]                    # two query heads alike
            total = p + (0 if w_in is None else w_in[b, :, :n].cpu().double())
            # (at 2^30 the steps are 2^7, and 2^-128 is no normal number of fp32: what lies below 2^-126 may be 0)
            ref.close(w[b, :, :n], total, p * rest(n, dtype) + 4 * 2.0 ** -23 * total + 2.0 ** -126, "weights")


@pytest.mark.parametrize("splits", [1, 4])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_holes_weigh_nothing_beside_scores_that_are_no_numbers(splits, bad):
    """A score that is no number leaves no number in the sums of the tokens that are there; a hole's stay as they were."""
    c = Cache(1, 2, 64, 16, 160)
    c.table[0, 2], c.table[0, 7] = -1, c.k.shape[0]
    c.k[int(c.table[0, 4]), 1, 5, 6] = bad
    q = c.queries(4).abs()
    start = torch.rand(1, 2, 160, generator=c.g).cuda()
    w = torch.zeros_like(start)
    attend(c, q, splits=splits, weights=w, w_in=start, check=False)
    hole = torch.zeros(160, dtype=torch.bool)
    hole[32:48] = hole[112:128] = True
    assert torch.equal(w[0, :, hole.cuda()], start[0, :, hole.cuda()])
    assert torch.isnan(w[0, 1, 69]) and torch.isfinite(w[0, 0]).all()
    if bad != bad:
        assert torch.isnan(w[0, 1, ~hole.cuda()]).all()


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("N,splits", [(150, 1), (150, 3), (4100, 0)])
@pytest.mark.parametrize("weights", [False, True])
def test_what_is_read_in_place_of_a_hole(dtype, N, splits, weights):
    """Infinities and NaN in the pages that are free, in page 0 (which is read in a hole's place) and behind the ends of sequences
    with holes change nothing."""
    c = Cache(3, 2, 128, 16, N, dtype, spare=40)
    lens = [N - 80, N - 49, 0]
    c.table[c.table == 0] = -1
    c.table[0, 1] = -1
    c.table[1, ::2] = c.k.shape[0] + 1
    c.table[1, 1] = 2 ** 31 - 1
    c.k[0], c.v[0] = 0.0, 0.0
    q = c.queries(8)

    def once(check):
        w = torch.full((3, 2, N), 0.5, device="cuda") if weights else None
        return attend(c, q, lens, splits=splits, weights=w, check=check)

    clean = once(True)
    used = set(c.table.flatten().tolist())
    free = [i for i in range(c.k.shape[0]) if i not in used]
    assert 0 in free
    for x, bad in ((c.k, float("nan")), (c.v, float("inf")), (c.v, float("nan")), (c.k, float("-inf"))):
        x[free] = bad
        for b, n in enumerate(lens):
            for col in range(c.table.shape[1]):
                page = int(c.table[b, col])
                if 0 <= page < c.k.shape[0]:
                    x[page, :, max(0, n - 16 * col):] = bad
        again = once(False)
        assert all(torch.equal(a, b) for a, b in zip(again, clean) if a is not None)
