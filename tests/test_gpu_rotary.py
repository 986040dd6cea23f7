"""Rotary positions on the GPU against the formula in 64 bits."""
import numpy as np
import pytest
import torch

import paged_reference as ref
from paper_2510_06175_amd import binding as vb

pytestmark = pytest.mark.gpu
SCALINGS = {"plain": {}, "linear": dict(scaling=vb.ROTARY_LINEAR, factor=4.0), "base": dict(scaling=vb.ROTARY_BASE, factor=8.0),
            "parts": dict(scaling=vb.ROTARY_PARTS, factor=8.0, orig_len=8192, low_turns=1.0, high_turns=4.0, magnitude=1.2)}


def rows(g, B, H, T, D, dtype, how="tokens"):
    if how == "tokens":                          # tokens, then heads, as a projection leaves them
        return torch.randn(B, T, H, D, generator=g).to(dtype).transpose(1, 2)
    if how == "part":                            # part of a larger tensor
        return torch.randn(B, H + 2, T + 1, D + 8, generator=g).to(dtype)[:, 1:-1, :-1, :D]
    return torch.randn(B, H, T, D, generator=g).to(dtype)


def check(rot, x, positions, inverse=0, out=None, pos0=0, freqs=None, explicit=True):
    xg = x.cuda() if x.is_contiguous() else torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda").copy_(x)
    fr = None if freqs is None else torch.from_numpy(freqs).cuda()
    table = vb.new_rotary_table(rot, fr)
    out = torch.empty(x.shape, dtype=x.dtype, device="cuda") if out is None else out(xg)
    vb.vecinfer_rotary(rot, table, xg, out, positions=positions.to(torch.int32).cuda() if explicit else None, pos0=pos0, inverse=inverse)
    want, loose = ref.rotary(rot, x, positions, inverse, freqs)
    # (a value that the loose arithmetic carries over a power of two has steps twice as wide: 2^-21 of it, below the 1 %)
    ref.close(out, want, 1.01 * loose + ref.half_step(want.abs() + loose, x.dtype), f"{rot} inverse {inverse}")
    return out


@pytest.mark.parametrize("dtype", ref.DTYPES)
@pytest.mark.parametrize("D,R", [(128, 128), (128, 64), (128, 48), (128, 16), (64, 64), (64, 16)])
@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("scaling", SCALINGS)
def test_rows(dtype, D, R, interleaved, scaling):
    g = torch.Generator().manual_seed(R + D)
    rot = vb.Rotary(D, R, interleaved, base=500000.0, **SCALINGS[scaling])
    positions = torch.randint(0, 20000, (2, 7), generator=g)
    for inverse in (0, 1):
        check(rot, rows(g, 2, 5, 7, D, ref.DTYPES[dtype]), positions, inverse)


@pytest.mark.parametrize("B,H,T", [(1, 1, 1), (1, 32, 1), (3, 1, 1), (1, 71, 2), (2, 8, 513), (5, 3, 1029), (1, 40, 1500)])
@pytest.mark.parametrize("D", [64, 128])
def test_sizes(B, H, T, D):
    g = torch.Generator().manual_seed(T)
    rot = vb.Rotary(D, D)
    check(rot, rows(g, B, H, T, D, torch.bfloat16), torch.arange(T).expand(B, T) + 11, explicit=False, pos0=11)


@pytest.mark.parametrize("B,H,T,D,R,interleaved", [(1, 40, 3503, 128, 128, 0), (2, 33, 2103, 128, 80, 1), (3, 5, 9191, 128, 48, 0), (1, 64, 4500, 64, 64, 1)])
def test_more_than_the_caches_hold(B, H, T, D, R, interleaved):
    g = torch.Generator().manual_seed(T)
    check(vb.Rotary(D, R, interleaved, base=500000.0), rows(g, B, H, T, D, torch.float16), torch.randint(0, 9000, (B, T), generator=g), inverse=1)


@pytest.mark.parametrize("how", ["tokens", "part", "plain"])
@pytest.mark.parametrize("inverse", [0, 1])
def test_strides_and_in_place(how, inverse):
    g = torch.Generator().manual_seed(5)
    rot = vb.Rotary(128, 96, interleaved=inverse)
    x = rows(g, 2, 6, 33, 128, torch.float16, how)
    positions = torch.randint(0, 5000, (2, 33), generator=g)
    check(rot, x, positions, inverse)
    check(rot, x, positions, inverse, out=lambda xg: xg)
    check(rot, x, positions, inverse, out=lambda xg: torch.empty(2, 33, 6, 128, dtype=x.dtype, device="cuda").transpose(1, 2))


@pytest.mark.parametrize("pos0", [10 ** 6 + 7, 2 ** 31 - 4, -5, 2 ** 40 + 1])
def test_far_and_negative_positions(pos0):
    """Angles are exact at any distance.  (From 2^30 on the reference's own product in 64 bits is not: there the frequencies
    are powers of two of a turn, so that the position counts modulo 2^16.)"""
    g = torch.Generator().manual_seed(1)
    rot = vb.Rotary(64, 64)
    x = rows(g, 1, 4, 3, 64, torch.float16)
    if abs(pos0) < 2 ** 30:
        positions = torch.arange(3)[None] + pos0
        check(rot, x, positions, explicit=False, pos0=pos0)
        check(rot, x, positions)
    else:
        freqs = 2 * np.pi * 2.0 ** -(1.0 + np.arange(32) % 16)
        check(rot, x, (torch.arange(3) + pos0)[None] % 2 ** 16, freqs=freqs, explicit=False, pos0=pos0)


def test_table():
    """The formula within 2^-50 of it, cut to whole units of 2^-64 (which is 2^-42 of the smallest frequency here, 2^-22
    turns), and a table of given frequencies."""
    for how in SCALINGS.values():
        for D, R in ((128, 128), (64, 16)):
            rot = vb.Rotary(D, R, base=500000.0, **how)
            turns = vb.new_rotary_table(rot).cpu().numpy().view(np.uint64) / 2.0 ** 64
            want = ref.frequencies(rot) / (2 * np.pi)
            assert (np.abs(turns - want) <= 2.0 ** -64 + 2.0 ** -50 * want).all()
    freqs = np.array([0.0, 1.0, -1.0, 2 * np.pi * 1.25, -2 * np.pi * 0.25, np.inf, np.nan, 1e-18])
    freqs = torch.from_numpy(np.concatenate([freqs, freqs[::-1]]).copy())
    got = vb.new_rotary_table(vb.Rotary(64, 32), freqs.cuda()).cpu().numpy().view(np.uint64) / 2.0 ** 64
    want = [0, 1 / (2 * np.pi), 1 - 1 / (2 * np.pi), 0.25, 0.75, 0, 0, 1e-18 / (2 * np.pi)]
    assert np.allclose(got, want + want[::-1], rtol=1e-14, atol=2.0 ** -64)


@pytest.mark.parametrize("interleaved", [0, 1])
def test_gradient(interleaved):
    """The rotation is linear, so a difference along a channel is a column of it whatever the step: row j of the inverse's
    output for a gradient e_i is column j's entry i."""
    rot = vb.Rotary(64, 32, interleaved, base=100.0, magnitude=1.5)
    table = vb.new_rotary_table(rot)
    D, pos = 64, torch.tensor([[0], [3], [777]], dtype=torch.int32, device="cuda")
    eye = torch.eye(D, dtype=torch.float16, device="cuda").expand(3, D, D).reshape(3, D, 1, D).contiguous()
    base = torch.randn(3, 1, 1, D, device="cuda").half().expand(3, D, 1, D)
    out = lambda x, inverse=0: (lambda y: vb.vecinfer_rotary(rot, table, x, y, positions=pos, inverse=inverse) or y)(torch.empty_like(x))  # noqa: E731
    step = 4.0
    plus, minus = out((base + step * eye).contiguous()), out((base - step * eye).contiguous())
    x = (base + step * eye).double() - (base - step * eye).double()              # (as rounded)
    columns = (plus.double() - minus.double())[:, :, 0] / x[:, :, 0].amax(-1, keepdim=True)
    back = out(eye, 1)[:, :, 0].double()                                         # [.., i, j] = d out_i / d x_j
    # each of the two outputs, below 16, is off by 2^-11 of itself, their difference is divided by 8; the gradient by 2^-11
    assert ((columns.transpose(1, 2) - back).abs() <= 2 * 16 * 2.0 ** -11 / 8 + 2 * 2.0 ** -11).all()


def test_stream_and_graph():
    rot = vb.Rotary(128, 128)
    table = vb.new_rotary_table(rot)
    x, out = torch.randn(2, 4, 9, 128, device="cuda").half(), torch.empty(2, 4, 9, 128, dtype=torch.float16, device="cuda")
    vb.vecinfer_rotary(rot, table, x, out, pos0=3)
    torch.cuda.synchronize()
    want = out.clone()
    side = torch.cuda.Stream()
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    vb.vecinfer_rotary(rot, table, x, out, pos0=3, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vb.vecinfer_rotary(rot, table, x, out, pos0=3)
    for i in range(3):
        x.copy_(torch.randn(2, 4, 9, 128, device="cuda"))
        eager = torch.empty_like(out)
        vb.vecinfer_rotary(rot, table, x, eager, pos0=3)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)


def test_rows_refused():
    rot = vb.Rotary(64, 64)
    table = vb.new_rotary_table(rot)
    x = torch.zeros(2, 4, 8, 64, dtype=torch.float16, device="cuda")
    with pytest.raises(ValueError):
        vb.vecinfer_rotary(rot, table, x, x.float())
    with pytest.raises(ValueError):
        vb.vecinfer_rotary(rot, table, x, x[:, :, :7])
    with pytest.raises(ValueError):
        vb.vecinfer_rotary(rot, table[:16], x, x)
    with pytest.raises(ValueError):
        vb.vecinfer_rotary(rot, table, x, x[:1].expand(2, 4, 8, 64))
    with pytest.raises(ValueError):
        vb.vecinfer_rotary(rot, table, x, x, positions=torch.zeros(2, 8, dtype=torch.int64, device="cuda"))
    wide = torch.zeros(2, 4, 8, 68, dtype=torch.float16, device="cuda")
    for bad in (wide[..., :64], wide[..., 4:]):             # rows that start between 16-byte pieces
        with pytest.raises(vb.VecInferError) as e:
            vb.vecinfer_rotary(rot, table, bad, x)
        assert e.value.code == vb.EINVAL
    with pytest.raises(vb.VecInferError):
        vb.vecinfer_rotary(rot, table, x[:, :, :0], x[:, :, :0])
