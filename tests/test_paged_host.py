"""Refusals of the rotary and paged entry points: bad arguments are rejected with error codes before anything is launched
(no GPU needed), and the sizes that the host works out."""
import ctypes as C

import pytest
import torch

from paper_2510_06175_amd import binding as vb

FAKE = 0x10000          # non-null, 256-byte aligned; never dereferenced on the host
S3 = C.c_int64 * 3
EINVAL, EUNSUP, EWORK = vb.EINVAL, vb.EUNSUPPORTED, vb.EWORKSPACE


def rot(**change):
    d = dict(head_dim=128, rot_dim=128, interleaved=0, scaling=0, base=1e4, factor=1.0, low_turns=1.0, high_turns=4.0, orig_len=8192,
             magnitude=1.0)
    d.update(change)
    return vb._RotaryCfg(**d)


def pages(**change):
    d = dict(k=FAKE, v=FAKE, dtype=0, head_dim=128, num_kv_heads=8, page_size=16, num_pages=100,
             k_strides=S3(16 * 8 * 128, 16 * 128, 128), v_strides=S3(16 * 8 * 128, 16 * 128, 128))
    d.update(change)
    return vb._Pages(**d)


BAD_ROTARY = [(dict(head_dim=96), EUNSUP), (dict(rot_dim=0), EUNSUP), (dict(rot_dim=24), EUNSUP), (dict(rot_dim=144), EUNSUP),
              (dict(head_dim=64), EUNSUP), (dict(interleaved=2), EINVAL), (dict(scaling=4), EINVAL), (dict(scaling=-1), EINVAL),
              (dict(base=0.0), EINVAL), (dict(base=float("nan")), EINVAL), (dict(base=float("inf")), EINVAL),
              (dict(magnitude=float("nan")), EINVAL), (dict(magnitude=1e39), EINVAL), (dict(scaling=1, factor=0.0), EINVAL), (dict(scaling=2, factor=float("inf")), EINVAL),
              (dict(scaling=3, factor=2.0, low_turns=4.0), EINVAL), (dict(scaling=3, factor=2.0, orig_len=0), EINVAL),
              (dict(scaling=3, factor=2.0, high_turns=float("inf")), EINVAL)]
BAD_PAGES = [(dict(k=None), EINVAL), (dict(v=FAKE + 8), EINVAL), (dict(dtype=2), EINVAL), (dict(head_dim=96), EUNSUP),
             (dict(num_kv_heads=0), EINVAL), (dict(num_kv_heads=70000), EUNSUP), (dict(page_size=0), EINVAL), (dict(page_size=4), EUNSUP),
             (dict(page_size=24), EUNSUP), (dict(page_size=2048), EUNSUP), (dict(num_pages=0), EINVAL), (dict(num_pages=1 << 31), EUNSUP),
             (dict(k_strides=S3(128, 128, 4)), EINVAL), (dict(v_strides=S3(128, -128, 128)), EINVAL),
             (dict(k_strides=S3(1 << 30, 128, 128)), EINVAL)]


@pytest.mark.parametrize("change,code", BAD_ROTARY)
def test_table_refuses(change, code):
    assert vb.lib().vecinfer_rotary_table(C.byref(rot(**change)), None, FAKE, None) == code


def test_table_refuses_pointers():
    f = vb.lib().vecinfer_rotary_table
    assert f(None, None, FAKE, None) == EINVAL
    assert f(C.byref(rot()), None, None, None) == EINVAL
    assert f(C.byref(rot()), None, FAKE + 4, None) == EINVAL
    assert f(C.byref(rot()), FAKE + 4, FAKE, None) == EINVAL


def call_rotary(**change):
    a = dict(cfg=rot(), table=FAKE, dtype=0, x=FAKE, xs=S3(8 * 4 * 128, 4 * 128, 128), out=FAKE, os=S3(8 * 4 * 128, 4 * 128, 128), B=2, H=8,
             T=4, positions=None, pos0=0, inverse=0)
    a.update(change)
    cfg = a.pop("cfg")
    return vb.lib().vecinfer_rotary(None if cfg is None else C.byref(cfg), *a.values(), None)


@pytest.mark.parametrize("change,code", [
    (dict(cfg=None), EINVAL), (dict(table=None), EINVAL), (dict(x=None), EINVAL), (dict(out=None), EINVAL), (dict(xs=None), EINVAL),
    (dict(os=None), EINVAL), (dict(dtype=2), EINVAL), (dict(dtype=-1), EINVAL), (dict(B=0), EINVAL), (dict(H=0), EINVAL), (dict(T=0), EINVAL),
    (dict(T=-1), EINVAL), (dict(x=FAKE + 2), EINVAL), (dict(out=FAKE + 8), EINVAL), (dict(positions=FAKE + 2), EINVAL),
    (dict(xs=S3(0, 0, 7)), EINVAL), (dict(xs=S3(0, -8, 8)), EINVAL), (dict(os=S3(0, 1 << 41, 8)), EINVAL), (dict(T=1 << 30), EUNSUP), (dict(H=65536), EUNSUP)])
def test_rotary_refuses(change, code):
    assert call_rotary(**change) == code


@pytest.mark.parametrize("change,code", BAD_ROTARY)
def test_rotary_refuses_cfg(change, code):
    assert call_rotary(cfg=rot(**change)) == code


def call_append(**change):
    s = S3(8 * 128, 128, 8 * 128)
    a = dict(pages=pages(), rot=rot(), table=FAKE, k=FAKE, ks=s, v=FAKE, vs=s, q=FAKE, qs=s, qo=FAKE, qos=s, Hq=32, bt=FAKE, mp=10, lens=FAKE,
             new=None, pos=None, B=2, T=4, w=None, w_cap=0)
    a.update(change)
    ref = lambda x: None if x is None else C.byref(x)  # noqa: E731
    a["pages"], a["rot"] = ref(a["pages"]), ref(a["rot"])
    return vb.lib().vecinfer_paged_append(*a.values(), None)


@pytest.mark.parametrize("change,code", [
    (dict(pages=None), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(ks=None), EINVAL), (dict(vs=None), EINVAL),
    (dict(bt=None), EINVAL), (dict(lens=None), EINVAL), (dict(rot=None), EINVAL), (dict(table=None), EINVAL),
    (dict(rot=None, table=None), EINVAL), (dict(q=None), EINVAL), (dict(qo=None), EINVAL), (dict(qs=None), EINVAL), (dict(qos=None), EINVAL),
    (dict(Hq=0), EINVAL), (dict(rot=rot(head_dim=64, rot_dim=64)), EINVAL), (dict(B=0), EINVAL), (dict(T=0), EINVAL), (dict(mp=0), EINVAL),
    (dict(w=FAKE), EINVAL), (dict(w=FAKE + 2, w_cap=4), EINVAL), (dict(k=FAKE + 4), EINVAL), (dict(bt=FAKE + 1), EINVAL),
    (dict(lens=FAKE + 2), EINVAL), (dict(new=FAKE + 1), EINVAL), (dict(pos=FAKE + 3), EINVAL), (dict(ks=S3(8, 8, 12)), EINVAL),
    (dict(vs=S3(-8, 8, 8)), EINVAL), (dict(qs=S3(8, 8, 12)), EINVAL), (dict(T=1 << 30), EUNSUP), (dict(Hq=70000), EUNSUP)])
def test_append_refuses(change, code):
    assert call_append(**change) == code


@pytest.mark.parametrize("change,code", BAD_PAGES)
def test_append_refuses_pages(change, code):
    assert call_append(pages=pages(**change)) == code


def call_attention(**change):
    a = dict(pages=pages(), q=FAKE, qs=(C.c_int64 * 2)(32 * 128, 128), Hq=32, bt=FAKE, mp=10, lens=None, B=2, N=150, scale=0.1, S=0, ws=FAKE,
             wb=1 << 30, out=FAKE, lse=None, wi=None, wo=None, w_cap=0)
    a.update(change)
    a["pages"] = None if a["pages"] is None else C.byref(a["pages"])
    return vb.lib().vecinfer_paged_attention(*a.values(), None)


@pytest.mark.parametrize("change,code", [
    (dict(pages=None), EINVAL), (dict(q=None), EINVAL), (dict(qs=None), EINVAL), (dict(bt=None), EINVAL), (dict(out=None), EINVAL),
    (dict(Hq=0), EINVAL), (dict(Hq=12), EINVAL), (dict(Hq=8 * 17), EUNSUP), (dict(B=0), EINVAL), (dict(B=70000), EUNSUP), (dict(N=0), EINVAL),
    (dict(N=161), EINVAL), (dict(mp=0), EINVAL), (dict(S=-1), EINVAL), (dict(S=257), EINVAL), (dict(scale=float("nan")), EINVAL),
    (dict(scale=float("inf")), EINVAL), (dict(scale=3e38), EINVAL), (dict(q=FAKE + 8), EINVAL), (dict(out=FAKE + 2), EINVAL), (dict(qs=(C.c_int64 * 2)(8, 4)), EINVAL),
    (dict(bt=FAKE + 2), EINVAL), (dict(lens=FAKE + 2), EINVAL), (dict(lse=FAKE + 2), EINVAL), (dict(wi=FAKE, w_cap=200), EINVAL),
    (dict(wo=FAKE, w_cap=149), EINVAL), (dict(wo=FAKE + 1, w_cap=200), EINVAL), (dict(ws=None), EWORK), (dict(ws=FAKE + 16), EWORK),
    (dict(wb=0), EWORK), (dict(S=4, wb=1 << 10), EWORK), (dict(N=(1 << 30) + 1, mp=1 << 30), EUNSUP), (dict(mp=1 << 31), EUNSUP)])
def test_attention_refuses(change, code):
    assert call_attention(**change) == code


@pytest.mark.parametrize("change,code", BAD_PAGES)
def test_attention_refuses_pages(change, code):
    assert call_attention(pages=pages(**change)) == code


def call_evict(**change):
    a = dict(src=pages(), w=FAKE, w_cap=160, bt=FAKE, mp=10, lens=None, B=2, N=150, keep=40, first=4, recent=8, dst=pages(k=FAKE + 256),
             dt=FAKE, dmp=3, dl=FAKE + 256, dw=None, dwc=0, kept=None, ws=FAKE, wb=1 << 20)
    a.update(change)
    for n in ("src", "dst"):
        a[n] = None if a[n] is None else C.byref(a[n])
    return vb.lib().vecinfer_paged_evict(*a.values(), None)


@pytest.mark.parametrize("change,code", [
    (dict(src=None), EINVAL), (dict(dst=None), EINVAL), (dict(w=None), EINVAL), (dict(bt=None), EINVAL), (dict(dt=None), EINVAL),
    (dict(dl=None), EINVAL), (dict(dst=pages(dtype=1)), EINVAL), (dict(dst=pages(head_dim=64)), EINVAL),
    (dict(dst=pages(num_kv_heads=4)), EINVAL), (dict(B=0), EINVAL), (dict(N=0), EINVAL), (dict(N=161, w_cap=200), EINVAL),
    (dict(w_cap=149), EINVAL), (dict(keep=0), EINVAL), (dict(keep=49), EINVAL), (dict(first=-1), EINVAL), (dict(recent=-1), EINVAL),
    (dict(first=33), EINVAL), (dict(first=41, recent=0), EINVAL), (dict(recent=1 << 62), EINVAL), (dict(lens=FAKE + 256), EINVAL),
    (dict(dw=FAKE, dwc=40), EINVAL), (dict(dw=FAKE + 4, dwc=39), EINVAL), (dict(kept=FAKE + 2), EINVAL), (dict(dl=FAKE + 2), EINVAL),
    (dict(ws=None), EWORK), (dict(ws=FAKE + 64), EWORK), (dict(wb=2559), EWORK), (dict(B=70000, wb=1 << 40), EUNSUP),
    (dict(N=(1 << 30) + 1, mp=1 << 40, w_cap=1 << 40), EUNSUP)])
def test_evict_refuses(change, code):
    assert call_evict(**change) == code


@pytest.mark.parametrize("change,code", BAD_PAGES)
def test_evict_refuses_pages(change, code):
    assert call_evict(src=pages(**change)) == code
    assert call_evict(dst=pages(**change)) == code


def test_workspace_sizes():
    L = vb.lib()
    p = pages()
    size = lambda *a: L.vecinfer_paged_workspace_bytes(C.byref(p), *a)  # noqa: E731
    assert size(32, 2, 150, 0, 0) > 0
    assert size(32, 2, 150, 4, 0) >= 2 * 32 * 4 * (128 + 2) * 4
    assert size(32, 2, 150, 4, 1) >= size(32, 2, 150, 4, 0) + 2 * 32 * 150 * 4
    for bad in ((0, 2, 150, 0, 0), (12, 2, 150, 0, 0), (32, 0, 150, 0, 0), (32, 2, 0, 0, 0), (32, 2, 150, 257, 0), (32, 2, 150, -1, 0),
                (32, 2, (1 << 30) + 1, 0, 0)):
        assert size(*bad) == 0
    for change, _ in BAD_PAGES:
        assert L.vecinfer_paged_workspace_bytes(C.byref(pages(**change)), 32, 2, 150, 0, 0) == 0
    e = L.vecinfer_evict_workspace_bytes
    assert e(8, 2, 150, 40) >= 8 * 2 * 40 * 4 and e(8, 2, 30, 40) >= 8 * 2 * 30 * 4
    assert e(0, 2, 150, 40) == e(8, 0, 150, 40) == e(8, 2, 0, 40) == e(8, 2, 150, 0) == 0


def test_a_workspace_of_more_sequences_serves_fewer():
    """Automatic splits take what there is room for: the size for one split is enough."""
    L, p = vb.lib(), pages()
    for B in (1, 2, 3, 8, 40):
        assert L.vecinfer_paged_workspace_bytes(C.byref(p), 32, B, 100000, 1, 0) <= L.vecinfer_paged_workspace_bytes(C.byref(p), 32, B, 100000, 0, 0)


def test_binding_refuses_host_tensors():
    x = torch.zeros(2, 2, 16, 64, dtype=torch.float16)
    with pytest.raises(TypeError):
        vb.Pages(x, x)
    with pytest.raises(TypeError):
        vb.vecinfer_rotary(vb.Rotary(64, 64), torch.zeros(32, dtype=torch.int64), x, x)
    with pytest.raises(ValueError):
        vb.vecinfer_rotary(vb.Rotary(64, 64), torch.zeros(32, dtype=torch.int64), x.float(), x)
    with pytest.raises(TypeError):
        vb.vecinfer_paged_attention(x, x[0], None, None, None)


def test_steps_of_odd_tensors():
    x = torch.zeros(3, 2, 16, 64)
    assert list(vb._steps(x.transpose(1, 2), "x", True)) == [2048, 64, 1024]
    assert list(vb._steps(x[:1, :, :1], "x", True)) == [0, 1024, 0]           # an axis of one index has no stride
    assert list(vb._steps(x[:1].expand(3, 2, 16, 64), "x", False)) == [0, 1024, 64]
    with pytest.raises(ValueError):
        vb._steps(x[:1].expand(3, 2, 16, 64), "x", True)
    with pytest.raises(ValueError):
        vb._steps(x.transpose(2, 3), "x", False)


def test_an_eviction_workspace_serves_fewer():
    """The size grows with the batch, the tokens and what is kept, across the length from which a row is shared by workgroups."""
    size = vb.lib().vecinfer_evict_workspace_bytes
    for Hkv in (1, 8, 24):
        for N in (32767, 32768, 32769, 40000, 65536, 100003, 131072, 1 << 20, 1 << 22):
            sizes = [size(Hkv, B, N, 2048) for B in range(1, 80)]
            assert sizes == sorted(sizes)
    for B in (1, 3, 4, 7, 32, 33, 64):
        for keep in (1, 2048, 50000):
            sizes = [size(8, B, N, keep) for N in (1, 2000, 32768, 32769, 36865, 40000, 49152, 49153, 100000, 262144, 262145, 1 << 20, 1 << 21)]
            assert sizes == sorted(sizes)
    for N in (1000, 40000):
        sizes = [size(8, 3, N, keep) for keep in (1, 100, 999, 1000, 1001, 39999, 40000, 40001)]
        assert sizes == sorted(sizes)


@pytest.mark.parametrize("weights", [0, 1])
def test_an_attention_workspace_serves_smaller_batches(weights):
    """What one made for a batch has to hold for fewer and shorter sequences is their size for one split, to which an automatic call
    goes down."""
    L, p = vb.lib(), pages()
    shapes = [(B, N) for B in (1, 2, 3, 5, 8, 33, 64, 65) for N in (1, 31, 33, 256, 257, 3999, 4000, 100000)]
    size = {(B, N, s): L.vecinfer_paged_workspace_bytes(C.byref(p), 32, B, N, s, weights) for B, N in shapes for s in (0, 1)}
    for B, N in shapes:
        for b, n in shapes:
            if b <= B and n <= N:
                assert 0 < size[b, n, 1] <= size[B, N, 0]
