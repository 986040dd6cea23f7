"""Binding of ``libvecinfer.so``: same names as the C ABI, argument marshalling only, by ctypes and, for the calls
of a decode step and the cache fill, by a native module that makes the same checks in less time (``csrc/fastcall.cpp``).

Tensors are torch CUDA (HIP) tensors used purely as device buffers; shapes, dtypes,
contiguity and device are checked here and the raw pointers handed to the library,
which enqueues on torch's current stream unless ``stream`` is given.  If the library
has not been built the import of it fails loudly: there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvecinfer.so")

VARIANT_AUTO, VARIANT_LUT, VARIANT_MFMA, VARIANT_ROLES = 0, 1, 2, 3
MAX_SPLITS = 256
MAX_RESIDUAL = 128
OK, EINVAL, EUNSUPPORTED, EWORKSPACE, ELAUNCH = 0, -1, -2, -3, -4

EXPORTS = [
    "vecinfer_encode_keys", "vecinfer_encode_values", "vecinfer_append_kv", "vecinfer_decode_auto_splits",
    "vecinfer_decode_workspace_bytes",
    "vecinfer_decode_attention", "vecinfer_decode_attention_residual", "vecinfer_decode_step",
    "vecinfer_decode_attention_static",
    "vecinfer_kmeans_workspace_bytes", "vecinfer_kmeans_step", "vecinfer_kmeans_train",
    "vecinfer_index_row_bytes", "vecinfer_codebook_elems", "vecinfer_calibrate_lambda", "vecinfer_read_probe",
    "vecinfer_export_value_codes",
    "vecinfer_rotary_table", "vecinfer_rotary", "vecinfer_paged_append", "vecinfer_paged_workspace_bytes",
    "vecinfer_paged_attention", "vecinfer_evict_workspace_bytes", "vecinfer_paged_evict",
    "vecinfer_strerror", "vecinfer_version",
]


class _Cfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("head_dim", "num_q_heads", "num_kv_heads", "k_sub_dim",
                                         "v_sub_dim", "k_bits", "v_bits", "v_tiled")]


class _once:
    """A value worked out when it is first asked for and then kept in the object's own dictionary, which
    from then on answers by itself.  (functools.cached_property takes a lock for it; here two threads may
    both work it out, and the one that is kept first is everybody's: `_p` is the address of `_c`.)"""

    def __init__(self, f):
        self.f = f

    def __set_name__(self, owner, name):
        self.name = name

    def __get__(self, obj, owner=None):
        if obj is None:
            return self
        return obj.__dict__.setdefault(self.name, self.f(obj))


@dataclass(frozen=True)
class Config:
    """Mirror of ``vecinfer_cfg``."""
    head_dim: int
    num_q_heads: int
    num_kv_heads: int
    k_sub_dim: int
    v_sub_dim: int
    k_bits: int = 8
    v_bits: int = 8
    v_tiled: int = 0            # 1: value codes stored in tiles of 64 tokens (8-bit value codes)

    def c(self) -> _Cfg:
        return _Cfg(self.head_dim, self.num_q_heads, self.num_kv_heads, self.k_sub_dim,
                    self.v_sub_dim, self.k_bits, self.v_bits, self.v_tiled)

    # What every call needs of a configuration, worked out once per (immutable) object.
    @_once
    def _c(self) -> _Cfg:
        return self.c()

    @_once
    def _p(self) -> int:
        return C.addressof(self._c)

    @_once
    def _lam_shape(self) -> tuple:
        return (self.num_kv_heads, self.head_dim)

    @_once
    def _cb_k(self) -> tuple:
        return self.cb_shape(True)

    @_once
    def _cb_v(self) -> tuple:
        return self.cb_shape(False)

    @_once
    def _row_k(self) -> int:
        return self.row_bytes(True)

    @_once
    def _row_v(self) -> int:
        return self.row_bytes(False)

    def __getstate__(self):                 # (pickles and copies carry the fields alone)
        return {f: self.__dict__[f] for f in self.__dataclass_fields__}

    def cb_shape(self, keys: bool) -> tuple:
        """Codebook tensor shape: one 256-entry table per (KV head, sub-space) for 8-bit codes, one
        table of 2^bits entries per KV head for wider ones."""
        d, bits = (self.k_sub_dim, self.k_bits) if keys else (self.v_sub_dim, self.v_bits)
        if bits == 8:
            return (self.num_kv_heads, self.head_dim // d, 256, d)
        return (self.num_kv_heads, 1 << bits, d)

    def row_bytes(self, keys: bool) -> int:
        """Bytes of one token's code row: M codes of `bits` bits, end to end."""
        d, bits = (self.k_sub_dim, self.k_bits) if keys else (self.v_sub_dim, self.v_bits)
        return self.head_dim // d * bits // 8


ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_BASE, ROTARY_PARTS = 0, 1, 2, 3
_TYPES = {torch.float16: 0, torch.bfloat16: 1}


class _RotaryCfg(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("head_dim", "rot_dim", "interleaved", "scaling")] +
                [(n, C.c_double) for n in ("base", "factor", "low_turns", "high_turns")] +
                [("orig_len", C.c_int64), ("magnitude", C.c_double)])


class _Pages(C.Structure):
    _fields_ = ([("k", C.c_void_p), ("v", C.c_void_p)] +
                [(n, C.c_int32) for n in ("dtype", "head_dim", "num_kv_heads", "page_size")] +
                [("num_pages", C.c_int64), ("k_strides", C.c_int64 * 3), ("v_strides", C.c_int64 * 3)])


@dataclass(frozen=True)
class Rotary:
    """Mirror of ``vecinfer_rotary_cfg``."""
    head_dim: int
    rot_dim: int
    interleaved: int = 0        # 0: pairs (i, i + R / 2), 1: pairs (2 i, 2 i + 1)
    base: float = 10000.0
    scaling: int = ROTARY_PLAIN
    factor: float = 1.0
    orig_len: int = 0
    low_turns: float = 1.0
    high_turns: float = 32.0
    magnitude: float = 1.0

    @_once
    def _c(self) -> _RotaryCfg:
        return _RotaryCfg(self.head_dim, self.rot_dim, self.interleaved, self.scaling, self.base, self.factor, self.low_turns,
                          self.high_turns, self.orig_len, self.magnitude)

    @_once
    def _p(self) -> int:
        return C.addressof(self._c)

    def __getstate__(self):
        return {f: self.__dict__[f] for f in self.__dataclass_fields__}


class Pages:
    """A pool of pages for the paged calls: keys and values [num_pages, H_kv, page_size, D], fp16 or bf16 of any strides
    with adjacent channels (``pool.transpose(1, 2)`` of a [num_pages, page_size, H_kv, D] tensor, say)."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        if not isinstance(k, torch.Tensor) or not isinstance(v, torch.Tensor) or not k.is_cuda or not v.is_cuda:
            raise TypeError("pages: expected tensors on the GPU")
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.dtype not in _TYPES or k.device != v.device:
            raise ValueError("pages: expected two fp16 or bf16 tensors [num_pages, H_kv, page_size, D] of one shape on one device")
        self.k, self.v = k, v
        self.num_pages, self.num_kv_heads, self.page_size, self.head_dim = k.shape
        self._c = _Pages(k.data_ptr(), v.data_ptr(), _TYPES[k.dtype], self.head_dim, self.num_kv_heads, self.page_size,
                         self.num_pages, _steps(k, "k", True), _steps(v, "v", True))
        self._p, self._dev = C.addressof(self._c), k.device.index


def _steps(t: torch.Tensor, name: str, written: bool):
    """Strides of all axes but the last, whose elements have to be adjacent; an axis of one index has none."""
    s = [st if n > 1 else 0 for n, st in zip(t.shape, t.stride())]
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the last axis has to be contiguous")
    if written and any(n > 1 and st == 0 for n, st in zip(t.shape, s)):
        raise ValueError(f"{name}: is written, and has rows on top of each other")
    return (C.c_int64 * (len(s) - 1))(*s[:-1])


class VecInferError(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        super().__init__(f"vecinfer error {code}: {strerror(code)}")


_lib = None


def lib() -> C.CDLL:
    """Load the built library (raises if it is missing: build it first)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is not built; run `python -m paper_2510_06175_amd.build` "
                "(or __graft_entry__.build()) first")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        cfgp = C.POINTER(_Cfg)
        L.vecinfer_encode_keys.argtypes = [cfgp, vp, vp, vp, vp, i32, i64, i64, i64, vp]
        L.vecinfer_encode_keys.restype = C.c_int
        L.vecinfer_encode_values.argtypes = [cfgp, vp, vp, vp, i32, i64, i64, i64, vp]
        L.vecinfer_encode_values.restype = C.c_int
        L.vecinfer_append_kv.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp, i32, i64, i64, i64, vp]
        L.vecinfer_append_kv.restype = C.c_int
        L.vecinfer_decode_auto_splits.argtypes = [cfgp, i32, i64]
        L.vecinfer_decode_auto_splits.restype = i32
        L.vecinfer_decode_workspace_bytes.argtypes = [cfgp, i32, i64, i32]
        L.vecinfer_decode_workspace_bytes.restype = sz
        L.vecinfer_decode_attention.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp, i32, i64, i64, i32,
                                                i32, vp, sz, vp, vp, vp]
        L.vecinfer_decode_attention.restype = C.c_int
        L.vecinfer_decode_attention_static.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp, i32, i64, i64, i32,
                                                       i32, vp, vp, vp]
        L.vecinfer_decode_attention_static.restype = C.c_int
        L.vecinfer_decode_attention_residual.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp, i32, i64, i64, vp, vp,
                                                         vp, i32, i64, i32, i32, vp, sz, vp, vp, vp]
        L.vecinfer_decode_attention_residual.restype = C.c_int
        L.vecinfer_decode_step.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i64, i64, i32, i32, vp, sz,
                                           vp, vp, vp]
        L.vecinfer_decode_step.restype = C.c_int
        L.vecinfer_kmeans_workspace_bytes.argtypes = [cfgp, i32]
        L.vecinfer_kmeans_workspace_bytes.restype = sz
        L.vecinfer_kmeans_step.argtypes = [cfgp, vp, vp, vp, vp, vp, vp, i32, i64, vp, sz, vp]
        L.vecinfer_kmeans_step.restype = C.c_int
        L.vecinfer_kmeans_train.argtypes = [cfgp, vp, vp, vp, vp, vp, i32, i64, i32, C.c_float, vp, vp, vp, sz, vp]
        L.vecinfer_kmeans_train.restype = C.c_int
        L.vecinfer_calibrate_lambda.argtypes = [cfgp, vp, vp, i32, i64, vp]
        L.vecinfer_calibrate_lambda.restype = C.c_int
        L.vecinfer_read_probe.argtypes = [vp, sz, vp, vp]
        L.vecinfer_read_probe.restype = C.c_int
        L.vecinfer_export_value_codes.argtypes = [cfgp, vp, vp, i32, i64, i64, vp]
        L.vecinfer_export_value_codes.restype = C.c_int
        L.vecinfer_index_row_bytes.argtypes = [cfgp, i32]
        L.vecinfer_index_row_bytes.restype = sz
        L.vecinfer_codebook_elems.argtypes = [cfgp, i32]
        L.vecinfer_codebook_elems.restype = sz
        rotp, pagesp, i64p = C.POINTER(_RotaryCfg), C.POINTER(_Pages), C.POINTER(i64)
        L.vecinfer_rotary_table.argtypes = [rotp, vp, vp, vp]
        L.vecinfer_rotary_table.restype = C.c_int
        L.vecinfer_rotary.argtypes = [rotp, vp, i32, vp, i64p, vp, i64p, i32, i32, i64, vp, i64, i32, vp]
        L.vecinfer_rotary.restype = C.c_int
        L.vecinfer_paged_append.argtypes = [pagesp, rotp, vp, vp, i64p, vp, i64p, vp, i64p, vp, i64p, i32, vp, i64, vp, vp, vp,
                                            i32, i64, vp, i64, vp]
        L.vecinfer_paged_append.restype = C.c_int
        L.vecinfer_paged_workspace_bytes.argtypes = [pagesp, i32, i32, i64, i32, i32]
        L.vecinfer_paged_workspace_bytes.restype = sz
        L.vecinfer_paged_attention.argtypes = [pagesp, vp, i64p, i32, vp, i64, vp, i32, i64, C.c_float, i32, vp, sz, vp, vp, vp,
                                               vp, i64, vp]
        L.vecinfer_paged_attention.restype = C.c_int
        L.vecinfer_evict_workspace_bytes.argtypes = [i32, i32, i64, i64]
        L.vecinfer_evict_workspace_bytes.restype = sz
        L.vecinfer_paged_evict.argtypes = [pagesp, vp, i64, vp, i64, vp, i32, i64, i64, i64, i64, pagesp, vp, i64, vp, vp, i64,
                                           vp, vp, sz, vp]
        L.vecinfer_paged_evict.restype = C.c_int
        L.vecinfer_strerror.argtypes = [C.c_int]
        L.vecinfer_strerror.restype = C.c_char_p
        L.vecinfer_version.restype = C.c_int
        _lib = L
        _bind_fast(L)
    return _lib


# The module that does the hot calls' checks and conversions natively, once the library is loaded.  Its functions
# return None for arguments they leave to the checks here; without it every call takes that way.
_fast = None


def _bind_fast(L: C.CDLL) -> None:
    global _fast
    try:
        from . import _fastcall as m
    except ImportError:
        return
    if m.torch_version == torch.__version__.split("+")[0]:
        m.bind(*(C.cast(getattr(L, "vecinfer_" + n), C.c_void_p).value for n in (
            "encode_keys", "encode_values", "append_kv", "decode_attention", "decode_attention_residual", "decode_step")), _stream)
        m.bind_paged(*(C.cast(getattr(L, "vecinfer_" + n), C.c_void_p).value for n in (
            "rotary", "paged_append", "paged_attention", "paged_evict")), _stream_on,
                     getattr(torch._C, "_cuda_getDevice", None), getattr(torch._C, "_cuda_getCurrentRawStream", None))
        _fast = m


def strerror(code: int) -> str:
    return lib().vecinfer_strerror(int(code)).decode()


def vecinfer_version() -> int:
    return int(lib().vecinfer_version())


def _check(rc: int) -> None:
    if rc != 0:
        raise VecInferError(rc)


# The current stream's handle without a Stream object around it, where this torch offers that.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _dev(t: torch.Tensor, dtype, shape, name: str) -> int:
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a tensor on the GPU")
    raise ValueError(f"{name}: expected contiguous {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")


def _stream(stream) -> int:
    if stream is None:
        return _raw_stream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _stream_on(stream, device: int) -> int:
    """_stream for work on tensors of that device, which has to be the current one."""
    if device != torch.cuda.current_device():
        raise ValueError(f"the tensors are on cuda:{device}, the current device is cuda:{torch.cuda.current_device()}")
    return _raw_stream(device) if stream is None else _stream(stream)


def vecinfer_encode_keys(cfg: Config, k_f16, lam, cb_k, k_idx, pos0: int = 0, stream=None) -> None:
    """Smooth + Hadamard + VQ of T new keys into rows pos0.. of the code cache."""
    if _fast is not None:
        rc = _fast.encode(cfg._p, k_f16, lam, cb_k, k_idx, pos0, stream) if lam is not None else None
        if rc is not None:
            return _check(rc)
    B, Hkv, T, D = k_f16.shape
    n_cap = k_idx.shape[2]
    _check(lib().vecinfer_encode_keys(
        C.byref(cfg._c), _dev(k_f16, torch.float16, (B, cfg.num_kv_heads, T, cfg.head_dim), "k_f16"),
        _dev(lam, torch.float32, cfg._lam_shape, "lambda"),
        _dev(cb_k, torch.float16, cfg._cb_k, "cb_k"),
        _dev(k_idx, torch.uint8, (B, cfg.num_kv_heads, n_cap, cfg._row_k), "k_idx"),
        B, T, pos0, n_cap, _stream(stream)))


def vecinfer_encode_values(cfg: Config, v_f16, cb_v, v_idx, pos0: int = 0, stream=None) -> None:
    """VQ of T new (untransformed) values into rows pos0.. of the code cache."""
    if _fast is not None:
        rc = _fast.encode(cfg._p, v_f16, None, cb_v, v_idx, pos0, stream)
        if rc is not None:
            return _check(rc)
    B, Hkv, T, D = v_f16.shape
    n_cap = v_idx.shape[2]
    _check(lib().vecinfer_encode_values(
        C.byref(cfg._c), _dev(v_f16, torch.float16, (B, cfg.num_kv_heads, T, cfg.head_dim), "v_f16"),
        _dev(cb_v, torch.float16, cfg._cb_v, "cb_v"),
        _dev(v_idx, torch.uint8, (B, cfg.num_kv_heads, n_cap, cfg._row_v), "v_idx"),
        B, T, pos0, n_cap, _stream(stream)))


def vecinfer_append_kv(cfg: Config, k_f16, v_f16, lam, cb_k, cb_v, k_idx, v_idx, pos0: int, stream=None) -> None:
    """Decode-time append (Eq. 9): encode T <= 16 new keys and values in one launch."""
    if _fast is not None:
        rc = _fast.append(cfg._p, k_f16, v_f16, lam, cb_k, cb_v, k_idx, v_idx, pos0, stream)
        if rc is not None:
            return _check(rc)
    B, Hkv, T, D = k_f16.shape
    n_cap = k_idx.shape[2]
    _check(lib().vecinfer_append_kv(
        C.byref(cfg._c), _dev(k_f16, torch.float16, (B, cfg.num_kv_heads, T, cfg.head_dim), "k_f16"),
        _dev(v_f16, torch.float16, (B, cfg.num_kv_heads, T, cfg.head_dim), "v_f16"),
        _dev(lam, torch.float32, cfg._lam_shape, "lambda"),
        _dev(cb_k, torch.float16, cfg._cb_k, "cb_k"),
        _dev(cb_v, torch.float16, cfg._cb_v, "cb_v"),
        _dev(k_idx, torch.uint8, (B, cfg.num_kv_heads, n_cap, cfg._row_k), "k_idx"),
        _dev(v_idx, torch.uint8, (B, cfg.num_kv_heads, n_cap, cfg._row_v), "v_idx"),
        B, T, pos0, n_cap, _stream(stream)))


def vecinfer_decode_auto_splits(cfg: Config, B: int, N: int) -> int:
    return int(lib().vecinfer_decode_auto_splits(C.byref(cfg._c), B, N))


def vecinfer_decode_workspace_bytes(cfg: Config, B: int, N: int, num_splits: int = 0) -> int:
    return int(lib().vecinfer_decode_workspace_bytes(C.byref(cfg._c), B, N, num_splits))


def new_workspace(cfg: Config, B: int, N: int, num_splits: int = 0, device="cuda") -> torch.Tensor:
    """Allocate (with torch) a workspace for vecinfer_decode_attention."""
    nbytes = vecinfer_decode_workspace_bytes(cfg, B, N, num_splits)
    if nbytes == 0:
        raise VecInferError(EUNSUPPORTED)
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def vecinfer_decode_attention(cfg: Config, q_f16, lam, cb_k, cb_v, k_idx, v_idx, workspace, out_f16,
                              lse=None, seq_lens=None, N: int | None = None, num_splits: int = 0,
                              variant: int = VARIANT_AUTO, stream=None) -> None:
    """One fused VQ decode-attention step; writes out_f16 [B, Hq, D] (and lse [B, Hq])."""
    if _fast is not None:
        rc = _fast.decode(cfg._p, q_f16, lam, cb_k, cb_v, k_idx, v_idx, workspace, out_f16, lse, seq_lens, N, num_splits,
                          variant, stream)
        if rc is not None:
            return _check(rc)
    B = q_f16.shape[0]
    n_cap = k_idx.shape[2]
    N = n_cap if N is None else N
    _check(lib().vecinfer_decode_attention(
        C.byref(cfg._c), _dev(q_f16, torch.float16, (B, cfg.num_q_heads, cfg.head_dim), "q_f16"),
        _dev(lam, torch.float32, cfg._lam_shape, "lambda"),
        _dev(cb_k, torch.float16, cfg._cb_k, "cb_k"),
        _dev(cb_v, torch.float16, cfg._cb_v, "cb_v"),
        _dev(k_idx, torch.uint8, (B, cfg.num_kv_heads, n_cap, cfg._row_k), "k_idx"),
        _dev(v_idx, torch.uint8, (B, cfg.num_kv_heads, n_cap, cfg._row_v), "v_idx"),
        None if seq_lens is None else _dev(seq_lens, torch.int32, (B,), "seq_lens"),
        B, N, n_cap, num_splits, variant, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
        _dev(out_f16, torch.float16, (B, cfg.num_q_heads, cfg.head_dim), "out_f16"),
        None if lse is None else _dev(lse, torch.float32, (B, cfg.num_q_heads), "lse"),
        _stream(stream)))


STATIC_SCRATCH_BYTES = 4 << 20


def vecinfer_decode_attention_static(cfg: Config, q_f16, lam, cb_k, cb_v, k_idx, v_idx, out_f16,
                                     lse=None, seq_lens=None, N: int | None = None, num_splits: int = 0,
                                     variant: int = VARIANT_AUTO, stream=None) -> None:
    """vecinfer_decode_attention without a workspace argument: the split partials live in a fixed
    array inside the library (STATIC_SCRATCH_BYTES per GPU); the call allocates nothing."""
    B = q_f16.shape[0]
    n_cap = k_idx.shape[2]
    N = n_cap if N is None else N
    _check(lib().vecinfer_decode_attention_static(
        C.byref(cfg._c), _dev(q_f16, torch.float16, (B, cfg.num_q_heads, cfg.head_dim), "q_f16"),
        _dev(lam, torch.float32, cfg._lam_shape, "lambda"),
        _dev(cb_k, torch.float16, cfg._cb_k, "cb_k"),
        _dev(cb_v, torch.float16, cfg._cb_v, "cb_v"),
        _dev(k_idx, torch.uint8, (B, cfg.num_kv_heads, n_cap, cfg._row_k), "k_idx"),
        _dev(v_idx, torch.uint8, (B, cfg.num_kv_heads, n_cap, cfg._row_v), "v_idx"),
        None if seq_lens is None else _dev(seq_lens, torch.int32, (B,), "seq_lens"),
        B, N, n_cap, num_splits, variant,
        _dev(out_f16, torch.float16, (B, cfg.num_q_heads, cfg.head_dim), "out_f16"),
        None if lse is None else _dev(lse, torch.float32, (B, cfg.num_q_heads), "lse"),
        _stream(stream)))


def vecinfer_decode_attention_residual(cfg: Config, q_f16, lam, cb_k, cb_v, k_idx, v_idx, k_res, v_res, workspace,
                                       out_f16, lse=None, seq_lens=None, res_lens=None, N: int | None = None,
                                       R: int | None = None, num_splits: int = 0, variant: int = VARIANT_AUTO,
                                       stream=None) -> None:
    """Decode step over the code cache plus a full-precision window k_res / v_res [B, Hkv, r_cap, D]."""
    if _fast is not None:
        rc = _fast.decode(cfg._p, q_f16, lam, cb_k, cb_v, k_idx, v_idx, workspace, out_f16, lse, seq_lens, N, num_splits,
                          variant, stream, k_res, v_res, res_lens, R)
        if rc is not None:
            return _check(rc)
    B = q_f16.shape[0]
    n_cap = k_idx.shape[2]
    N = n_cap if N is None else N
    r_cap = k_res.shape[2]
    R = r_cap if R is None else R
    _check(lib().vecinfer_decode_attention_residual(
        C.byref(cfg._c), _dev(q_f16, torch.float16, (B, cfg.num_q_heads, cfg.head_dim), "q_f16"),
        _dev(lam, torch.float32, cfg._lam_shape, "lambda"),
        _dev(cb_k, torch.float16, cfg._cb_k, "cb_k"),
        _dev(cb_v, torch.float16, cfg._cb_v, "cb_v"),
        _dev(k_idx, torch.uint8, (B, cfg.num_kv_heads, n_cap, cfg._row_k), "k_idx"),
        _dev(v_idx, torch.uint8, (B, cfg.num_kv_heads, n_cap, cfg._row_v), "v_idx"),
        None if seq_lens is None else _dev(seq_lens, torch.int32, (B,), "seq_lens"),
        B, N, n_cap,
        _dev(k_res, torch.float16, (B, cfg.num_kv_heads, r_cap, cfg.head_dim), "k_res"),
        _dev(v_res, torch.float16, (B, cfg.num_kv_heads, r_cap, cfg.head_dim), "v_res"),
        None if res_lens is None else _dev(res_lens, torch.int32, (B,), "res_lens"),
        R, r_cap, num_splits, variant, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
        _dev(out_f16, torch.float16, (B, cfg.num_q_heads, cfg.head_dim), "out_f16"),
        None if lse is None else _dev(lse, torch.float32, (B, cfg.num_q_heads), "lse"),
        _stream(stream)))


def vecinfer_decode_step(cfg: Config, q_f16, k_new, v_new, lam, cb_k, cb_v, k_idx, v_idx, workspace, out_f16,
                         lse=None, seq_lens=None, N: int | None = None, num_splits: int = 0,
                         variant: int = VARIANT_AUTO, stream=None) -> None:
    """Append the new token (k_new, v_new [B, Hkv, 1, D]) as each sequence's last one and attend."""
    if _fast is not None:
        rc = _fast.decode(cfg._p, q_f16, lam, cb_k, cb_v, k_idx, v_idx, workspace, out_f16, lse, seq_lens, N, num_splits,
                          variant, stream, k_new, v_new)
        if rc is not None:
            return _check(rc)
    B = q_f16.shape[0]
    n_cap = k_idx.shape[2]
    N = n_cap if N is None else N
    _check(lib().vecinfer_decode_step(
        C.byref(cfg._c), _dev(q_f16, torch.float16, (B, cfg.num_q_heads, cfg.head_dim), "q_f16"),
        _dev(k_new, torch.float16, (B, cfg.num_kv_heads, 1, cfg.head_dim), "k_new"),
        _dev(v_new, torch.float16, (B, cfg.num_kv_heads, 1, cfg.head_dim), "v_new"),
        _dev(lam, torch.float32, cfg._lam_shape, "lambda"),
        _dev(cb_k, torch.float16, cfg._cb_k, "cb_k"),
        _dev(cb_v, torch.float16, cfg._cb_v, "cb_v"),
        _dev(k_idx, torch.uint8, (B, cfg.num_kv_heads, n_cap, cfg._row_k), "k_idx"),
        _dev(v_idx, torch.uint8, (B, cfg.num_kv_heads, n_cap, cfg._row_v), "v_idx"),
        None if seq_lens is None else _dev(seq_lens, torch.int32, (B,), "seq_lens"),
        B, N, n_cap, num_splits, variant, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
        _dev(out_f16, torch.float16, (B, cfg.num_q_heads, cfg.head_dim), "out_f16"),
        None if lse is None else _dev(lse, torch.float32, (B, cfg.num_q_heads), "lse"),
        _stream(stream)))


def vecinfer_index_row_bytes(cfg: Config, keys: bool) -> int:
    return int(lib().vecinfer_index_row_bytes(C.byref(cfg._c), 1 if keys else 0))


def vecinfer_codebook_elems(cfg: Config, keys: bool) -> int:
    return int(lib().vecinfer_codebook_elems(C.byref(cfg._c), 1 if keys else 0))


LAMBDA_FLOOR = 1e-5


def vecinfer_calibrate_lambda(cfg: Config, k_f16, lam, stream=None) -> None:
    """Eq. 4: lam [Hkv, D] = sqrt(max |k|) over all tokens of k_f16 [B, Hkv, T, D], floored at LAMBDA_FLOOR."""
    B, Hkv, T, D = k_f16.shape
    _check(lib().vecinfer_calibrate_lambda(
        C.byref(cfg._c), _dev(k_f16, torch.float16, (B, cfg.num_kv_heads, T, cfg.head_dim), "k_f16"),
        _dev(lam, torch.float32, cfg._lam_shape, "lambda"), B, T, _stream(stream)))


def vecinfer_export_value_codes(cfg: Config, v_idx_tiled, v_idx_rows, N: int | None = None, stream=None) -> None:
    """Rows form [B, Hkv, n_cap, M_v] (rows 0 .. N-1) of a value code cache kept in the tiled layout."""
    B, n_cap = v_idx_rows.shape[0], v_idx_rows.shape[2]
    shape = (B, cfg.num_kv_heads, n_cap, cfg._row_v)
    _check(lib().vecinfer_export_value_codes(
        C.byref(cfg._c), _dev(v_idx_tiled, torch.uint8, shape, "v_idx_tiled"),
        _dev(v_idx_rows, torch.uint8, shape, "v_idx_rows"), B, n_cap if N is None else N, n_cap, _stream(stream)))


def vecinfer_read_probe(src, sink, stream=None) -> None:
    """Plain streaming read of the whole tensor `src` (measurement aid); `sink`: any device tensor of >= 4 bytes."""
    if not src.is_cuda or not sink.is_cuda or not src.is_contiguous():
        raise TypeError("read probe: expected contiguous device tensors")
    _check(lib().vecinfer_read_probe(src.data_ptr(), src.numel() * src.element_size(), sink.data_ptr(),
                                     _stream(stream)))


def vecinfer_kmeans_workspace_bytes(cfg: Config, keys: bool) -> int:
    return int(lib().vecinfer_kmeans_workspace_bytes(C.byref(cfg._c), 1 if keys else 0))


def new_kmeans_workspace(cfg: Config, keys: bool, device="cuda") -> torch.Tensor:
    return torch.empty(vecinfer_kmeans_workspace_bytes(cfg, keys), dtype=torch.uint8, device=device)


def vecinfer_kmeans_step(cfg: Config, x_f16, lam, cb_in, cb_out, codes, workspace, counts=None, stream=None) -> None:
    """One Lloyd iteration of the codebook training on x_f16 [B, Hkv, T, D]; lam = None trains a
    value codebook (no transform).  Writes cb_out, codes [B, Hkv, T, row bytes] and, if given, counts
    (one per centroid: the codebook's shape without its last axis)."""
    B, Hkv, T, D = x_f16.shape
    keys = lam is not None
    ws = workspace
    cb_shape = cfg.cb_shape(keys)
    _check(lib().vecinfer_kmeans_step(
        C.byref(cfg._c), _dev(x_f16, torch.float16, (B, cfg.num_kv_heads, T, cfg.head_dim), "x_f16"),
        None if lam is None else _dev(lam, torch.float32, cfg._lam_shape, "lambda"),
        _dev(cb_in, torch.float16, cb_shape, "cb_in"),
        _dev(cb_out, torch.float16, cb_shape, "cb_out"),
        _dev(codes, torch.uint8, (B, cfg.num_kv_heads, T, cfg.row_bytes(keys)), "codes"),
        None if counts is None else _dev(counts, torch.int32, cb_shape[:-1], "counts"),
        B, T, ws.data_ptr(), ws.numel(), _stream(stream)))


KMEANS_MAX_ITERS = 30


def vecinfer_kmeans_train(cfg: Config, x_f16, lam, cb, codes, workspace, counts=None, max_iters: int = 30,
                          tol: float = 1e-4, iters_run=None, errors=None, stream=None) -> None:
    """K-Means training in place on cb (at most max_iters Lloyd iterations, stopping rule on the device).
    iters_run: int32 device tensor [1] or None; errors: float64 device tensor [max_iters] or None."""
    B, Hkv, T, D = x_f16.shape
    keys = lam is not None
    cb_shape = cfg.cb_shape(keys)
    _check(lib().vecinfer_kmeans_train(
        C.byref(cfg._c), _dev(x_f16, torch.float16, (B, cfg.num_kv_heads, T, cfg.head_dim), "x_f16"),
        None if lam is None else _dev(lam, torch.float32, cfg._lam_shape, "lambda"),
        _dev(cb, torch.float16, cb_shape, "cb"),
        _dev(codes, torch.uint8, (B, cfg.num_kv_heads, T, cfg.row_bytes(keys)), "codes"),
        None if counts is None else _dev(counts, torch.int32, cb_shape[:-1], "counts"),
        B, T, max_iters, tol,
        None if iters_run is None else _dev(iters_run, torch.int32, (1,), "iters_run"),
        None if errors is None else _dev(errors, torch.float64, (max_iters,), "errors"),
        workspace.data_ptr(), workspace.numel(), _stream(stream)))


def _here(t: torch.Tensor, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a tensor on the GPU")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name}: is on {t.device}, the current device is cuda:{torch.cuda.current_device()}")
    return t


def _rows(t: torch.Tensor, dtype, shape, name: str, written: bool = False):
    """Pointer and strides of a tensor of any strides with adjacent channels."""
    if _here(t, name).dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name}: expected {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    return t.data_ptr(), _steps(t, name, written)


def _flat(t: torch.Tensor | None, dtype, shape, name: str) -> int | None:
    """Pointer of a contiguous tensor on the current device, or None."""
    return None if t is None else _dev(_here(t, name), dtype, shape, name)


def _workspace(t: torch.Tensor) -> tuple:
    if not _here(t, "workspace").is_contiguous():
        raise ValueError("workspace: expected a contiguous tensor")
    return t.data_ptr(), t.numel() * t.element_size()


def _pool(p: Pages, name: str) -> "C._Pointer":
    if not isinstance(p, Pages):
        raise TypeError(f"{name}: expected Pages")
    _here(p.k, name)
    return C.byref(p._c)


def vecinfer_rotary_table(rot: Rotary, table, freqs=None, stream=None) -> None:
    """Turns per position of every pair into table, int64 [R / 2] (64-bit fractions of a turn); freqs: float64 [R / 2]
    radians per position in place of the configuration's formula."""
    n = rot.rot_dim // 2
    _check(lib().vecinfer_rotary_table(C.byref(rot._c), _flat(freqs, torch.float64, (n,), "freqs"),
                                       _flat(table, torch.int64, (n,), "table"), _stream(stream)))


def new_rotary_table(rot: Rotary, freqs=None, device="cuda") -> torch.Tensor:
    table = torch.empty(max(rot.rot_dim // 2, 0), dtype=torch.int64, device=device)
    vecinfer_rotary_table(rot, table, freqs)
    return table


def vecinfer_rotary(rot: Rotary, table, x, out, positions=None, pos0: int = 0, inverse: int = 0, stream=None) -> None:
    """Turn x [B, H, T, D] (fp16 or bf16, any strides) into out by its positions: int32 [B, T], or pos0 + t.  out may be
    x.  inverse: turn back, which takes the gradient of out to that of x."""
    if _fast is not None and type(rot) is Rotary:
        rc = _fast.rotary(rot._p, table, x, out, positions, pos0, inverse, stream)
        if rc is not None:
            return _check(rc)
    if not isinstance(x, torch.Tensor) or x.dim() != 4 or x.dtype not in _TYPES:
        raise ValueError("x: expected fp16 or bf16 [B, H, T, D]")
    B, H, T, D = x.shape
    px, sx = _rows(x, x.dtype, (B, H, T, rot.head_dim), "x")
    po, so = _rows(out, x.dtype, (B, H, T, rot.head_dim), "out", True)
    _check(lib().vecinfer_rotary(C.byref(rot._c), _flat(table, torch.int64, (rot.rot_dim // 2,), "table"), _TYPES[x.dtype],
                                 px, sx, po, so, B, H, T, _flat(positions, torch.int32, (B, T), "positions"), pos0,
                                 1 if inverse else 0, _stream(stream)))


def vecinfer_paged_append(pages: Pages, k_new, v_new, block_table, seq_lens, new_lens=None, rot: Rotary | None = None,
                          table=None, positions=None, q=None, q_out=None, weights=None, stream=None) -> None:
    """Write T new tokens per sequence, k_new and v_new [B, Hkv, T, D], to their pages (block_table int32 [B, max_pages]),
    keys turned by `rot`; turn the queries q [B, Hq, T, D] into q_out.  seq_lens [B] count the new tokens, of which
    sequence b has new_lens[b] (or T)."""
    if _fast is not None and type(pages) is Pages and (rot is None or type(rot) is Rotary):
        rc = _fast.paged_append(pages._p, pages._dev, None if rot is None else rot._p, table, k_new, v_new, q, q_out, block_table,
                                seq_lens, new_lens, positions, weights, stream)
        if rc is not None:
            return _check(rc)
    pool, dtype = _pool(pages, "pages"), pages.k.dtype
    B, Hkv, T, D = k_new.shape
    shape = (B, pages.num_kv_heads, T, pages.head_dim)
    pk, sk = _rows(k_new, dtype, shape, "k_new")
    pv, sv = _rows(v_new, dtype, shape, "v_new")
    pq = sq = po = so = None
    Hq = 0
    if q is not None:
        Hq = q.shape[1]
        pq, sq = _rows(q, dtype, (B, Hq, T, pages.head_dim), "q")
    if q_out is not None:
        po, so = _rows(q_out, dtype, (B, Hq, T, pages.head_dim), "q_out", True)
    w_cap = 0 if weights is None else weights.shape[-1]
    _check(lib().vecinfer_paged_append(
        pool, None if rot is None else C.byref(rot._c),
        None if rot is None else _flat(table, torch.int64, (rot.rot_dim // 2,), "table"), pk, sk, pv, sv, pq, sq, po, so, Hq,
        _flat(block_table, torch.int32, (B, block_table.shape[-1]), "block_table"), block_table.shape[-1],
        _flat(seq_lens, torch.int32, (B,), "seq_lens"), _flat(new_lens, torch.int32, (B,), "new_lens"),
        _flat(positions, torch.int32, (B, T), "positions"), B, T,
        _flat(weights, torch.float32, (B, pages.num_kv_heads, w_cap), "weights"), w_cap, _stream(stream)))


def vecinfer_paged_workspace_bytes(pages: Pages, num_q_heads: int, B: int, N: int, num_splits: int = 0, weights: int = 0) -> int:
    return int(lib().vecinfer_paged_workspace_bytes(_pool(pages, "pages"), num_q_heads, B, N, num_splits, 1 if weights else 0))


def new_paged_workspace(pages: Pages, num_q_heads: int, B: int, N: int, num_splits: int = 0, weights: int = 0) -> torch.Tensor:
    """Allocate (with torch) a workspace for vecinfer_paged_attention."""
    nbytes = vecinfer_paged_workspace_bytes(pages, num_q_heads, B, N, num_splits, weights)
    if nbytes == 0:
        raise VecInferError(EUNSUPPORTED)
    return torch.empty(nbytes, dtype=torch.uint8, device=pages.k.device)


def vecinfer_paged_attention(pages: Pages, q, block_table, workspace, out, lse=None, seq_lens=None, N: int | None = None,
                             scale: float | None = None, num_splits: int = 0, weights_in=None, weights_out=None,
                             stream=None) -> None:
    """Attention of one new token per sequence, q [B, Hq, D] (any strides), over its pages; writes out [B, Hq, D] (and lse
    [B, Hq]).  scale: 1 / sqrt(D) unless given.  weights_out [B, Hkv, w_cap] = weights_in (or 0) + the attention weights
    of the step, summed over the heads of a KV head; weights_in may be weights_out."""
    if _fast is not None and type(pages) is Pages:
        rc = _fast.paged_attention(pages._p, pages._dev, q, block_table, workspace, out, lse, seq_lens, N, scale, num_splits,
                                   weights_in, weights_out, stream)
        if rc is not None:
            return _check(rc)
    pool = _pool(pages, "pages")
    B, Hq, D = q.shape
    dtype = pages.k.dtype
    pq, sq = _rows(q, dtype, (B, Hq, pages.head_dim), "q")
    max_pages = block_table.shape[-1]
    N = max_pages * pages.page_size if N is None else N
    w_cap = 0 if weights_out is None else weights_out.shape[-1]
    if weights_out is None and weights_in is not None:
        raise VecInferError(EINVAL)
    wp, wb = _workspace(workspace)
    _check(lib().vecinfer_paged_attention(
        pool, pq, sq, Hq, _flat(block_table, torch.int32, (B, max_pages), "block_table"), max_pages,
        _flat(seq_lens, torch.int32, (B,), "seq_lens"), B, N, pages.head_dim ** -0.5 if scale is None else scale, num_splits,
        wp, wb, _flat(out, dtype, (B, Hq, pages.head_dim), "out"), _flat(lse, torch.float32, (B, Hq), "lse"),
        _flat(weights_in, torch.float32, (B, pages.num_kv_heads, w_cap), "weights_in"),
        _flat(weights_out, torch.float32, (B, pages.num_kv_heads, w_cap), "weights_out"), w_cap, _stream(stream)))


def vecinfer_evict_workspace_bytes(num_kv_heads: int, B: int, N: int, keep: int) -> int:
    return int(lib().vecinfer_evict_workspace_bytes(num_kv_heads, B, N, keep))


def new_evict_workspace(pages: Pages, B: int, N: int, keep: int) -> torch.Tensor:
    """Allocate (with torch) a workspace for vecinfer_paged_evict."""
    nbytes = vecinfer_evict_workspace_bytes(pages.num_kv_heads, B, N, keep)
    if nbytes == 0:
        raise VecInferError(EUNSUPPORTED)
    return torch.empty(nbytes, dtype=torch.uint8, device=pages.k.device)


def vecinfer_paged_evict(pages: Pages, weights, block_table, dst_pages: Pages, dst_table, dst_lens, workspace, keep: int,
                         first: int = 0, recent: int = 0, seq_lens=None, N: int | None = None, dst_weights=None, kept=None,
                         stream=None) -> None:
    """Keep, per sequence and KV head, the first `first` and last `recent` tokens and those of the largest weights
    [B, Hkv, w_cap], `keep` in all, in order, in the pages of dst_table [B, dst_max_pages] (of `dst_pages`, which may be
    `pages`; not pages that are read).  Writes dst_lens [B] and, if given, dst_weights [B, Hkv, dst_w_cap] and the kept
    tokens' old indices, kept [B, Hkv, keep].  N: as many tokens as weights has, at most, unless given."""
    if _fast is not None and type(pages) is Pages and type(dst_pages) is Pages:
        rc = _fast.paged_evict(pages._p, pages._dev, weights, block_table, dst_pages._p, dst_pages._dev, dst_table, dst_lens, workspace,
                               keep, first, recent, seq_lens, N, dst_weights, kept, stream)
        if rc is not None:
            return _check(rc)
    src, dst = _pool(pages, "pages"), _pool(dst_pages, "dst_pages")
    B, max_pages = block_table.shape
    Hkv, w_cap = pages.num_kv_heads, weights.shape[-1]
    dst_w_cap = 0 if dst_weights is None else dst_weights.shape[-1]
    N = min(w_cap, max_pages * pages.page_size) if N is None else N
    wp, wb = _workspace(workspace)
    _check(lib().vecinfer_paged_evict(
        src, _flat(weights, torch.float32, (B, Hkv, w_cap), "weights"), w_cap,
        _flat(block_table, torch.int32, (B, max_pages), "block_table"), max_pages, _flat(seq_lens, torch.int32, (B,), "seq_lens"),
        B, N, keep, first, recent, dst, _flat(dst_table, torch.int32, (B, dst_table.shape[-1]), "dst_table"), dst_table.shape[-1],
        _flat(dst_lens, torch.int32, (B,), "dst_lens"), _flat(dst_weights, torch.float32, (B, Hkv, dst_w_cap), "dst_weights"),
        dst_w_cap, _flat(kept, torch.int32, (B, Hkv, keep), "kept"), wp, wb, _stream(stream)))
