"""ctypes binding of libiwdft.so -- same names as include/iwdft.h, argument marshalling only.

torch is used for device buffers and streams; every arithmetic step runs in the
library's HIP kernels.  There is no fallback: if the shared library is missing
or a call fails, an exception is raised.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import os
import warnings
from typing import Optional, Sequence

import numpy as np
import torch

IWDFT_OK = 0
IWDFT_ERR_ARG, IWDFT_ERR_BINS, IWDFT_ERR_SIZE = -1, -2, -3
IWDFT_ERR_STATE, IWDFT_ERR_HIP, IWDFT_ERR_UNSUPPORTED = -4, -5, -6
IWDFT_F32, IWDFT_BF16 = 0, 1
IWDFT_FLAG_DIRECT_SYNTHESIS = 1
IWDFT_FLAG_DENSE_PREFILL = 2
IWDFT_FLAG_FFT_PREFILL = 4
IWDFT_FLAG_SHORTCUT = 8
IWDFT_FLAG_SERIAL_PHASES = 16
IWDFT_STATIC_SCRATCH_BYTES = 64 << 20

EXPORTED = [
    "iwdft_query_bytes", "iwdft_create", "iwdft_destroy", "iwdft_prefill", "iwdft_append",
    "iwdft_reconstruct", "iwdft_reconstruct_grid", "compressed_decode_attn", "iwdft_append_attn", "iwdft_export_coeffs", "iwdft_export_bins",
    "iwdft_num_tokens", "iwdft_set_num_tokens", "iwdft_last_error", "iwdft_phase_timing", "iwdft_phase_times", "iwdft_prefill_kind", "iwdft_attn_kind", "iwdft_attn_pipelined",
    "iwdft_select_bins", "iwdft_ablate_chunk", "iwdft_flush", "compressed_decode_attn_static", "iwdft_query_attn",
    "iwdft_pages_query_bytes", "iwdft_pages_resize", "iwdft_pages_resize_bytes", "iwdft_pages_write", "iwdft_pages_attn", "iwdft_pages_attn_bytes", "iwdft_pages_read",
    "iwdft_pages_fork", "iwdft_pages_fork_bytes", "iwdft_pages_resize_shared", "iwdft_pages_copy", "iwdft_pages_compact", "iwdft_pages_compact_bytes",
    "iwdft_pages_plan", "iwdft_pages_plan_bytes", "iwdft_pages_attn_shared", "iwdft_pages_attn_shared_bytes",
]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libiwdft.so")


class IwdftError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libiwdft error {code}: {msg}")
        self.code = code


class iwdft_desc(ctypes.Structure):
    _fields_ = [
        ("n_layers", ctypes.c_int32), ("batch", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("n_q_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("kv_dtype", ctypes.c_int32),
        ("M", ctypes.c_int64),
        ("bin_offsets", ctypes.POINTER(ctypes.c_int64)),
        ("bins", ctypes.POINTER(ctypes.c_int32)),
        ("bin_weights", ctypes.POINTER(ctypes.c_float)),
        ("flags", ctypes.c_uint32), ("n_sink", ctypes.c_int32), ("n_recent", ctypes.c_int32),
        ("write_every", ctypes.c_uint32),
    ]


class iwdft_pages_desc(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("n_layers", "n_pages", "n_kv_heads", "n_q_heads", "head_dim", "page_tokens", "max_pages", "kv_dtype")]


_lib = None


def load_library() -> ctypes.CDLL:
    """Loads libiwdft.so from the package directory; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} not found: build it with `python -m paper_2507_20030_amd.build` "
                          "(there is no fallback implementation)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    dp = ctypes.POINTER(iwdft_desc)
    szp = ctypes.POINTER(ctypes.c_size_t)
    lib.iwdft_query_bytes.argtypes = [dp, szp, szp]
    lib.iwdft_query_attn.argtypes = [dp, i32, i32, ctypes.POINTER(i32)]
    lib.iwdft_create.argtypes = [dp, vp, ctypes.c_size_t, vp, ctypes.c_size_t, ctypes.POINTER(vp)]
    lib.iwdft_destroy.argtypes = [vp]
    lib.iwdft_prefill.argtypes = [vp, vp, vp, vp]
    lib.iwdft_append.argtypes = [vp, vp, vp, vp]
    lib.iwdft_reconstruct.argtypes = [vp, i32, i64, i64, vp, vp, vp]
    lib.iwdft_reconstruct_grid.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp]
    lib.compressed_decode_attn.argtypes = [vp, vp, vp, f32, vp]
    lib.compressed_decode_attn_static.argtypes = [vp, vp, vp, f32, vp]
    lib.iwdft_append_attn.argtypes = [vp, vp, vp, vp, vp, f32, vp]
    lib.iwdft_prefill_kind.argtypes = [vp]
    lib.iwdft_attn_kind.argtypes = [vp]
    lib.iwdft_attn_pipelined.argtypes = [vp]
    lib.iwdft_flush.argtypes = [vp, vp]
    lib.iwdft_select_bins.argtypes = [ctypes.POINTER(ctypes.c_float), i32, i32, i64, ctypes.c_double,
                                      ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int32), i64]
    lib.iwdft_ablate_chunk.argtypes = [vp, vp, i64, i64, i32, i32, i32, i32, vp]
    lib.iwdft_phase_timing.argtypes = [vp, i32]
    lib.iwdft_phase_times.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    lib.iwdft_export_coeffs.argtypes = [vp, i32, vp, vp, vp]
    lib.iwdft_export_bins.argtypes = [vp, i32, vp, vp]
    pp = ctypes.POINTER(iwdft_pages_desc)
    lib.iwdft_pages_query_bytes.argtypes = [pp, szp, szp]
    lib.iwdft_pages_resize.argtypes = [i32, i32, i32, vp, i32, vp, vp, vp, vp, vp, i32, vp, ctypes.c_size_t, vp]
    lib.iwdft_pages_resize_bytes.argtypes = [i32, i32, szp]
    lib.iwdft_pages_write.argtypes = [pp, i32, i32, vp, vp, vp, i32, vp, vp, vp]
    lib.iwdft_pages_attn.argtypes = [pp, i32, i32, vp, vp, i32, vp, vp, i32, vp, vp, vp, i32, i32, f32, vp, ctypes.c_size_t, vp]
    lib.iwdft_pages_attn_bytes.argtypes = [pp, i32, i32, i32, szp]
    lib.iwdft_pages_read.argtypes = [pp, i32, i32, vp, vp, i32, i32, vp, vp, vp, vp, vp]
    lib.iwdft_pages_fork.argtypes = [i32, i32, i32, vp, vp, i32, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.iwdft_pages_fork_bytes.argtypes = [i32, i32, szp]
    lib.iwdft_pages_resize_shared.argtypes = [i32, i32, i32, vp, i32, vp, vp, vp, vp, vp, vp, i32, vp, vp]
    lib.iwdft_pages_copy.argtypes = [pp, i32, i32, vp, i32, vp, vp, i32, vp, vp, vp]
    lib.iwdft_pages_compact.argtypes = [i32, i32, i32, i32, vp, vp, vp, vp, vp, i32, vp, ctypes.c_size_t, vp]
    lib.iwdft_pages_compact_bytes.argtypes = [i32, szp]
    lib.iwdft_pages_plan.argtypes = [pp, i32, vp, i32, vp, vp, i32, i32, i32, vp, ctypes.c_size_t, vp]
    lib.iwdft_pages_plan_bytes.argtypes = [pp, i32, i32, i32, szp]
    lib.iwdft_pages_attn_shared.argtypes = [pp, i32, i32, vp, i32, vp, ctypes.c_size_t, vp, i32, vp, vp, vp, i32, i32, f32, vp, ctypes.c_size_t, vp]
    lib.iwdft_pages_attn_shared_bytes.argtypes = [pp, i32, i32, i32, szp]
    lib.iwdft_num_tokens.argtypes = [vp]
    lib.iwdft_num_tokens.restype = i64
    lib.iwdft_set_num_tokens.argtypes = [vp, i64]
    lib.iwdft_last_error.argtypes = []
    lib.iwdft_last_error.restype = ctypes.c_char_p
    for name in EXPORTED:
        if name not in ("iwdft_num_tokens", "iwdft_last_error"):
            getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def iwdft_last_error() -> str:
    return load_library().iwdft_last_error().decode()


def _check(rc: int) -> None:
    if rc != IWDFT_OK:
        raise IwdftError(rc, iwdft_last_error())


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


class Descriptor:
    """Host-side description of a cache; keeps the numpy arrays the C struct points into."""

    def __init__(self, n_layers: int, batch: int, n_kv_heads: int, n_q_heads: int, head_dim: int,
                 kv_dtype: int, M: int, bins: Sequence[np.ndarray],
                 bin_weights: Optional[Sequence[np.ndarray]] = None, flags: int = 0,
                 n_sink: int = 0, n_recent: int = 0, write_every: int = 0):
        self.bins = [np.ascontiguousarray(b, dtype=np.int32) for b in bins]
        self._offsets = np.zeros(len(self.bins) + 1, dtype=np.int64)
        self._offsets[1:] = np.cumsum([len(b) for b in self.bins])
        self._flat = np.ascontiguousarray(np.concatenate(self.bins) if self.bins else np.zeros(0, np.int32))
        self._w = None
        if bin_weights is not None:
            self._w = np.ascontiguousarray(np.concatenate([np.asarray(w, np.float32) for w in bin_weights]))
        self.c = iwdft_desc(
            n_layers, batch, n_kv_heads, n_q_heads, head_dim, kv_dtype, M,
            self._offsets.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)),
            self._flat.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
            self._w.ctypes.data_as(ctypes.POINTER(ctypes.c_float)) if self._w is not None else None,
            flags, n_sink, n_recent, write_every)


def iwdft_query_bytes(desc: Descriptor):
    s, w = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(load_library().iwdft_query_bytes(ctypes.byref(desc.c), ctypes.byref(s), ctypes.byref(w)))
    return s.value, w.value


def iwdft_query_attn(desc: Descriptor, pending: int = 0, write_back: bool = False) -> int:
    """0: decode attention in one launch; n >= 1: n workgroups per pair of query heads in the softmax."""
    n = ctypes.c_int32(0)
    _check(load_library().iwdft_query_attn(ctypes.byref(desc.c), pending, int(write_back), ctypes.byref(n)))
    return n.value


def iwdft_create(desc: Descriptor, state: torch.Tensor, workspace: torch.Tensor) -> ctypes.c_void_p:
    ctx = ctypes.c_void_p()
    _check(load_library().iwdft_create(ctypes.byref(desc.c), _ptr(state), state.numel() * state.element_size(),
                                       _ptr(workspace), workspace.numel() * workspace.element_size(),
                                       ctypes.byref(ctx)))
    return ctx


def iwdft_destroy(ctx) -> None:
    _check(load_library().iwdft_destroy(ctx))


def iwdft_prefill(ctx, K: torch.Tensor, V: torch.Tensor, stream=None) -> None:
    _check(load_library().iwdft_prefill(ctx, _ptr(K), _ptr(V), _stream(stream)))


def iwdft_append(ctx, tok_k: torch.Tensor, tok_v: torch.Tensor, stream=None) -> None:
    _check(load_library().iwdft_append(ctx, _ptr(tok_k), _ptr(tok_v), _stream(stream)))


def iwdft_reconstruct(ctx, layer: int, a0: int, n_slots: int, Kt, Vt, stream=None) -> None:
    _check(load_library().iwdft_reconstruct(ctx, layer, a0, n_slots, _ptr(Kt), _ptr(Vt), _stream(stream)))


def iwdft_reconstruct_grid(ctx, layer: int, a0: int, stride: int, n_slots: int, Kt, Vt, stream=None) -> None:
    _check(load_library().iwdft_reconstruct_grid(ctx, layer, a0, stride, n_slots, _ptr(Kt), _ptr(Vt), _stream(stream)))


def compressed_decode_attn(ctx, q: torch.Tensor, out: torch.Tensor, scale: float = 0.0, stream=None) -> None:
    _check(load_library().compressed_decode_attn(ctx, _ptr(q), _ptr(out), scale, _stream(stream)))


def compressed_decode_attn_static(ctx, q: torch.Tensor, out: torch.Tensor, scale: float = 0.0, stream=None) -> None:
    _check(load_library().compressed_decode_attn_static(ctx, _ptr(q), _ptr(out), scale, _stream(stream)))


def iwdft_append_attn(ctx, tok_k, tok_v, q, out, scale: float = 0.0, stream=None) -> None:
    _check(load_library().iwdft_append_attn(ctx, _ptr(tok_k), _ptr(tok_v), _ptr(q), _ptr(out), scale,
                                            _stream(stream)))


def iwdft_select_bins(delta: np.ndarray, M: int, r: float):
    """Per-layer kept-bin lists (int32 arrays) from a [layers, chunks] importance matrix."""
    delta = np.ascontiguousarray(delta, dtype=np.float32)
    n_layers, n_chunks = delta.shape
    lib = load_library()
    off = (ctypes.c_int64 * (n_layers + 1))()
    dp = delta.ctypes.data_as(ctypes.POINTER(ctypes.c_float))
    rc = lib.iwdft_select_bins(dp, n_layers, n_chunks, M, float(r), off, None, 0)   # sizing call
    if rc != IWDFT_ERR_SIZE:
        _check(rc)
    bins = np.empty(max(int(off[n_layers]), 1), dtype=np.int32)
    _check(lib.iwdft_select_bins(dp, n_layers, n_chunks, M, float(r), off,
                                 bins.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), bins.size))
    return [bins[off[l]:off[l + 1]].copy() for l in range(n_layers)]


def iwdft_ablate_chunk(x: torch.Tensor, out: torch.Tensor, n_chunks: int, chunk: int, stream=None) -> None:
    """x, out: [..., M, head_dim] contiguous device tensors of the same shape and dtype."""
    M, D = x.shape[-2], x.shape[-1]
    n_slices = x.numel() // (M * D)
    _check(load_library().iwdft_ablate_chunk(_ptr(x), _ptr(out), n_slices, M, D,
                                             IWDFT_F32 if x.dtype == torch.float32 else IWDFT_BF16,
                                             n_chunks, chunk, _stream(stream)))


def iwdft_flush(ctx, stream=None) -> None:
    _check(load_library().iwdft_flush(ctx, _stream(stream)))


def iwdft_prefill_kind(ctx) -> str:
    """"chirp" stands for all lengths that are no power of two: their prefill is interpolated from power-of-two transforms."""
    return {0: "dense", 1: "fft", 2: "chirp"}[load_library().iwdft_prefill_kind(ctx)]


def iwdft_attn_kind(ctx) -> str:
    """"chirp" stands for all lengths that are no power of two: chirp-z transforms or transforms interpolated from a power-of-two grid."""
    return {0: "direct", 1: "fft", 2: "chirp"}[load_library().iwdft_attn_kind(ctx)]


def iwdft_attn_pipelined(ctx) -> bool:
    return load_library().iwdft_attn_pipelined(ctx) == 1


def iwdft_phase_timing(ctx, enable: bool) -> None:
    _check(load_library().iwdft_phase_timing(ctx, 1 if enable else 0))


def iwdft_phase_times(ctx):
    """(ms of phases A, B, C summed over the marked calls since the last read-out, number of calls)."""
    ms = (ctypes.c_double * 3)()
    n = ctypes.c_int64(0)
    _check(load_library().iwdft_phase_times(ctx, ms, ctypes.byref(n)))
    return [ms[0], ms[1], ms[2]], n.value


def iwdft_export_coeffs(ctx, layer: int, SK, SV, stream=None) -> None:
    _check(load_library().iwdft_export_coeffs(ctx, layer, _ptr(SK), _ptr(SV), _stream(stream)))


def iwdft_export_bins(ctx, layer: int, out: torch.Tensor, stream=None) -> None:
    _check(load_library().iwdft_export_bins(ctx, layer, _ptr(out), _stream(stream)))


def iwdft_num_tokens(ctx) -> int:
    return int(load_library().iwdft_num_tokens(ctx))


def iwdft_set_num_tokens(ctx, T: int) -> None:
    _check(load_library().iwdft_set_num_tokens(ctx, T))


class Cache:
    """Owns the torch buffers behind one iwdft_ctx; methods forward to the C calls."""

    def __init__(self, n_layers, batch, n_kv_heads, n_q_heads, head_dim, dtype: torch.dtype, M,
                 bins, bin_weights=None, flags=0, device="cuda:0", n_sink=0, n_recent=0, write_every=0):
        if dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("dtype must be float32 or bfloat16")
        self.dtype, self.device = dtype, torch.device(device)
        self.desc = Descriptor(n_layers, batch, n_kv_heads, n_q_heads, head_dim,
                               IWDFT_F32 if dtype == torch.float32 else IWDFT_BF16, M, bins, bin_weights, flags,
                               n_sink, n_recent, write_every)
        self.state_bytes, self.ws_bytes = iwdft_query_bytes(self.desc)
        with torch.cuda.device(self.device):
            self.state = torch.empty(self.state_bytes, dtype=torch.uint8, device=self.device)
            self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=self.device)
            self.ctx = iwdft_create(self.desc, self.state, self.workspace)
        self.shape = (n_layers, batch, n_kv_heads, n_q_heads, head_dim)

    def close(self):
        if self.ctx is not None:
            iwdft_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def T(self) -> int:
        return iwdft_num_tokens(self.ctx)

    def prefill(self, K, V, stream=None):
        iwdft_prefill(self.ctx, K, V, stream)

    def append(self, tok_k, tok_v, stream=None):
        iwdft_append(self.ctx, tok_k, tok_v, stream)

    def attend(self, q, out=None, scale=0.0, stream=None):
        if out is None:
            out = torch.empty_like(q)
        compressed_decode_attn(self.ctx, q, out, scale, stream)
        return out

    def step(self, tok_k, tok_v, q, out=None, scale=0.0, stream=None):
        """Fused decode step: append (tok_k, tok_v), then attend with q."""
        if out is None:
            out = torch.empty_like(q)
        iwdft_append_attn(self.ctx, tok_k, tok_v, q, out, scale, stream)
        return out

    def flush(self, stream=None):
        iwdft_flush(self.ctx, stream)

    def reconstruct(self, layer, a0, n_slots, want_k=True, want_v=True, stream=None, stride=1):
        L, B, H, _, D = self.shape
        mk = lambda: torch.empty((B, H, n_slots, D), dtype=self.dtype, device=self.device)
        Kt, Vt = (mk() if want_k else None), (mk() if want_v else None)
        if stride == 1:
            iwdft_reconstruct(self.ctx, layer, a0, n_slots, Kt, Vt, stream)
        else:
            iwdft_reconstruct_grid(self.ctx, layer, a0, stride, n_slots, Kt, Vt, stream)
        return Kt, Vt

    def export_coeffs(self, layer, stream=None):
        L, B, H, _, D = self.shape
        nb = len(self.desc.bins[layer])
        SK = torch.empty((B, H, nb, D, 2), dtype=torch.float32, device=self.device)
        SV = torch.empty_like(SK)
        iwdft_export_coeffs(self.ctx, layer, SK, SV, stream)
        return torch.view_as_complex(SK), torch.view_as_complex(SV)

    def export_bins(self, layer, stream=None):
        out = torch.empty(len(self.desc.bins[layer]), dtype=torch.int32, device=self.device)
        iwdft_export_bins(self.ctx, layer, out, stream)
        return out


# ------------------------------------------------------------------------------------------------------------------ 8-bit pages
# What include/iwdft.h says of the arrays; sizes come from the tensors' shapes:
#   values uint8 [layers, pages, KV heads, 2, P * 128], exponents int32 [layers, pages, KV heads, 2], table int32 [batch, max_pages],
#   lens int32 [batch], free int32 [1 + pages], starts int32 [batch + 1], slots int32 [tokens].
def pages_desc(n_layers, n_pages, n_kv_heads, n_q_heads=None, head_dim=128, page_tokens=32, max_pages=1, dtype=torch.bfloat16) -> iwdft_pages_desc:
    if dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("dtype must be float32 or bfloat16")
    return iwdft_pages_desc(n_layers, n_pages, n_kv_heads, n_kv_heads if n_q_heads is None else n_q_heads, head_dim, page_tokens, max_pages,
                            IWDFT_F32 if dtype == torch.float32 else IWDFT_BF16)


@functools.lru_cache(maxsize=1024)
def _pages_ref(*sizes):
    return ctypes.byref(pages_desc(*sizes))  # as the calls take it; keeps a descriptor of its own, which no caller can change


def _bytes_of(call, *args) -> int:
    n = ctypes.c_size_t(0)
    _check(call(*args, ctypes.byref(n)))
    return n.value


@functools.lru_cache(maxsize=1024)
def _resize_bytes(batch, n_slots):
    return _bytes_of(load_library().iwdft_pages_resize_bytes, batch, n_slots)


@functools.lru_cache(maxsize=1024)
def _attn_sizes(n_layers, batch, n_tokens, *desc):
    """The descriptor, as the call takes it, and the workspace's bytes."""
    ref = _pages_ref(*desc)
    return ref, _bytes_of(load_library().iwdft_pages_attn_bytes, ref, n_layers, batch, n_tokens)


def iwdft_pages_query_bytes(desc: iwdft_pages_desc):
    v, e = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(load_library().iwdft_pages_query_bytes(ctypes.byref(desc), ctypes.byref(v), ctypes.byref(e)))
    return v.value, e.value


def iwdft_pages_resize_bytes(batch: int, n_slots: int) -> int:
    return _resize_bytes(batch, n_slots)


def iwdft_pages_attn_bytes(desc: iwdft_pages_desc, n_layers: int, batch: int, n_tokens: int) -> int:
    return _bytes_of(load_library().iwdft_pages_attn_bytes, ctypes.byref(desc), n_layers, batch, n_tokens)


def _expect(name: str, t: torch.Tensor, dtype, shape, device) -> None:
    """shape: None where any size will do."""
    if t.dtype != dtype:
        raise ValueError(f"{name} is {t.dtype}, not {dtype}")
    if len(t.shape) != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape)):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple('any' if n is None else n for n in shape)}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _pool_sizes(values: torch.Tensor, exponents: torch.Tensor):
    """(index of the GPU, layers, pages, KV heads, page tokens)."""
    shape, index = values.shape, values.get_device()
    if len(shape) != 5 or shape[3] != 2 or shape[4] % 128:
        raise ValueError(f"values has shape {tuple(shape)}, not (layers, pages, heads, 2, 128 * page tokens)")
    if index < 0:
        raise ValueError("values must be device memory")
    n_layers, n_pages, heads, _, row = shape
    if not (values.dtype is torch.uint8 and values.is_contiguous() and exponents.dtype is torch.int32 and exponents.shape == (n_layers, n_pages, heads, 2)
            and exponents.get_device() == index and exponents.is_contiguous()):
        _expect("values", values, torch.uint8, shape, values.device)
        _expect("exponents", exponents, torch.int32, (n_layers, n_pages, heads, 2), values.device)
    return index, n_layers, n_pages, heads, row // 128


def _kv_dtype(name: str, t: torch.Tensor):
    if t.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"{name} is {t.dtype}, not float32 or bfloat16")
    return t.dtype


def _stream_of(stream, index: int):
    """The given stream or the device's current one."""
    return torch._C._cuda_getCurrentRawStream(index) if stream is None else _stream(stream)


def _on_stream(stream, device):
    """Allocations and fills in the order of the call's stream."""
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream), device))


def _scratch(n_bytes: int, device: torch.device, stream, workspace):
    """The caller's workspace, or memory of this call alone that is allocated and freed in the order of the call's stream."""
    if workspace is None:
        if not n_bytes:
            return None
        if stream is None:
            return torch.empty(n_bytes, dtype=torch.uint8, device=device)
        with _on_stream(stream, device):
            return torch.empty(n_bytes, dtype=torch.uint8, device=device)
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous and on {device}, not on {workspace.device}")
    return workspace


# The calls check their tensors in one expression -- a decode step makes one of these calls per layer -- and say what is wrong where it fails.
def iwdft_pages_resize(want, table, lens, free, starts, slots, page_tokens: int, stream=None, workspace=None) -> None:
    """Brings the sequences to want[b] tokens (negative: as they are): table, lens, free, starts and slots are brought up to date."""
    index, shape, i32 = table.get_device(), table.shape, torch.int32
    if len(shape) != 2 or index < 0:
        raise ValueError(f"table must be a device tensor [batch, max_pages], not {tuple(shape)} on {table.device}")
    batch, max_pages = shape
    n_free, n_slots = free.numel(), slots.numel()
    if not (table.dtype is want.dtype is lens.dtype is free.dtype is starts.dtype is slots.dtype is i32
            and index == want.get_device() == lens.get_device() == free.get_device() == starts.get_device() == slots.get_device()
            and want.shape == lens.shape == (batch,) and starts.shape == (batch + 1,) and free.dim() == slots.dim() == 1
            and table.is_contiguous() and want.is_contiguous() and lens.is_contiguous() and free.is_contiguous() and starts.is_contiguous()
            and slots.is_contiguous()):
        for name, t, size in (("table", table, shape), ("want", want, (batch,)), ("lens", lens, (batch,)), ("free", free, (n_free,)),
                              ("starts", starts, (batch + 1,)), ("slots", slots, (n_slots,))):
            _expect(name, t, i32, size, table.device)
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return iwdft_pages_resize(want, table, lens, free, starts, slots, page_tokens, stream, workspace)
    need = _resize_bytes(batch, n_slots)
    ws = _scratch(need, table.device, stream, workspace) if need or workspace is not None else None
    rc = load_library().iwdft_pages_resize(page_tokens, n_free - 1, max_pages, want.data_ptr(), batch, table.data_ptr(), lens.data_ptr(), free.data_ptr(),
                                           starts.data_ptr(), slots.data_ptr(), n_slots, ws.data_ptr() if ws is not None else None,
                                           ws.nbytes if ws is not None else 0, _stream_of(stream, index))
    if rc:
        _check(rc)


def iwdft_pages_write(values, exponents, k, v, slots, layer: int = 0, stream=None) -> None:
    """k, v [layers written, tokens, KV heads, 128] into layers layer, layer + 1, ... at slots."""
    index, n_layers, n_pages, heads, P = _pool_sizes(values, exponents)
    dtype, n, shape = _kv_dtype("k", k), slots.numel(), k.shape
    if not (slots.dtype is torch.int32 and slots.dim() == 1 and v.dtype is dtype and index == slots.get_device() == k.get_device() == v.get_device()
            and shape == v.shape and shape[1:] == (n, heads, 128) and slots.is_contiguous() and k.is_contiguous() and v.is_contiguous()):
        device = values.device
        _expect("slots", slots, torch.int32, (n,), device)
        _expect("k", k, dtype, (None, n, heads, 128), device)
        _expect("v", v, dtype, shape, device)
    if shape[0] == 0:
        return
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return iwdft_pages_write(values, exponents, k, v, slots, layer, stream)
    rc = load_library().iwdft_pages_write(_pages_ref(n_layers, n_pages, heads, heads, 128, P, 1, dtype), layer, shape[0], k.data_ptr(), v.data_ptr(),
                                          slots.data_ptr(), n, values.data_ptr(), exponents.data_ptr(), _stream_of(stream, index))
    if rc:
        _check(rc)


def iwdft_pages_attn(values, exponents, q, starts, table, lens, out, layer: int = 0, n_sink: int = 0, n_recent: int = 0, scale: float = 0.0, stream=None,
                     workspace=None) -> None:
    """q, out [layers, tokens, query heads, 128]: the new tokens' attention over their sequences in layers layer, layer + 1, ...  fp32 calls hold queries and
    weights in 22 bits, bf16 calls weights in 11."""
    index, n_layers, n_pages, heads, P = _pool_sizes(values, exponents)
    dtype, shape, size = _kv_dtype("q", q), q.shape, table.shape
    if not (len(shape) == 4 and len(size) == 2 and shape[3] == 128 and out.dtype is dtype and shape == out.shape
            and starts.dtype is table.dtype is lens.dtype is torch.int32 and lens.shape == size[:1] and starts.shape == (size[0] + 1,)
            and index == q.get_device() == out.get_device() == starts.get_device() == table.get_device() == lens.get_device()
            and q.is_contiguous() and out.is_contiguous()
            and starts.is_contiguous() and table.is_contiguous() and lens.is_contiguous()):
        device = values.device
        _expect("q", q, dtype, (None, None, None, 128), device)
        _expect("out", out, dtype, shape, device)
        _expect("table", table, torch.int32, (None, None), device)
        _expect("lens", lens, torch.int32, size[:1], device)
        _expect("starts", starts, torch.int32, (size[0] + 1,), device)
    n, n_tokens, n_q_heads, _ = shape
    batch, max_pages = size
    if n == 0:
        return
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return iwdft_pages_attn(values, exponents, q, starts, table, lens, out, layer, n_sink, n_recent, scale, stream, workspace)
    desc, need = _attn_sizes(n, batch, n_tokens, n_layers, n_pages, heads, n_q_heads, 128, P, max_pages, dtype)
    ws = _scratch(need, values.device, stream, workspace) if need or workspace is not None else None
    rc = load_library().iwdft_pages_attn(desc, layer, n, q.data_ptr(), starts.data_ptr(), n_tokens, table.data_ptr(), lens.data_ptr(), batch,
                                         values.data_ptr(), exponents.data_ptr(), out.data_ptr(), n_sink, n_recent, scale,
                                         ws.data_ptr() if ws is not None else None, ws.nbytes if ws is not None else 0, _stream_of(stream, index))
    if rc:
        _check(rc)


def iwdft_pages_read(values, exponents, table, lens, K, V, layer: int = 0, stream=None) -> None:
    """K, V [layers, batch, KV heads, tokens, 128] (either may be None) from the first tokens of every sequence; 0 where it has fewer."""
    index, n_layers, n_pages, heads, P = _pool_sizes(values, exponents)
    some = K if K is not None else V
    if some is None:
        return
    dtype, shape, size = _kv_dtype("K or V", some), some.shape, table.shape
    if not (len(size) == 2 and len(shape) == 5 and shape[1:3] == (size[0], heads) and shape[4] == 128 and table.dtype is lens.dtype is torch.int32
            and lens.shape == size[:1] and index == table.get_device() == lens.get_device() == some.get_device() and table.is_contiguous()
            and lens.is_contiguous() and some.is_contiguous()
            and (V is None or (V.dtype is dtype and V.shape == shape and V.get_device() == index and V.is_contiguous()))):
        device = values.device
        _expect("table", table, torch.int32, (None, None), device)
        _expect("lens", lens, torch.int32, size[:1], device)
        for name, t in (("K", K), ("V", V)):
            if t is not None:
                _expect(name, t, dtype, (shape[0], size[0], heads, shape[3] if len(shape) == 5 else None, 128), device)
    if shape[0] == 0:
        return
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return iwdft_pages_read(values, exponents, table, lens, K, V, layer, stream)
    rc = load_library().iwdft_pages_read(_pages_ref(n_layers, n_pages, heads, heads, 128, P, size[1], dtype), layer, shape[0], table.data_ptr(), lens.data_ptr(),
                                         size[0], shape[3], values.data_ptr(), exponents.data_ptr(), K.data_ptr() if K is not None else None,
                                         V.data_ptr() if V is not None else None, _stream_of(stream, index))
    if rc:
        _check(rc)


# Pages that sequences share: refs int32 [pages], copies int32 [n, 2].
@functools.lru_cache(maxsize=1024)
def iwdft_pages_fork_bytes(batch: int, max_pages: int) -> int:
    return _bytes_of(load_library().iwdft_pages_fork_bytes, batch, max_pages)


@functools.lru_cache(maxsize=1024)
def iwdft_pages_compact_bytes(n_pages: int) -> int:
    return _bytes_of(load_library().iwdft_pages_compact_bytes, n_pages)


def _check_tables(table, refs, batch, n_pages, others):
    """Says which tensor does not fit; others: (name, tensor, shape)."""
    if len(table.shape) != 2 or table.get_device() < 0:
        raise ValueError(f"table must be a device tensor [batch, max_pages], not {tuple(table.shape)} on {table.device}")
    for name, t, size in (("table", table, table.shape), ("refs", refs, (n_pages,)), *others):
        _expect(name, t, torch.int32, size, table.device)


def iwdft_pages_fork(parent, keep, table, lens, free, refs, page_tokens: int, stream=None, workspace=None) -> None:
    """Sequence b becomes the first keep[b] tokens (keep None, or negative: all) of what sequence parent[b] was: table, lens, free and refs are brought up to date."""
    index, shape, i32, n_pages = table.get_device(), table.shape, torch.int32, refs.numel()
    batch, max_pages = shape if len(shape) == 2 else (0, 0)
    if not (len(shape) == 2 and index >= 0 and parent.dtype is table.dtype is lens.dtype is free.dtype is refs.dtype is i32
            and index == parent.get_device() == lens.get_device() == free.get_device() == refs.get_device()
            and parent.shape == lens.shape == (batch,) and free.shape == (n_pages + 1,) and refs.dim() == 1
            and (keep is None or (keep.dtype is i32 and keep.get_device() == index and keep.shape == (batch,) and keep.is_contiguous()))
            and parent.is_contiguous() and table.is_contiguous() and lens.is_contiguous() and free.is_contiguous() and refs.is_contiguous()):
        _check_tables(table, refs, batch, n_pages, [("parent", parent, (batch,)), ("lens", lens, (batch,)), ("free", free, (n_pages + 1,))]
                      + ([] if keep is None else [("keep", keep, (batch,))]))
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return iwdft_pages_fork(parent, keep, table, lens, free, refs, page_tokens, stream, workspace)
    need = iwdft_pages_fork_bytes(batch, max_pages)
    ws = _scratch(need, table.device, stream, workspace) if need or workspace is not None else None
    rc = load_library().iwdft_pages_fork(page_tokens, n_pages, max_pages, parent.data_ptr(), None if keep is None else keep.data_ptr(), batch, table.data_ptr(),
                                         lens.data_ptr(), free.data_ptr(), refs.data_ptr(), ws.data_ptr() if ws is not None else None,
                                         ws.nbytes if ws is not None else 0, _stream_of(stream, index))
    if rc:
        _check(rc)


def iwdft_pages_resize_shared(want, table, lens, free, refs, starts, slots, copies, page_tokens: int, stream=None) -> None:
    """iwdft_pages_resize where pages are shared; copies [batch, 2] says what iwdft_pages_copy has to do before anything is written."""
    index, shape, i32, n_pages = table.get_device(), table.shape, torch.int32, refs.numel()
    batch, max_pages = shape if len(shape) == 2 else (0, 0)
    if not (len(shape) == 2 and index >= 0 and want.dtype is table.dtype is lens.dtype is free.dtype is refs.dtype is starts.dtype is slots.dtype is copies.dtype is i32
            and index == want.get_device() == lens.get_device() == free.get_device() == refs.get_device() == starts.get_device() == slots.get_device() == copies.get_device()
            and want.shape == lens.shape == (batch,) and starts.shape == (batch + 1,) and copies.shape == (batch, 2) and free.shape == (n_pages + 1,)
            and refs.dim() == slots.dim() == 1 and want.is_contiguous() and table.is_contiguous() and lens.is_contiguous() and free.is_contiguous()
            and refs.is_contiguous() and starts.is_contiguous() and slots.is_contiguous() and copies.is_contiguous()):
        _check_tables(table, refs, batch, n_pages, [("want", want, (batch,)), ("lens", lens, (batch,)), ("free", free, (n_pages + 1,)), ("starts", starts, (batch + 1,)),
                                                    ("slots", slots, (None,)), ("copies", copies, (batch, 2))])
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return iwdft_pages_resize_shared(want, table, lens, free, refs, starts, slots, copies, page_tokens, stream)
    rc = load_library().iwdft_pages_resize_shared(page_tokens, n_pages, max_pages, want.data_ptr(), batch, table.data_ptr(), lens.data_ptr(), free.data_ptr(),
                                                  refs.data_ptr(), starts.data_ptr(), slots.data_ptr(), slots.numel(), copies.data_ptr(), _stream_of(stream, index))
    if rc:
        _check(rc)


def iwdft_pages_compact(table, lens, free, refs, moves, page_tokens: int, stream=None, workspace=None) -> None:
    """Held pages together at the pool's beginning, moves.shape[0] of them at most: moves [n, 2] says what iwdft_pages_copy has to do."""
    index, shape, i32, n_pages = table.get_device(), table.shape, torch.int32, refs.numel()
    batch, max_pages = shape if len(shape) == 2 else (0, 0)
    if not (len(shape) == 2 and index >= 0 and table.dtype is lens.dtype is free.dtype is refs.dtype is moves.dtype is i32
            and index == lens.get_device() == free.get_device() == refs.get_device() == moves.get_device()
            and lens.shape == (batch,) and free.shape == (n_pages + 1,) and refs.dim() == 1 and moves.dim() == 2 and moves.shape[1] == 2
            and table.is_contiguous() and lens.is_contiguous() and free.is_contiguous() and refs.is_contiguous() and moves.is_contiguous()):
        _check_tables(table, refs, batch, n_pages, [("lens", lens, (batch,)), ("free", free, (n_pages + 1,)), ("moves", moves, (None, 2))])
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return iwdft_pages_compact(table, lens, free, refs, moves, page_tokens, stream, workspace)
    ws = _scratch(iwdft_pages_compact_bytes(n_pages), table.device, stream, workspace)
    rc = load_library().iwdft_pages_compact(page_tokens, n_pages, max_pages, batch, table.data_ptr(), lens.data_ptr(), free.data_ptr(), refs.data_ptr(),
                                            moves.data_ptr(), moves.shape[0], ws.data_ptr(), ws.nbytes, _stream_of(stream, index))
    if rc:
        _check(rc)


def iwdft_pages_copy(copies, values, exponents, to_values=None, to_exponents=None, layer: int = 0, n_layers: Optional[int] = None, stream=None) -> None:
    """Pages copies[:, 0] of values, exponents to copies[:, 1] of the other pool, or (None) of the same one, in n_layers layers from `layer` on (None: all that follow)."""
    index, all_layers, n_pages, heads, P = _pool_sizes(values, exponents)
    if (to_values is None) != (to_exponents is None):
        raise ValueError("to_values and to_exponents belong together")
    if to_values is None:
        to_values, to_exponents = values, exponents
    to_index, to_layers, to_pages, to_heads, to_P = _pool_sizes(to_values, to_exponents)
    if (to_index, to_layers, to_heads, to_P) != (index, all_layers, heads, P):
        raise ValueError(f"the pools differ: {tuple(values.shape)} on {values.device} and {tuple(to_values.shape)} on {to_values.device}")
    if not (copies.dtype is torch.int32 and copies.dim() == 2 and copies.shape[1] == 2 and copies.get_device() == index and copies.is_contiguous()):
        _expect("copies", copies, torch.int32, (None, 2), values.device)
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return iwdft_pages_copy(copies, values, exponents, to_values, to_exponents, layer, n_layers, stream)
    n = all_layers - layer if n_layers is None else n_layers
    rc = load_library().iwdft_pages_copy(_pages_ref(all_layers, n_pages, heads, heads, 128, P, 1, torch.float32), layer, n, copies.data_ptr(), copies.shape[0],
                                         values.data_ptr(), exponents.data_ptr(), to_pages, to_values.data_ptr(), to_exponents.data_ptr(), _stream_of(stream, index))
    if rc:
        _check(rc)


@functools.lru_cache(maxsize=1024)
def _shared_sizes(n_layers, batch, n_tokens, *desc):
    """The descriptor, as the calls take it, the plan's bytes and the workspace's."""
    ref, lib = _pages_ref(*desc), load_library()
    return ref, _bytes_of(lib.iwdft_pages_plan_bytes, ref, n_layers, batch, n_tokens), _bytes_of(lib.iwdft_pages_attn_shared_bytes, ref, n_layers, batch, n_tokens)


def iwdft_pages_plan_bytes(desc: iwdft_pages_desc, n_layers: int, batch: int, n_tokens: int) -> int:
    return _bytes_of(load_library().iwdft_pages_plan_bytes, ctypes.byref(desc), n_layers, batch, n_tokens)


def iwdft_pages_attn_shared_bytes(desc: iwdft_pages_desc, n_layers: int, batch: int, n_tokens: int) -> int:
    return _bytes_of(load_library().iwdft_pages_attn_shared_bytes, ctypes.byref(desc), n_layers, batch, n_tokens)


def _raw(stream, index: int) -> int:
    """The call's stream, as a number that can be compared."""
    return torch._C._cuda_getCurrentRawStream(index) if stream is None else _stream(stream).value or 0


def _used_on(buffer, stream: int) -> None:
    """The memory of `buffer`, which its owner may drop at any time, is not given to anyone else before the work of that stream is done."""
    if not torch.cuda.is_current_stream_capturing():  # who replays a graph keeps what it reads
        buffer.record_stream(torch.cuda.ExternalStream(stream, buffer.device) if stream else torch.cuda.default_stream(buffer.device))


class PagesPlan:
    """Who shares what in a step: iwdft_pages_plan's buffer and what it was made for.  It may be dropped as soon as the last call that reads it has been made, on whatever
    stream that lives as long as it does; one that a captured graph reads is kept as long as the graph."""

    __slots__ = ("buffer", "n_layers", "n_tokens", "batch", "max_pages", "n_pages", "n_kv_heads", "n_q_heads", "page_tokens", "dtype", "n_sink", "n_recent", "stream")

    def __init__(self, buffer, made_for, stream):
        self.buffer, self.stream = buffer, stream  # whose order the buffer was allocated in
        (self.n_layers, self.n_tokens, self.batch, self.max_pages, self.n_pages, self.n_kv_heads, self.n_q_heads, self.page_tokens, self.dtype, self.n_sink,
         self.n_recent) = made_for

    def made_for(self):
        return (self.n_layers, self.n_tokens, self.batch, self.max_pages, self.n_pages, self.n_kv_heads, self.n_q_heads, self.page_tokens, self.dtype, self.n_sink,
                self.n_recent)


def iwdft_pages_plan(starts, table, lens, n_tokens: int, n_pages: int, n_kv_heads: int, n_q_heads: int, page_tokens: int, dtype: torch.dtype, n_layers: int = 1,
                     n_sink: int = 0, n_recent: int = 0, stream=None, plan: Optional[PagesPlan] = None) -> PagesPlan:
    """The plan of a step for iwdft_pages_attn_shared, whose calls have n_tokens rows and n_layers layers each; `plan`: an earlier one of these sizes and windows, made
    anew in its buffer (as a captured graph needs it)."""
    index, size = table.get_device(), table.shape
    if len(size) != 2 or index < 0:
        raise ValueError(f"table must be a device tensor [batch, max_pages], not {tuple(size)} on {table.device}")
    if not (starts.dtype is table.dtype is lens.dtype is torch.int32 and lens.shape == size[:1] and starts.shape == (size[0] + 1,)
            and index == starts.get_device() == lens.get_device() and starts.is_contiguous() and table.is_contiguous() and lens.is_contiguous()):
        for name, t, shape in (("table", table, size), ("starts", starts, (size[0] + 1,)), ("lens", lens, size[:1])):
            _expect(name, t, torch.int32, shape, table.device)
    if dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("dtype must be float32 or bfloat16")
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return iwdft_pages_plan(starts, table, lens, n_tokens, n_pages, n_kv_heads, n_q_heads, page_tokens, dtype, n_layers, n_sink, n_recent, stream, plan)
    batch, max_pages = size
    desc, need, _ = _shared_sizes(n_layers, batch, n_tokens, n_layers, n_pages, n_kv_heads, n_q_heads, 128, page_tokens, max_pages, dtype)
    made_for = (n_layers, n_tokens, batch, max_pages, n_pages, n_kv_heads, n_q_heads, page_tokens, dtype, n_sink, n_recent)
    if plan is None:
        plan = PagesPlan(_scratch(need, table.device, stream, None), made_for, _raw(stream, index))
    elif made_for != plan.made_for() or (need and plan.buffer.get_device() != index):
        raise ValueError(f"the plan was made for {dict(zip(PagesPlan.__slots__[1:-1], plan.made_for()))}, not {made_for}")
    buffer, on = plan.buffer, _raw(stream, index)
    if on != plan.stream and buffer is not None:
        _used_on(buffer, on)
    rc = load_library().iwdft_pages_plan(desc, n_layers, starts.data_ptr(), n_tokens, table.data_ptr(), lens.data_ptr(), batch, n_sink, n_recent,
                                         buffer.data_ptr() if buffer is not None else None, buffer.nbytes if buffer is not None else 0, on)
    if rc:
        _check(rc)
    return plan


def iwdft_pages_attn_shared(values, exponents, q, plan: PagesPlan, table, out, layer: int = 0, scale: float = 0.0, stream=None, workspace=None) -> None:
    """iwdft_pages_attn with pages that sequences share read once: q, out [layers, tokens, query heads, 128], as many layers and tokens as the plan was made for."""
    index, n_layers, n_pages, heads, P = _pool_sizes(values, exponents)
    dtype, shape = _kv_dtype("q", q), q.shape
    if not (shape == (plan.n_layers, plan.n_tokens, plan.n_q_heads, 128) and out.dtype is dtype is plan.dtype and shape == out.shape and table.dtype is torch.int32
            and table.shape == (plan.batch, plan.max_pages) and (n_pages, heads, P) == (plan.n_pages, plan.n_kv_heads, plan.page_tokens)
            and index == q.get_device() == out.get_device() == table.get_device() and (plan.buffer is None or plan.buffer.get_device() == index)
            and q.is_contiguous() and out.is_contiguous() and table.is_contiguous()):
        device = values.device
        _expect("q", q, plan.dtype, (plan.n_layers, plan.n_tokens, plan.n_q_heads, 128), device)
        _expect("out", out, dtype, shape, device)
        _expect("table", table, torch.int32, (plan.batch, plan.max_pages), device)
        raise ValueError(f"the plan was made for {plan.n_pages} pages of {plan.page_tokens} tokens and {plan.n_kv_heads} heads, not {tuple(values.shape)} on {device}")
    if index != torch._C._cuda_getDevice():
        with torch.cuda.device(index):
            return iwdft_pages_attn_shared(values, exponents, q, plan, table, out, layer, scale, stream, workspace)
    desc, _, need = _shared_sizes(plan.n_layers, plan.batch, plan.n_tokens, n_layers, n_pages, heads, plan.n_q_heads, 128, P, plan.max_pages, dtype)
    ws = _scratch(need, values.device, stream, workspace) if need or workspace is not None else None
    buffer, on = plan.buffer, _raw(stream, index)
    if on != plan.stream and buffer is not None:
        _used_on(buffer, on)
    rc = load_library().iwdft_pages_attn_shared(desc, layer, plan.n_layers, q.data_ptr(), plan.n_tokens, buffer.data_ptr() if buffer is not None else None,
                                                buffer.nbytes if buffer is not None else 0, table.data_ptr(), plan.batch, values.data_ptr(), exponents.data_ptr(),
                                                out.data_ptr(), plan.n_sink, plan.n_recent, scale, ws.data_ptr() if ws is not None else None,
                                                ws.nbytes if ws is not None else 0, on)
    if rc:
        _check(rc)


class PagedCache:
    """Owns the arrays of an 8-bit paged cache of up to max_batch sequences of max_tokens tokens; methods forward to the C calls.

    A step: ``starts, slots = resize(want, n)``, and for each layer ``write(k, v, slots, layer)`` and ``attend(q, starts, layer)``; a sequence
    that is to have 0 tokens gives its pages back.  ``compress`` hands what it holds to a frequency-domain cache.

    With ``shared`` sequences may hold the same pages: ``fork`` lets them begin as others do, ``resize`` copies a page that others hold before its sequence writes to it,
    ``plan`` finds out who shares what in a step, and ``attend`` with that plan reads shared pages once; ``compact`` and ``repool`` give memory back.
    Up to 1024 sequences then."""

    def __init__(self, n_layers, n_pages, n_kv_heads, n_q_heads, head_dim, dtype: torch.dtype, max_batch, max_tokens, page_tokens=32, device="cuda:0", shared=False):
        if dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("dtype must be float32 or bfloat16")
        self.dtype, self.device, self.page_tokens = dtype, torch.device(device), page_tokens
        max_pages = -(-max_tokens // max(page_tokens, 1))
        iwdft_pages_query_bytes(pages_desc(n_layers, n_pages, n_kv_heads, n_q_heads, head_dim, page_tokens, max_pages, dtype))  # checks the sizes
        self.shape = (n_layers, n_kv_heads, n_q_heads, head_dim)
        ints = dict(dtype=torch.int32, device=self.device)
        self.values = torch.zeros((n_layers, n_pages, n_kv_heads, 2, page_tokens * head_dim), dtype=torch.uint8, device=self.device)
        self.exponents = torch.zeros((n_layers, n_pages, n_kv_heads, 2), **ints)
        self.table = torch.full((max_batch, max_pages), -1, **ints)
        self.lens = torch.zeros(max_batch, **ints)
        self.free = torch.cat([torch.tensor([n_pages], **ints), torch.arange(n_pages, **ints)])
        if shared:
            iwdft_pages_fork_bytes(max_batch, max_pages)  # checks the sizes
        self.refs = torch.zeros(n_pages, **ints) if shared else None

    def _shares(self) -> None:
        if self.refs is None:
            raise ValueError("this cache was made without shared=True: a page belongs to one sequence")

    def resize(self, want: torch.Tensor, n_slots: int, stream=None):
        """want: int32 [max_batch] on the device.  Returns starts, slots; lens tells which sequences could not grow."""
        with _on_stream(stream, self.device):
            starts, slots = (torch.empty(n, dtype=torch.int32, device=self.device) for n in (self.lens.shape[0] + 1, n_slots))
            copies = None if self.refs is None else torch.empty((self.lens.shape[0], 2), dtype=torch.int32, device=self.device)
        if self.refs is None:
            iwdft_pages_resize(want, self.table, self.lens, self.free, starts, slots, self.page_tokens, stream)
        else:
            iwdft_pages_resize_shared(want, self.table, self.lens, self.free, self.refs, starts, slots, copies, self.page_tokens, stream)
            iwdft_pages_copy(copies, self.values, self.exponents, stream=stream)
        return starts, slots

    def fork(self, parent: torch.Tensor, keep: Optional[torch.Tensor] = None, stream=None) -> None:
        """parent, keep: int32 [max_batch] on the device.  Sequence b becomes the first keep[b] tokens (None, negative: all) of what sequence parent[b] was; b itself
        where parent[b] is b or negative.  Nothing is copied."""
        self._shares()
        iwdft_pages_fork(parent, keep, self.table, self.lens, self.free, self.refs, self.page_tokens, stream)

    def plan(self, starts, n_tokens: int, n_layers: int = 1, n_sink: int = 0, n_recent: int = 0, stream=None, plan: Optional[PagesPlan] = None) -> PagesPlan:
        """Who shares what, for the step's ``attend`` calls on n_layers layers and n_tokens rows each; valid until the tables change.  With `plan`, an earlier one of these sizes
        and windows, in its buffer; else in a new one: 15 bytes for each entry of the table and some 0.6 KB for each row."""
        L, H, G, _ = self.shape
        return iwdft_pages_plan(starts, self.table, self.lens, n_tokens, self.values.shape[1], H, G, self.page_tokens, self.dtype, n_layers, n_sink, n_recent, stream, plan)

    def compact(self, n_moves: Optional[int] = None, stream=None) -> torch.Tensor:
        """Moves held pages together at the pool's beginning, n_moves of them at most (None: all that have to).  Returns the moves, int32 [n_moves, 2]."""
        self._shares()
        most = self.values.shape[1] // 2
        with _on_stream(stream, self.device):
            moves = torch.empty((most if n_moves is None else n_moves, 2), dtype=torch.int32, device=self.device)
        iwdft_pages_compact(self.table, self.lens, self.free, self.refs, moves, self.page_tokens, stream)
        iwdft_pages_copy(moves[:most], self.values, self.exponents, stream=stream)  # the others are none
        return moves

    def repool(self, n_pages: int, stream=None) -> None:
        """The sequences in a pool of n_pages pages, larger or smaller; plans made before are void.  Needs both pools at a time, and waits for the stream: to learn how
        many pages are held, and before the old pool's memory is given back."""
        self._shares()
        L, H, G, D = self.shape
        iwdft_pages_query_bytes(pages_desc(L, n_pages, H, G, D, self.page_tokens, self.table.shape[1], self.dtype))
        with _on_stream(stream, self.device):
            held = self.values.shape[1] - int(self.free[0])
        if held > n_pages:
            raise ValueError(f"{held} pages are held, more than {n_pages}")
        self.compact(stream=stream)
        with _on_stream(stream, self.device):
            ints = dict(dtype=torch.int32, device=self.device)
            values = torch.zeros((L, n_pages, *self.values.shape[2:]), dtype=torch.uint8, device=self.device)
            exponents = torch.zeros((L, n_pages, H, 2), **ints)
            copies = torch.arange(held, **ints)[:, None].repeat(1, 2)
            refs, free = torch.zeros(n_pages, **ints), torch.zeros(1 + n_pages, **ints)
            refs[:held] = self.refs[:held]
            none = torch.empty((0, 2), **ints)
        iwdft_pages_copy(copies, self.values, self.exponents, values, exponents, stream=stream)
        iwdft_pages_compact(self.table, self.lens, free, refs, none, self.page_tokens, stream)  # nothing moves: the stack of the new pool
        with _on_stream(stream, self.device):
            torch.cuda.current_stream(self.device).synchronize()
        self.values, self.exponents, self.refs, self.free = values, exponents, refs, free

    def write(self, k, v, slots, layer=0, stream=None):
        iwdft_pages_write(self.values, self.exponents, k, v, slots, layer, stream)

    def attend(self, q, starts, layer=0, out=None, n_sink=0, n_recent=0, scale=0.0, stream=None, plan: Optional[PagesPlan] = None):
        """Without `out` a new tensor, which costs one more launch: rows behind the last sequence, which the attention leaves as they are, are 0 in it.  With a plan
        of this step shared pages are read once; windows are the plan's."""
        if out is None:
            with _on_stream(stream, self.device):
                out = torch.zeros_like(q)  # rows behind the last sequence
        if plan is not None:
            if (n_sink, n_recent) not in ((0, 0), (plan.n_sink, plan.n_recent)):
                raise ValueError(f"the plan was made for windows {(plan.n_sink, plan.n_recent)}, not {(n_sink, n_recent)}")
            iwdft_pages_attn_shared(self.values, self.exponents, q, plan, self.table, out, layer, scale, stream)
            return out
        iwdft_pages_attn(self.values, self.exponents, q, starts, self.table, self.lens, out, layer, n_sink, n_recent, scale, stream)
        return out

    def read(self, n_tokens, stream=None):
        """K, V of all layers, [layers, max_batch, KV heads, n_tokens, 128]."""
        L, H, _, D = self.shape
        with _on_stream(stream, self.device):
            K, V = (torch.empty((L, self.lens.shape[0], H, n_tokens, D), dtype=self.dtype, device=self.device) for _ in range(2))
        iwdft_pages_read(self.values, self.exponents, self.table, self.lens, K, V, 0, stream)
        return K, V

    def compress(self, cache: Cache, stream=None, sequences: Optional[Sequence[int]] = None):
        """The first S + M + R tokens of the given sequences through iwdft_prefill into `cache`, which has to have this cache's layers, heads and dtype and a
        batch of as many.  Tokens behind those stay here only: hand them to ``cache.append``, or give their pages back.  Returns by how many tokens each sequence is
        longer than S + M + R.

        The prefill knows no shorter sequences, it would take zeros for the tokens that are missing: a given sequence that has fewer is refused.  None stands for the
        whole batch as it is, idle places included: there they are zeros, a warning names the places, and what attends to them is worth nothing.  The lengths are read for all
        this, which waits for the stream.  While a graph is captured they cannot be: None is returned, and a given sequence that is too short at a replay becomes NaN."""
        device = self.values.device
        if device.index != torch.cuda.current_device():  # whose stream the prefill takes
            with torch.cuda.device(device):
                return self.compress(cache, stream, sequences)
        L, H, G, D = self.shape
        rows = list(range(self.lens.shape[0])) if sequences is None else [int(b) for b in sequences]
        if any(not 0 <= b < self.lens.shape[0] for b in rows):
            raise ValueError(f"sequences {rows} of {self.lens.shape[0]}")
        if cache.shape != (L, len(rows), H, G, D) or cache.dtype != self.dtype or cache.state.device != device:
            raise ValueError(f"cache holds {cache.shape} {cache.dtype} on {cache.state.device}, these pages {(L, len(rows), H, G, D)} {self.dtype} on {device}")
        d = cache.desc.c
        n = d.n_sink + d.M + d.n_recent
        with _on_stream(stream, self.device):
            table, lens = (self.table, self.lens) if sequences is None else (torch.cat([x[b:b + 1] for b in rows]) for x in (self.table, self.lens))
            captured = torch.cuda.is_current_stream_capturing()
            over = None if captured else [m - n for m in lens.tolist()]
            short = [b for b, m in zip(rows, over or []) if m < 0]
            if short and sequences is not None:
                raise ValueError(f"sequences {short} have fewer than {n} tokens")
            if short:
                warnings.warn(f"sequences {short} have fewer than {n} tokens: zeros are compressed in their place", stacklevel=2)
            K, V = (torch.empty((L, len(rows), H, n, D), dtype=self.dtype, device=self.device) for _ in range(2))
        iwdft_pages_read(self.values, self.exponents, table, lens, K, V, 0, stream)
        if captured and sequences is not None:
            with _on_stream(stream, self.device):
                for x in (K, V):
                    x[:, :, :, 0].masked_fill_((lens < n).view(-1, 1, 1), float("nan"))
        cache.prefill(K, V, stream)
        return over
