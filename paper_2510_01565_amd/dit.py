"""Python binding of the C ABI in ``include/dit.h`` (ctypes; argument
marshalling only -- every step runs in the HIP library).

Device buffers are passed as torch tensors (their data pointers) or raw
integers; streams as torch streams, raw ``hipStream_t`` integers, or None for
torch's current stream.  The library must be built (``build.py``); importing
this module does not load it, the first call does, and fails loudly when the
shared library is missing.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence, Tuple

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdit_mi355x.so")

DIT_OK, DIT_ERR_INVALID_ARG, DIT_ERR_UNSUPPORTED, DIT_ERR_WORKSPACE, DIT_ERR_HIP = range(5)
DIT_F32, DIT_BF16 = 0, 1
DIT_MAX_REQUESTS = 16
DIT_MAX_GRID = 256
DIT_FLAG_BATCH_INVARIANT = 1
DIT_NOALLOC_SCRATCH_BYTES = 256 << 20
DIT_FP8_BLOCK = 128
DIT_SPARSE_QUERIES, DIT_SPARSE_KEYS, DIT_SPARSE_MAX_KEY_BLOCKS = 128, 64, 2048
DIT_SELECT_TEXT = 1
DIT_FP4_BLOCK = 32
DIT_ROPE_MAX_DIM = 256
DIT_ROPE_HALF, DIT_ROPE_PAIRS = 0, 1
DIT_MAX_SEQUENCES = 128
DIT_CAUSAL = 1

EXPORTED = ("dit_weight_count", "dit_weight_manifest", "dit_workspace_size", "dit_step", "dit_step_noalloc",
            "dit_block_forward", "euler_update", "dit_attention_workspace_size", "dit_attention", "dit_linear",
            "dit_fp8_layout", "dit_quantize_fp8", "dit_linear_fp8", "dit_attention_query_blocks",
            "dit_attention_select_workspace_size", "dit_attention_select", "dit_attention_sparse_workspace_size",
            "dit_attention_sparse", "dit_fp4_layout", "dit_quantize_fp4", "dit_dequantize_fp4", "dit_linear_fp4",
            "dit_rope_frequencies", "dit_rope", "dit_attention_grouped_workspace_size", "dit_attention_grouped",
            "dit_profile_start", "dit_profile_stop", "dit_profile_entry", "dit_last_error")


class DitError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"dit status {status}: {msg}")
        self.status = status


class dit_config(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int), ("heads", ctypes.c_int), ("head_dim", ctypes.c_int),
                ("mlp_ratio", ctypes.c_int), ("n_double", ctypes.c_int), ("n_single", ctypes.c_int),
                ("in_channels", ctypes.c_int), ("text_dim", ctypes.c_int), ("time_freq_dim", ctypes.c_int),
                ("tie_streams", ctypes.c_int), ("rope_theta", ctypes.c_float), ("ln_eps", ctypes.c_float),
                ("dtype", ctypes.c_int), ("flags", ctypes.c_int)]


class dit_batch(ctypes.Structure):
    _fields_ = [("n_req", ctypes.c_int), ("grid_h", ctypes.POINTER(ctypes.c_int)),
                ("grid_w", ctypes.POINTER(ctypes.c_int)), ("n_txt", ctypes.POINTER(ctypes.c_int)),
                ("t", ctypes.POINTER(ctypes.c_float))]


class dit_sequences(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int), ("q_len", ctypes.POINTER(ctypes.c_int)), ("kv_len", ctypes.POINTER(ctypes.c_int)),
                ("kv_row", ctypes.POINTER(ctypes.c_longlong))]


class dit_weights(ctypes.Structure):
    _fields_ = [("tensors", ctypes.POINTER(ctypes.c_void_p)), ("n_tensors", ctypes.c_int)]


_lib = None


def lib() -> ctypes.CDLL:
    """Loads the HIP library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"HIP library not built: {LIB_PATH} is missing (run paper_2510_01565_amd/build.py)")
        L = ctypes.CDLL(LIB_PATH)
        vp, ip, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        L.dit_last_error.restype = ctypes.c_char_p
        L.dit_weight_count.argtypes = [ctypes.POINTER(dit_config), ctypes.POINTER(ctypes.c_int)]
        L.dit_weight_manifest.argtypes = [ctypes.POINTER(dit_config), ip, ctypes.POINTER(ctypes.c_char_p),
                                          ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_int)]
        L.dit_workspace_size.argtypes = [ctypes.POINTER(dit_config), ctypes.POINTER(dit_batch),
                                         ctypes.POINTER(ctypes.c_size_t)]
        L.dit_step.argtypes = [ctypes.POINTER(dit_config), ctypes.POINTER(dit_weights), ctypes.POINTER(dit_batch),
                               vp, vp, vp, vp, sz, vp]
        L.dit_step_noalloc.argtypes = [ctypes.POINTER(dit_config), ctypes.POINTER(dit_weights),
                                       ctypes.POINTER(dit_batch), vp, vp, vp, vp]
        L.dit_block_forward.argtypes = [ctypes.POINTER(dit_config), ctypes.POINTER(dit_weights), ip, ip,
                                        ctypes.POINTER(dit_batch), vp, vp, vp, sz, vp]
        L.euler_update.argtypes = [ctypes.POINTER(dit_batch), ip, ip, vp, vp, ctypes.POINTER(ctypes.c_float), vp]
        L.dit_attention_workspace_size.argtypes = [ctypes.POINTER(dit_batch), ip, ip, ip,
                                                   ctypes.POINTER(ctypes.c_size_t)]
        L.dit_attention.argtypes = [ctypes.POINTER(dit_batch), ip, ip, ip, vp, vp, vp, vp, vp, sz, vp]
        L.dit_linear.argtypes = [ip, ip, ip, ip, vp, vp, vp, vp, ip, vp]
        bp, sp = ctypes.POINTER(dit_batch), ctypes.POINTER(ctypes.c_size_t)
        L.dit_fp8_layout.argtypes = [ip, ip, ip, sp, sp]
        L.dit_quantize_fp8.argtypes = [ip, ip, ip, ip, vp, vp, vp, vp]
        L.dit_linear_fp8.argtypes = [ip, ip, ip, vp, vp, vp, vp, vp, ip, vp, ip, vp]
        L.dit_attention_query_blocks.argtypes = [bp, ctypes.POINTER(ctypes.c_int)]
        L.dit_attention_select_workspace_size.argtypes = [bp, ip, ip, ip, sp]
        L.dit_attention_select.argtypes = [bp, ip, ip, ip, vp, vp, ip, ip, vp, vp, sz, vp]
        L.dit_attention_sparse_workspace_size.argtypes = [bp, ip, ip, ip, sp]
        L.dit_attention_sparse.argtypes = [bp, ip, ip, ip, vp, vp, vp, vp, ip, vp, vp, sz, vp]
        dbl, lng, flt, qp = ctypes.c_double, ctypes.c_long, ctypes.c_float, ctypes.POINTER(dit_sequences)
        L.dit_fp4_layout.argtypes = [ip, ip, sp, sp]
        L.dit_quantize_fp4.argtypes = [ip, ip, ip, vp, vp, vp, vp]
        L.dit_dequantize_fp4.argtypes = [ip, ip, vp, vp, ip, vp, vp]
        L.dit_linear_fp4.argtypes = [ip, ip, ip, vp, vp, vp, vp, vp, ip, vp, ip, vp]
        L.dit_rope_frequencies.argtypes = [ip, dbl, dbl, dbl, dbl, dbl, ctypes.POINTER(dbl)]
        L.dit_rope.argtypes = [ip, ip, ip, ip, ip, ip, vp, ctypes.POINTER(dbl), flt, vp, lng, vp, lng, vp]
        L.dit_attention_grouped_workspace_size.argtypes = [qp, ip, ip, ip, ip, sp]
        L.dit_attention_grouped.argtypes = [qp, ip, ip, ip, ip, ip, flt, vp, lng, vp, vp, lng, vp, lng, vp, sz, vp]
        L.dit_profile_start.argtypes = []
        L.dit_profile_stop.argtypes = [ctypes.POINTER(ctypes.c_int)]
        L.dit_profile_entry.argtypes = [ip, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_long),
                                        ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double),
                                        ctypes.POINTER(ctypes.c_double)]
        for name in EXPORTED:
            if name != "dit_last_error":
                getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _check(st: int) -> None:
    if st != DIT_OK:
        raise DitError(st, lib().dit_last_error().decode())


def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _stream(s) -> Optional[int]:
    if s is None:
        import torch
        # the raw handle: 0.3 us, where torch.cuda.current_stream() takes 2.7 to build its object, but no public name
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        return torch.cuda.current_stream().cuda_stream if raw is None else raw(torch.cuda.current_device())
    if isinstance(s, int):
        return s
    return s.cuda_stream


def make_config(shape, flags: int = 0) -> dit_config:
    """dit_config from a ``workloads.ModelShape``-like object; ``flags``: DIT_FLAG_* bits."""
    return dit_config(shape.hidden, shape.heads, shape.head_dim, shape.mlp_ratio, shape.n_double, shape.n_single,
                      shape.in_channels, shape.text_dim, shape.time_freq_dim, 1 if shape.tie_streams else 0,
                      float(shape.rope_theta), float(shape.ln_eps), DIT_BF16 if shape.dtype == "bf16" else DIT_F32,
                      flags)


class Batch:
    """Owns the host arrays of a dit_batch."""

    def __init__(self, grid_h: Sequence[int], grid_w: Sequence[int], n_txt: Sequence[int],
                 t: Optional[Sequence[float]] = None):
        n = len(grid_h)
        self.n = n
        self._gh = (ctypes.c_int * n)(*grid_h)
        self._gw = (ctypes.c_int * n)(*grid_w)
        self._nt = (ctypes.c_int * n)(*n_txt)
        self._t = (ctypes.c_float * n)(*t) if t is not None else None
        self.c = dit_batch(n, self._gh, self._gw, self._nt,
                           ctypes.cast(self._t, ctypes.POINTER(ctypes.c_float)) if self._t is not None else None)


class Weights:
    """Owns the pointer array of a dit_weights (tensors must stay alive)."""

    def __init__(self, tensors: Sequence):
        self.tensors = list(tensors)
        self._arr = (ctypes.c_void_p * len(tensors))(*[_ptr(t) for t in tensors])
        self.c = dit_weights(self._arr, len(tensors))


def weight_count(cfg: dit_config) -> int:
    n = ctypes.c_int()
    _check(lib().dit_weight_count(ctypes.byref(cfg), ctypes.byref(n)))
    return n.value


def weight_manifest(cfg: dit_config) -> List[Tuple[str, Tuple[int, ...]]]:
    out = []
    for i in range(weight_count(cfg)):
        name = ctypes.c_char_p()
        shape = (ctypes.c_int * 2)()
        nd = ctypes.c_int()
        _check(lib().dit_weight_manifest(ctypes.byref(cfg), i, ctypes.byref(name), shape, ctypes.byref(nd)))
        out.append((name.value.decode(), tuple(shape[:nd.value])))
    return out


def workspace_size(cfg: dit_config, batch: Batch) -> int:
    n = ctypes.c_size_t()
    _check(lib().dit_workspace_size(ctypes.byref(cfg), ctypes.byref(batch.c), ctypes.byref(n)))
    return n.value


def dit_step(cfg: dit_config, w: Weights, batch: Batch, latents, text_emb, velocity, ws, ws_bytes: int,
             stream=None) -> None:
    _check(lib().dit_step(ctypes.byref(cfg), ctypes.byref(w.c), ctypes.byref(batch.c), _ptr(latents),
                          _ptr(text_emb), _ptr(velocity), _ptr(ws), ws_bytes, _stream(stream)))


def dit_step_noalloc(cfg: dit_config, w: Weights, batch: Batch, latents, text_emb, velocity, stream=None) -> None:
    _check(lib().dit_step_noalloc(ctypes.byref(cfg), ctypes.byref(w.c), ctypes.byref(batch.c), _ptr(latents),
                                  _ptr(text_emb), _ptr(velocity), _stream(stream)))


def dit_block_forward(cfg: dit_config, w: Weights, kind: int, index: int, batch: Batch, hidden, cond, ws,
                      ws_bytes: int, stream=None) -> None:
    _check(lib().dit_block_forward(ctypes.byref(cfg), ctypes.byref(w.c), kind, index, ctypes.byref(batch.c),
                                   _ptr(hidden), _ptr(cond), _ptr(ws), ws_bytes, _stream(stream)))


def euler_update(batch: Batch, channels: int, dtype: int, latents, velocity, dt: Sequence[float],
                 stream=None) -> None:
    arr = (ctypes.c_float * len(dt))(*dt)
    _check(lib().euler_update(ctypes.byref(batch.c), channels, dtype, _ptr(latents), _ptr(velocity), arr,
                              _stream(stream)))


def attention_workspace_size(batch: Batch, heads: int, head_dim: int, dtype: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().dit_attention_workspace_size(ctypes.byref(batch.c), heads, head_dim, dtype, ctypes.byref(n)))
    return n.value


def dit_attention(batch: Batch, heads: int, head_dim: int, dtype: int, q, k, v, o, ws, ws_bytes: int,
                  stream=None) -> None:
    _check(lib().dit_attention(ctypes.byref(batch.c), heads, head_dim, dtype, _ptr(q), _ptr(k), _ptr(v), _ptr(o),
                               _ptr(ws), ws_bytes, _stream(stream)))


def dit_linear(M: int, N: int, K: int, dtype: int, x, w, b, y, out_dtype: int, stream=None) -> None:
    _check(lib().dit_linear(M, N, K, dtype, _ptr(x), _ptr(w), _ptr(b), _ptr(y), out_dtype, _stream(stream)))


def fp8_layout(rows: int, K: int, block_rows: int) -> Tuple[int, int]:
    """Bytes of the codes and of the scales of a [rows, K] 8-bit matrix."""
    c, s = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().dit_fp8_layout(rows, K, block_rows, ctypes.byref(c), ctypes.byref(s)))
    return c.value, s.value


def dit_quantize_fp8(rows: int, K: int, block_rows: int, dtype: int, x, codes, scales, stream=None) -> None:
    _check(lib().dit_quantize_fp8(rows, K, block_rows, dtype, _ptr(x), _ptr(codes), _ptr(scales), _stream(stream)))


def dit_linear_fp8(M: int, N: int, K: int, x_codes, x_scales, w_codes, w_scales, b, b_dtype: int, y, out_dtype: int,
                   stream=None) -> None:
    _check(lib().dit_linear_fp8(M, N, K, _ptr(x_codes), _ptr(x_scales), _ptr(w_codes), _ptr(w_scales), _ptr(b), b_dtype,
                                _ptr(y), out_dtype, _stream(stream)))


def attention_query_blocks(batch: Batch) -> int:
    """Query blocks of all requests: the second dimension of the lists of a block-sparse attention."""
    n = ctypes.c_int()
    _check(lib().dit_attention_query_blocks(ctypes.byref(batch.c), ctypes.byref(n)))
    return n.value


def attention_select_workspace_size(batch: Batch, heads: int, head_dim: int, dtype: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().dit_attention_select_workspace_size(ctypes.byref(batch.c), heads, head_dim, dtype, ctypes.byref(n)))
    return n.value


def dit_attention_select(batch: Batch, heads: int, head_dim: int, dtype: int, q, k, n_keep: int, flags: int, blocks, ws,
                         ws_bytes: int, stream=None) -> None:
    _check(lib().dit_attention_select(ctypes.byref(batch.c), heads, head_dim, dtype, _ptr(q), _ptr(k), n_keep, flags,
                                      _ptr(blocks), _ptr(ws), ws_bytes, _stream(stream)))


def attention_sparse_workspace_size(batch: Batch, heads: int, head_dim: int, dtype: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().dit_attention_sparse_workspace_size(ctypes.byref(batch.c), heads, head_dim, dtype, ctypes.byref(n)))
    return n.value


def dit_attention_sparse(batch: Batch, heads: int, head_dim: int, dtype: int, q, k, v, blocks, n_keep: int, o, ws,
                         ws_bytes: int, stream=None) -> None:
    _check(lib().dit_attention_sparse(ctypes.byref(batch.c), heads, head_dim, dtype, _ptr(q), _ptr(k), _ptr(v),
                                      _ptr(blocks), n_keep, _ptr(o), _ptr(ws), ws_bytes, _stream(stream)))


def fp4_layout(rows: int, K: int) -> Tuple[int, int]:
    """Bytes of the codes and of the scales of a [rows, K] 4-bit matrix."""
    c, s = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().dit_fp4_layout(rows, K, ctypes.byref(c), ctypes.byref(s)))
    return c.value, s.value


def dit_quantize_fp4(rows: int, K: int, dtype: int, x, codes, scales, stream=None) -> None:
    _check(lib().dit_quantize_fp4(rows, K, dtype, _ptr(x), _ptr(codes), _ptr(scales), _stream(stream)))


def dit_dequantize_fp4(rows: int, K: int, codes, scales, dtype: int, y, stream=None) -> None:
    _check(lib().dit_dequantize_fp4(rows, K, _ptr(codes), _ptr(scales), dtype, _ptr(y), _stream(stream)))


def dit_linear_fp4(M: int, N: int, K: int, x_codes, x_scales, w_codes, w_scales, b, b_dtype: int, y, out_dtype: int,
                   stream=None) -> None:
    _check(lib().dit_linear_fp4(M, N, K, _ptr(x_codes), _ptr(x_scales), _ptr(w_codes), _ptr(w_scales), _ptr(b), b_dtype,
                                _ptr(y), out_dtype, _stream(stream)))


def rope_frequencies(rot_dim: int, theta: float, factor: float = 1.0, original_len: Optional[float] = None,
                     low: Optional[float] = None, high: Optional[float] = None):
    """Host array of rot_dim / 2 angles per position (doubles), for ``dit_rope``.  A ``factor`` other than 1 needs the three
    behind it, which say what pairs it divides."""
    if factor != 1 and None in (original_len, low, high):
        raise ValueError(f"factor {factor} needs original_len, low and high")
    w = (ctypes.c_double * max(rot_dim // 2, 1))()
    _check(lib().dit_rope_frequencies(rot_dim, theta, factor, 1.0 if original_len is None else original_len,
                                      0.0 if low is None else low, 0.0 if high is None else high, w))
    return w


def dit_rope(rows: int, heads: int, head_dim: int, rot_dim: int, layout: int, dtype: int, positions, w, magnitude: float, x,
             ldx: int, y, ldy: int, stream=None) -> None:
    """``w``: what ``rope_frequencies`` returns, or a sequence of rot_dim / 2 numbers."""
    if w is not None and not isinstance(w, ctypes.Array):
        w = (ctypes.c_double * len(w))(*w)
    if w is not None and 2 * len(w) < rot_dim:
        raise ValueError(f"{len(w)} frequencies for {rot_dim} dimensions")
    _check(lib().dit_rope(rows, heads, head_dim, rot_dim, layout, dtype, _ptr(positions), w, magnitude, _ptr(x), ldx, _ptr(y),
                          ldy, _stream(stream)))


class Sequences:
    """Owns the host arrays of a dit_sequences."""

    def __init__(self, q_len: Sequence[int], kv_len: Sequence[int], kv_row: Optional[Sequence[int]] = None):
        n = len(q_len)
        if len(kv_len) != n or (kv_row is not None and len(kv_row) != n):
            raise ValueError("q_len, kv_len and kv_row must have one entry per sequence")
        self.n = n
        self._q = (ctypes.c_int * n)(*q_len)
        self._kv = (ctypes.c_int * n)(*kv_len)
        self._row = (ctypes.c_longlong * n)(*kv_row) if kv_row is not None else None
        self.c = dit_sequences(n, self._q, self._kv,
                               ctypes.cast(self._row, ctypes.POINTER(ctypes.c_longlong)) if self._row is not None else None)


def attention_grouped_workspace_size(seqs: Sequences, heads: int, kv_heads: int, head_dim: int, dtype: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().dit_attention_grouped_workspace_size(ctypes.byref(seqs.c), heads, kv_heads, head_dim, dtype, ctypes.byref(n)))
    return n.value


def dit_attention_grouped(seqs: Sequences, heads: int, kv_heads: int, head_dim: int, dtype: int, flags: int, scale: float, q,
                          ldq: int, k, v, ldkv: int, o, ldo: int, ws, ws_bytes: int, stream=None) -> None:
    _check(lib().dit_attention_grouped(ctypes.byref(seqs.c), heads, kv_heads, head_dim, dtype, flags, scale, _ptr(q), ldq,
                                       _ptr(k), _ptr(v), ldkv, _ptr(o), ldo, _ptr(ws), ws_bytes, _stream(stream)))


def profile_start() -> None:
    _check(lib().dit_profile_start())


def profile_stop() -> dict:
    """Stops kernel timing; returns {family: {launches, ms, flops, bytes}}."""
    n = ctypes.c_int()
    _check(lib().dit_profile_stop(ctypes.byref(n)))
    out = {}
    for i in range(n.value):
        name = ctypes.c_char_p()
        cnt = ctypes.c_long()
        ms, fl, by = ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
        _check(lib().dit_profile_entry(i, ctypes.byref(name), ctypes.byref(cnt), ctypes.byref(ms), ctypes.byref(fl),
                                       ctypes.byref(by)))
        out[name.value.decode()] = {"launches": cnt.value, "ms": ms.value, "flops": fl.value, "bytes": by.value}
    return out
