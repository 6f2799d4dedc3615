"""fp64 reference of the 8-bit products and of the block-sparse attention
(NumPy; used by tests only, shares no code with the HIP path)."""
from __future__ import annotations

from typing import List, Optional, Sequence

import numpy as np

FP8_MAX = 448.0
BLOCK = 128
QUERIES, KEYS = 128, 64


# ---------------------------------------------------------------- e4m3
def e4m3_values() -> np.ndarray:
    """The value of each of the 256 codes: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        if c & 0x7f == 0x7f:
            v = np.nan
        out[c] = -v if c & 0x80 else v
    return out


def e4m3_encode(v: np.ndarray) -> np.ndarray:
    """Codes of the nearest values, ties to the even mantissa, of |v| <= 448; NaN and infinities to 0x7f (sign dropped)."""
    pos = e4m3_values()[:127]
    a = np.abs(np.where(np.isfinite(v), v, 0.0))
    assert a.size == 0 or a.max() <= FP8_MAX
    hi = np.searchsorted(pos, a)                      # pos[hi - 1] < a <= pos[hi]
    lo = np.maximum(hi - 1, 0)
    up = (pos[hi] - a < a - pos[lo]) | ((pos[hi] - a == a - pos[lo]) & (hi % 2 == 0))
    c = np.where(up | (hi == 0), hi, lo) | np.where(np.signbit(v), 0x80, 0)
    return np.where(np.isfinite(v), c, 0x7f).astype(np.uint8)


def scale_exponent(a: float) -> int:
    """The smallest e >= -127 with a <= 448 * 2^e; 0 for a = 0."""
    if a == 0:
        return 0
    e = -127
    while a > FP8_MAX * 2.0 ** e:
        e += 1
    return e


def quantize_fp8(x: np.ndarray, block_rows: int):
    """Codes [rows, K up to 128] and scale bytes [row blocks, K blocks up to 4] of x [rows, K] (fp64 of what is stored)."""
    rows, K = x.shape
    kb, rb = -(-K // BLOCK), -(-rows // block_rows)
    q = np.zeros((rows, kb * BLOCK), np.uint8)
    s = np.full((rb, -(-kb // 4) * 4), 127, np.uint8)
    for i in range(rb):
        r = slice(i * block_rows, min(rows, (i + 1) * block_rows))
        for j in range(kb):
            c = slice(j * BLOCK, min(K, (j + 1) * BLOCK))
            t = x[r, c]
            fin = np.abs(t[np.isfinite(t)])
            e = scale_exponent(float(fin.max()) if fin.size else 0.0)
            with np.errstate(invalid="ignore"):
                q[r, c] = e4m3_encode(t / 2.0 ** e)
            s[i, j] = e + 127
    return q, s


def dequantize_fp8(q: np.ndarray, s: np.ndarray, block_rows: int, K: int) -> np.ndarray:
    scale = np.repeat(np.repeat(2.0 ** (s.astype(np.float64) - 127), block_rows, 0), BLOCK, 1)
    return (e4m3_values()[q] * scale[: q.shape[0], : q.shape[1]])[:, :K]


# ---------------------------------------------------------------- block-sparse attention
def block_means(x: np.ndarray, n: int) -> np.ndarray:
    """Means of every n tokens of x [L, heads, d]: [heads, blocks, d]."""
    return np.stack([x[i:i + n].mean(0) for i in range(0, x.shape[0], n)], 1)


def select_blocks(q: np.ndarray, k: np.ndarray, n_keep: int, n_text: int = 0) -> np.ndarray:
    """Lists [heads, query blocks, n_keep] of one request, q and k [L, heads, d]; the blocks of n_text leading tokens first."""
    s = np.matmul(block_means(q, QUERIES), block_means(k, KEYS).transpose(0, 2, 1))
    n = s.shape[2]
    out = np.full(s.shape[:2] + (n_keep,), -1, np.int32)
    text = -(-n_text // KEYS)
    for h in range(s.shape[0]):
        for i in range(s.shape[1]):
            # rank: text blocks, NaN, then descending; Python's sort keeps the lower index first
            rank = sorted(range(n), key=lambda j: (0, 0) if j < text else (1, 0) if np.isnan(s[h, i, j]) else (2, -s[h, i, j]))
            best = sorted(rank[:n_keep])
            out[h, i, : len(best)] = best
    return out


def sparse_attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, blocks: np.ndarray, mag: bool = False):
    """O [L, heads, d] of one request; blocks [heads, query blocks, n].  mag: also sum_j p_j |v_j|, the scale of its errors."""
    L, heads, d = q.shape
    o, g = np.zeros(q.shape), np.zeros(q.shape)
    nk = -(-L // KEYS)
    for h in range(heads):
        for i in range(-(-L // QUERIES)):
            rows = slice(i * QUERIES, min(L, (i + 1) * QUERIES))
            keys: List[int] = []
            for b in sorted({int(x) for x in blocks[h, i] if 0 <= x < nk}):
                keys += range(b * KEYS, min(L, (b + 1) * KEYS))
            if not keys:
                continue
            s = q[rows, h] @ k[keys, h].T / np.sqrt(d)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            o[rows, h] = p @ v[keys, h]
            g[rows, h] = p @ np.abs(v[keys, h])
    return (o, g) if mag else o
