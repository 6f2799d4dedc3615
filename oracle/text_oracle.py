"""Plain 64-bit reference of the 4-bit matrices, the rotary positions and the grouped attention (NumPy).

Written from the definitions in ``include/dit.h``; shares no code with the kernels."""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def round_e2m1(v):
    """Codes 0..7 of the e2m1 values nearest to |v|, ties to the even code."""
    a = np.abs(np.asarray(v, np.float64))
    mid = (E2M1[1:] + E2M1[:-1]) / 2
    n = np.zeros(a.shape, np.uint8)
    for i, m in enumerate(mid, 1):  # between codes i - 1 and i
        n[(a > m) | ((a == m) & (i % 2 == 0))] = i
    return n


def quantize_fp4(x):
    """Codes [rows, 128 ceil(K / 256)] and scale bytes [rows, 16 ceil(K / 512)] of x [rows, K]."""
    x = np.asarray(x, np.float64)
    rows, K = x.shape
    nb = -(-K // BLOCK)
    t = np.zeros((rows, nb * BLOCK))
    t[:, :K] = x
    t = t.reshape(rows, nb, BLOCK)
    bad = ~np.isfinite(t).all(axis=2)
    a = np.where(bad, 0.0, np.abs(np.where(np.isfinite(t), t, 0.0)).max(axis=2))
    byte = np.full((rows, nb), 127)
    for i in np.ndindex(a.shape):
        if a[i] > 0:
            e = -127
            while 6.0 * 2.0 ** e < a[i]:
                e += 1
            byte[i] = e + 127
    byte[bad] = 255
    v = np.where(bad[:, :, None], 0.0, t) / 2.0 ** (np.where(bad, 127, byte)[:, :, None] - 127.0)
    n = round_e2m1(v) | (np.signbit(v).astype(np.uint8) << 3)
    flat = np.zeros((rows, -(-K // 256) * 256), np.uint8)
    flat[:, :nb * BLOCK] = n.reshape(rows, -1)
    flat[:, K:] = 0
    s = np.full((rows, -(-K // 512) * 16), 127, np.uint8)
    for b in range(nb):
        s[:, scale_place(b)] = byte[:, b]
    return flat[:, 0::2] | flat[:, 1::2] << 4, s


def scale_place(b):
    """Byte of a row's scales that belongs to its block b."""
    return b // 16 * 16 + b % 4 * 4 + b // 4 % 4


def dequantize_fp4(codes, scales, K):
    n = np.stack([codes & 15, codes >> 4], axis=2).reshape(codes.shape[0], -1)[:, :K]
    v = np.where(n >= 8, -1.0, 1.0) * E2M1[n & 7]
    byte = scales[:, [scale_place(k // BLOCK) for k in range(K)]].astype(np.float64)
    return v * np.where(byte == 255, np.nan, 2.0 ** (np.where(byte == 255, 127, byte) - 127.0))


def rope(x, pos, w, layout, magnitude=1.0):
    """x [rows, heads, d] with its first 2 len(w) dimensions turned; layout "half" or "pairs"."""
    y = np.array(x, np.float64)
    n = len(w)
    ang = np.asarray(pos, np.float64)[:, None] * np.asarray(w, np.float64)
    c, s = magnitude * np.cos(ang), magnitude * np.sin(ang)
    for i in range(n):
        ia, ib = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
        a, b = np.array(x[:, :, ia], np.float64), np.array(x[:, :, ib], np.float64)
        y[:, :, ia] = a * c[:, None, i] - b * s[:, None, i]
        y[:, :, ib] = a * s[:, None, i] + b * c[:, None, i]
    return y


def grouped_attention(q, k, v, q_len, kv_len, kv_row, scale, causal):
    """o [queries, heads, d] and, for error bounds, the same with |v| in v's place."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    heads, group = q.shape[1], q.shape[1] // k.shape[1]
    o, mag = np.zeros(q.shape), np.zeros(q.shape)
    at = 0
    for n, m, f in zip(q_len, kv_len, kv_row):
        for h in range(heads):
            kh, vh = k[f:f + m, h // group], v[f:f + m, h // group]
            for i in range(n):
                seen = min(m, max(0, m - n + i + 1)) if causal else m
                if seen == 0:
                    continue
                s = scale * (kh[:seen] @ q[at + i, h])
                p = np.exp(s - s.max())
                p /= p.sum()
                o[at + i, h], mag[at + i, h] = p @ vh[:seen], p @ np.abs(vh[:seen])
        at += n
    return o, mag
