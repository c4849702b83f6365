"""Plain implementations in 64 bits (numpy) of the operators beside a round, for the tests to compare with."""
from __future__ import annotations

import math

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def bits_to_float(a):
    """float64 values of a float32, float16 or (as uint16 patterns) bfloat16 array."""
    if a.dtype == np.uint16:
        return (a.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    return a.astype(np.float64)


def mx4_block(v):
    """(codes [32] as integers 0..15, scale byte) of 32 float64 values, by the definition: the nearest of the eight magnitudes,
    of two equally near ones the even code."""
    a = np.max(np.abs(v))
    if not np.isfinite(a):
        return np.zeros(32, dtype=np.int64), 255
    if a == 0.0:
        return np.where(np.signbit(v), 8, 0), 0
    e = max(math.frexp(a)[1] - 1 - 2, -127)
    y = np.abs(v) * 2.0 ** -e
    d = np.abs(y[:, None] - MAGNITUDES[None, :])
    near = d == d.min(axis=1, keepdims=True)
    codes = np.empty(32, dtype=np.int64)
    for i in range(32):
        c = np.nonzero(near[i])[0]
        codes[i] = c[0] if len(c) == 1 or c[0] % 2 == 0 else c[1]
    return codes + 8 * np.signbit(v), e + 127


def mx4_quantise(x):
    """x float64 [R, C] -> (codes int [R, 128 W], bytes int [R, 4 W])."""
    rows, cols = x.shape
    words = -(-cols // 128)
    full = np.zeros((rows, 128 * words))
    full[:, :cols] = x
    codes = np.zeros((rows, 128 * words), dtype=np.int64)
    byte = np.zeros((rows, 4 * words), dtype=np.int64)
    for r in range(rows):
        for b in range(4 * words):
            codes[r, 32 * b:32 * b + 32], byte[r, b] = mx4_block(full[r, 32 * b:32 * b + 32])
    return codes, byte


def mx4_values(codes, byte):
    """What codes [R, 128 W] and bytes [R, 4 W] stand for, float64."""
    v = np.where(codes >= 8, -1.0, 1.0) * MAGNITUDES[codes & 7]
    scale = np.where(byte == 255, np.nan, np.ldexp(1.0, np.where(byte == 255, 0, byte) - 127))
    return v * np.repeat(scale, 32, axis=1)


def mx4_pack(codes, byte):
    """The stored form: uint8 [R, 64 W], uint32 [W, R]."""
    rows, blocks = byte.shape
    b = byte.astype(np.uint32).reshape(rows, blocks // 4, 4)
    words = b[..., 0] | b[..., 1] << 8 | b[..., 2] << 16 | b[..., 3] << 24
    return (codes[:, 0::2] | codes[:, 1::2] << 4).astype(np.uint8), np.ascontiguousarray(words.T)


def mx4_unpack(packed, words):
    """The stored form -> (codes, bytes)."""
    rows = packed.shape[0]
    codes = np.empty((rows, 2 * packed.shape[1]), dtype=np.int64)
    codes[:, 0::2], codes[:, 1::2] = packed & 15, packed >> 4
    byte = (words.T[:, :, None] >> np.array([0, 8, 16, 24], dtype=np.uint32)) & 255
    return codes, byte.reshape(rows, -1).astype(np.int64)


def without_minus_zero(codes):
    """Codes with the sign of zero taken off (both zeros are the same value)."""
    return np.where(codes == 8, 0, codes)


def update(g, h, starts):
    """(codes, bytes of all words, new h) of one worker's update; g, h float32."""
    L, d = len(starts) - 1, len(g)
    words = d // 128 + L
    codes = np.zeros((words, 128), dtype=np.int64)
    byte = np.zeros((words, 4), dtype=np.int64)
    h = h.copy()
    for i in range(L):
        lo, hi = int(starts[i]), int(starts[i + 1])
        if lo == hi:
            continue
        with np.errstate(all="ignore"):
            x = (g[lo:hi] - h[lo:hi]).astype(np.float64)
        c, b = mx4_quantise(x[None, :])
        w0, n = lo // 128 + i, c.shape[1] // 128
        codes[w0:w0 + n], byte[w0:w0 + n] = c.reshape(n, 128), b.reshape(n, 4)
        with np.errstate(all="ignore"):
            h[lo:hi] = h[lo:hi] + mx4_values(c, b)[0, :hi - lo].astype(np.float32)
    return codes, byte, h


def decode_update(codes, byte, starts):
    """The update as a flat float64 vector."""
    v = mx4_values(codes, byte).reshape(-1)
    return np.concatenate([v[128 * (int(lo) // 128 + i):][:int(hi - lo)] for i, (lo, hi) in enumerate(zip(starts[:-1], starts[1:]))])


def distill(z, idx, t, T, w):
    """(loss [R], stats [R, 2], grad [R, V]) in float64; z [R, V], idx int [R, k] (entries outside 0..V-1 are none), t [R, k]."""
    rows, vocab = z.shape
    loss, stats, grad = np.zeros(rows), np.zeros((rows, 2)), np.zeros((rows, vocab))
    with np.errstate(all="ignore"):
        for r in range(rows):
            there = (idx[r] >= 0) & (idx[r] < vocab)
            tv = t[r][there].astype(np.float64)
            if w[r] == 0 or not np.any(tv != -np.inf) or not np.any(z[r] != -np.inf):
                continue
            e = np.exp((tv - np.max(tv)) / T)
            p = np.zeros(vocab)
            np.add.at(p, idx[r][there], e / e.sum())
            m = np.fmax.reduce(z[r])
            s = np.exp((z[r] - m) / T)
            q = s / s.sum()
            on = p != 0
            loss[r] = w[r] * T * T * np.sum(p[on] * (np.log(p[on]) - ((z[r][on] - m) / T - np.log(s.sum()))))
            stats[r] = m, s.sum()
            grad[r] = w[r] * T * (q - p)
    return loss, stats, grad
