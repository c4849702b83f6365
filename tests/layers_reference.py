"""Plain implementations in 64 bits (numpy) of the layers in front of a loss, and bounds on how far sums of 16-bit products in fp32 may be from them."""
from __future__ import annotations

import math

import numpy as np

NONE, RELU, GELU, SILU = 0, 1, 2, 3
C = math.sqrt(2.0 / math.pi)


def _sigmoid(x):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-x))


def act(z, kind):
    if kind == RELU:
        return np.where(z < 0, 0.0, z)
    if kind in (GELU, SILU):
        s = _sigmoid(2 * C * (z + 0.044715 * z ** 3) if kind == GELU else z)
        with np.errstate(invalid="ignore"):
            return np.where(s == 0, 0.0, z * s)
    return z


def slope(z, kind):
    if kind == RELU:
        return np.where(np.isnan(z), np.nan, (z > 0).astype(float))
    if kind in (GELU, SILU):
        s = _sigmoid(2 * C * (z + 0.044715 * z ** 3) if kind == GELU else z)
        inner = 2 * C * (1 + 3 * 0.044715 * z * z) if kind == GELU else 1.0
        with np.errstate(invalid="ignore"):
            return np.where(s * (1 - s) == 0, s, s + z * s * (1 - s) * inner)
    return np.ones_like(z)


def linear(x, w, bias=None, residual=None, kind=NONE):
    """(out, z) in float64."""
    z = x @ w.T
    if bias is not None:
        z = z + bias
    y = act(z, kind)
    return (y if residual is None else y + residual), z


def linear_grad(dy, x, w, z=None, kind=NONE):
    """(dx, dw, db) in float64."""
    dz = dy if kind == NONE else dy * slope(z, kind)
    return dz @ w, dz.T @ x, dz.sum(0)


def xent(x, w, target, weight=None):
    """(loss, lse, dx, dw, G) in float64; rows without a target or of weight 0 do not count, whatever they hold."""
    rows, vocab = len(x), len(w)
    weight = np.ones(rows) if weight is None else weight.astype(np.float64)
    live = (target >= 0) & (target < vocab) & (weight != 0)
    loss, lse, G = np.zeros(rows), np.zeros(rows), np.zeros((rows, vocab))
    for r in np.nonzero(live)[0]:
        z = w @ x[r]
        m = z.max()
        lse[r] = m + math.log(np.exp(z - m).sum())
        loss[r] = weight[r] * (lse[r] - z[target[r]])
        G[r] = weight[r] * np.exp(z - lse[r])
        G[r, target[r]] = weight[r] * math.expm1(z[target[r]] - lse[r])
    return loss, lse, G @ w, G.T @ np.where(live[:, None], x, 0.0), G


def philox(block, offset, seed):
    """The four words of a block, by Python's whole numbers."""
    c = [block & 0xFFFFFFFF, block >> 32, offset & 0xFFFFFFFF, offset >> 32]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(q >> 32) ^ c[1] ^ k[0], q & 0xFFFFFFFF, (p >> 32) ^ c[3] ^ k[1], p & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(n, p, seed, offset):
    """(which of n elements are kept, what they are multiplied by)."""
    border = math.floor(65536 * p + 0.5)
    words = [w for b in range(-(-n // 8)) for w in philox(b, offset, seed)]
    halves = np.array([h for w in words for h in (w & 0xFFFF, w >> 16)][:n], dtype=np.int64)
    return halves >= border, 0.0 if border == 65536 else 65536.0 / (65536 - border)
