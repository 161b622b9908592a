"""fp64 CPU oracle of layer norm, counter-based dropout and the two joined.

TEST INFRASTRUCTURE ONLY, like the rest of this package.

The paper counts dropout and normalisation among the point-wise operations around
the convolutions (Sec. "Single GPU Performance").  On rows of C channels:
  layer norm   m = mean(x), v = mean((x - m)^2), r = 1 / sqrt(v + eps), y = (x - m) r gamma + beta
  dropout      y_i = residual_i + (u_i >= t ? 65536 / (65536 - t) x_i : 0),  t = rint(65536 p), with u_i the 16-bit
               field i % 8 of the Philox4x32-10 block of counter (i / 8, offset) under the key seed
  joined       s = residual + dropout(x), rounded to the storage type; y = layer norm of that
Gradients are written out term by term (the Jacobian applied row by row), not taken from the kernels' formula.
"""
from __future__ import annotations

import numpy as np


def philox4x32_10(counter, key) -> np.ndarray:
    """counter: [..., 4] and key: [2] 32-bit words -> [..., 4] words, round by round as published."""
    mask, c = (1 << 32) - 1, [np.asarray(counter, dtype=np.uint64)[..., j].copy() for j in range(4)]
    k = [int(key[0]), int(key[1])]
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        hi0, lo0 = p0 >> np.uint64(32), p0 & np.uint64(mask)
        hi1, lo1 = p1 >> np.uint64(32), p1 & np.uint64(mask)
        c = [hi1 ^ c[1] ^ np.uint64(k[0]), lo1, hi0 ^ c[3] ^ np.uint64(k[1]), lo0]
        k = [(k[0] + 0x9E3779B9) & mask, (k[1] + 0xBB67AE85) & mask]
    return np.stack(c, axis=-1)


def keep_mask(n: int, p: float, seed: int, offset: int, first: int = 0) -> np.ndarray:
    """Which of the elements first .. first + n - 1 are kept."""
    block = np.arange(first >> 3, (first + n + 7) >> 3, dtype=np.uint64)
    low = np.uint64((1 << 32) - 1)
    ctr = np.stack([block & low, block >> np.uint64(32), np.full_like(block, offset & int(low)),
                    np.full_like(block, (offset >> 32) & int(low))], axis=-1)
    w = philox4x32_10(ctr, (seed & int(low), seed >> 32))
    field = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], axis=-1).reshape(-1)      # low half of a word first
    return field[first & 7:(first & 7) + n] >= np.uint64(threshold(p))


def threshold(p: float) -> int:
    return int(np.rint(float(np.float32(p)) * 65536.0))


def dropout(x, p, seed, offset, residual=None, first: int = 0) -> np.ndarray:
    x = np.asarray(x, dtype=np.float64)
    t = threshold(p)
    scale = 65536.0 / (65536.0 - t) if t < 65536 else 0.0
    y = np.where(keep_mask(x.size, p, seed, offset, first).reshape(x.shape), x, 0.0) * scale
    return y if residual is None else y + np.asarray(residual, dtype=np.float64)


def layer_norm(x, gamma, beta, eps):
    """x [n, C] -> (y, mean [n], rstd [n])."""
    x = np.asarray(x, dtype=np.float64)
    m = x.mean(axis=1)
    r = 1.0 / np.sqrt(((x - m[:, None]) ** 2).mean(axis=1) + eps)
    y = (x - m[:, None]) * r[:, None]
    if gamma is not None:
        y = y * np.asarray(gamma, dtype=np.float64) + np.asarray(beta, dtype=np.float64)
    return y, m, r


def layer_norm_bwd(dy, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta): dy_c reaches x_j through d y_c / d x_j = gamma_c r (delta_cj - 1/C - h_c h_j / C)."""
    dy, x = np.asarray(dy, dtype=np.float64), np.asarray(x, dtype=np.float64)
    C = x.shape[1]
    r = np.asarray(rstd, dtype=np.float64)[:, None]
    h = (x - np.asarray(mean, dtype=np.float64)[:, None]) * r
    g = dy if gamma is None else dy * np.asarray(gamma, dtype=np.float64)
    dx = r * g - r * g.sum(axis=1, keepdims=True) / C - r * h * (g * h).sum(axis=1, keepdims=True) / C
    return dx, (dy * h).sum(axis=0), dy.sum(axis=0)


def joined_bwd(dy, ds, s, p, seed, offset, gamma, mean, rstd):
    """(dresidual, dx, dgamma, dbeta); p None: no dropout."""
    d, dgamma, dbeta = layer_norm_bwd(dy, s, gamma, mean, rstd)
    if ds is not None:
        d = d + np.asarray(ds, dtype=np.float64)
    return d, d if p is None else dropout(d, p, seed, offset), dgamma, dbeta
