"""Error bounds of the layer norm and dropout kernels against the fp64 oracle, term by term from the rounding of fp32
arithmetic and of the storage type."""
from __future__ import annotations

import numpy as np
import torch

from oracle import norm as N

DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
HALF = {k: torch.finfo(t).eps / 2 for k, t in DT.items()}              # half a step, relative
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134, "f32": 2.0 ** -150}    # half a step below the smallest normal number
U32 = 2.0 ** -24


def chain(C: int) -> float:
    """Roundings on the longest way through a sum over C channels: at most 32 serial terms or C / 64 of them in a thread, then
    a tree; 64 leaves room for both and for the division."""
    return 64.0 + C / 64


def chain_rows(n: int) -> float:
    """The same for a sum over n pixels: n / 256 serial terms at most where a workgroup has a row at a time, a tree, and up to
    1024 slabs."""
    return 1100.0 + n / 256


def f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().double().cpu().numpy()


def assert_within(got: torch.Tensor, ref: np.ndarray, bound: np.ndarray, what: str):
    err = np.abs(f64(got).reshape(ref.shape) - ref)
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(err / np.maximum(bound, 1e-300)):.3g} bounds"


def check_forward(x, gamma, beta, eps, y, mean, rstd, dtype):
    """x, y: [n, C] tensors as stored."""
    xs = f64(x)
    C = xs.shape[1]
    g = None if gamma is None else f64(gamma)
    ry, rm, rr = N.layer_norm(xs, g, None if beta is None else f64(beta), float(np.float32(eps)))
    K = chain(C)
    d = xs - rm[:, None]
    v = (d * d).mean(axis=1)
    em = K * U32 * np.abs(xs).mean(axis=1)
    ev = (K + 4) * U32 * v + 2 * em * np.abs(d).mean(axis=1) + em * em
    er = ev / (2 * (v + float(np.float32(eps)))) + 3 * U32             # relative error of 1/sqrt(v + eps)
    if mean is not None:
        assert_within(mean, rm, em + 1e-40, "mean")
        assert_within(rstd, rr, 1.01 * er * rr, "rstd")
    ag = np.ones(C) if g is None else np.abs(g)
    h = np.abs(d) * rr[:, None]
    bound = ag * (1.01 * rr[:, None] * em[:, None] + h * (1.01 * er[:, None] + 4 * U32)) + 2 * U32 * (ag * h + np.abs(ry)) + \
        1.01 * HALF[dtype] * np.abs(ry) + TINY[dtype]
    assert_within(y, ry, bound, "y")


def check_backward(dy, s, gamma, mean, rstd, dx, dgamma, dbeta, dtype, ds=None, drop=None, dropped=None):
    """dx: gradient of s (with ds added if given); dropped: (p, seed, offset) of its masked copy, drop."""
    gy, xs, m, r = f64(dy), f64(s), f64(mean).reshape(-1), f64(rstd).reshape(-1)
    n, C = gy.shape
    gm = None if gamma is None else f64(gamma)
    ref, rdg, rdb = N.layer_norm_bwd(gy, xs, gm, m, r)
    K = chain(C)
    g = gy if gm is None else gy * gm
    h = (xs - m[:, None]) * r[:, None]
    ma, mb = np.abs(g).mean(axis=1)[:, None], np.abs(g * h).mean(axis=1)[:, None]
    a, b = np.abs(g.mean(axis=1))[:, None], np.abs((g * h).mean(axis=1))[:, None]
    e = r[:, None] * (U32 * np.abs(g) + (K + 2) * U32 * ma + np.abs(h) * (K + 8) * U32 * mb +
                      6 * U32 * (np.abs(g) + a + np.abs(h) * b))
    if ds is not None:
        ref = ref + f64(ds)
        e = e + U32 * np.abs(ref)
    if dx is not None:
        assert_within(dx, ref, e + 1.01 * HALF[dtype] * np.abs(ref) + TINY[dtype], "dx")
    if drop is not None:
        p, seed, off = dropped
        t = N.threshold(p)
        scale = 65536 / (65536 - t) if t < 65536 else 0.0
        rd = N.dropout(ref, p, seed, off)
        assert_within(drop, rd, np.where(rd != 0, scale * e, 0) + (2 * U32 + 1.01 * HALF[dtype]) * np.abs(rd) + TINY[dtype], "dropped")
    if dgamma is not None:
        Kn = chain_rows(n)
        assert_within(dgamma, rdg, (Kn + 4) * U32 * np.abs(gy * h).sum(axis=0) + 1e-40, "dgamma")
        assert_within(dbeta, rdb, Kn * U32 * np.abs(gy).sum(axis=0) + 1e-40, "dbeta")


def check_dropout(x, p, seed, offset, residual, y, dtype, first=0):
    xs = f64(x)
    res = None if residual is None else f64(residual)
    ref = N.dropout(xs, p, seed, offset, res, first)
    t = N.threshold(p)
    scale = 65536 / (65536 - t) if t < 65536 else 0.0
    keep = N.keep_mask(xs.size, p, seed, offset, first).reshape(xs.shape)
    part = np.where(keep, np.abs(xs), 0) * scale
    bound = 3 * U32 * part + 1.01 * HALF[dtype] * np.abs(ref) + TINY[dtype] + (0 if res is None else U32 * np.abs(ref))
    assert_within(y, ref, np.where(keep, bound, 0), "dropout")         # what is dropped leaves the residual as it is
