"""GPU: layer norm of rows whose mean lies far above their spread.  Rows of equal values give their value and beta to the bit; other
rows lose no digits but those that the stored mean's own rounding takes."""
import numpy as np
import pytest
import torch

from oracle import norm as N

import norm_util as M

pytestmark = pytest.mark.gpu
DTYPES = ["f16", "bf16", "f32"]
# rows of one lane to a whole wave, whole pieces and odd ones, rows that waves share, rows beyond the registers (from 8193 fp32 or 16385
# 16-bit channels on)
CHANNELS = [1, 3, 7, 8, 24, 77, 208, 240, 304, 328, 513, 771, 1000, 1544, 2047, 3000, 4099, 8192, 9000, 12295, 16384, 16400, 20001]


@pytest.fixture(scope="module")
def api():
    from paper_1810_01993_amd import api as _api
    assert torch.cuda.is_available()
    return _api


def _vec(C, seed, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return mean + 0.3 * torch.randn(C, generator=g, device="cuda")


def _equal_rows(C, dtype):
    """Saturated and constant pixels: whole numbers (their sums are whole too), and fp32 values whose sums round."""
    v = torch.tensor([10000.0, 1000.0, 4096.0, 1.0, -2047.0, 0.0, 1000.1, 0.1, -333.3, 3e4, 1 / 3, -7e-3], device="cuda")
    return v.to(M.DT[dtype])[:, None].expand(-1, C).contiguous()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", CHANNELS)
def test_rows_of_equal_values(api, C, dtype):
    """mean is the value, y is beta, no gradient reaches gamma.  (The first mean is off by k steps of the value, k some tens at most:
    each deviation is that number of steps exactly, their sum a whole number of steps below 2^24, and its quotient by C exact.)"""
    print(f"[case] equal rows C={C} {dtype}", flush=True)
    x, eps = _equal_rows(C, dtype), 1e-5
    gamma, beta = _vec(C, 1, 1.0), _vec(C, 2)
    want = beta.to(M.DT[dtype]).expand(x.shape)

    def check(y, m, r):
        assert torch.equal(m, x[:, 0].float())
        assert torch.equal(y, want)
        # the deviations' square sum is at most (64 steps)^2, off by at most 64 roundings of it: seen against eps
        step = 2 * M.U32 * np.abs(M.f64(m))
        ref = np.full(len(step), float(np.float32(eps)) ** -0.5)
        M.assert_within(r, ref, ref * (4 * M.U32 + 64 * M.U32 * (64 * step) ** 2 / eps), "rstd")
    y, m, r = api.layer_norm_fwd(x, gamma, beta, eps)
    check(y, m, r)
    _, dgamma, _ = api.layer_norm_bwd(torch.ones_like(x), x, gamma, m, r)
    assert not dgamma.any()
    for residual, p in ((None, None), (torch.zeros_like(x), 0.0)):
        s, y, m, r = api.dropout_add_layer_norm_fwd(x, residual, None if p is None else api.DropoutDesc(p, 1), gamma, beta, eps)
        assert torch.equal(s, x)
        check(y, m, r)


@pytest.mark.parametrize("mean,spread", [(300.0, 1.0), (1e4, 1.0), (-1e4, 0.1), (1000.0, 30.0), (0.5, 1.0), (1.0, 1e-3)])
@pytest.mark.parametrize("C", CHANNELS[1:])
def test_means_far_above_the_spread(api, C, mean, spread):
    """fp32 rows.  With D = |x - m| + e0, e0 the first mean's error (K roundings of mean|x|), the deviations from it are rounded once
    (2^-24 D), their sum to K roundings of mean D, and the corrected deviation once more:
      mean   2^-24 |m| + (K + 3) 2^-24 mean D
      x - m  2^-24 (2 D + (K + 3) mean D)
      var    (K + 6) 2^-24 mean D^2 + 2 (K + 4) 2^-24 mean D (e0 + K 2^-24 mean D)"""
    print(f"[case] far means C={C} mean={mean} spread={spread}", flush=True)
    n, eps, U = 9, 1e-5, M.U32
    g = torch.Generator(device="cuda").manual_seed(C)
    x = torch.randn((n, C), generator=g, device="cuda") * spread + mean
    gamma, beta = _vec(C, 1, 1.0), _vec(C, 2)
    y, m, r = api.layer_norm_fwd(x, gamma, beta, eps)
    xs, gm = M.f64(x), M.f64(gamma)
    e32 = float(np.float32(eps))
    ry, rm, rr = N.layer_norm(xs, gm, M.f64(beta), e32)
    K = M.chain(C)
    e0 = K * U * np.abs(xs).mean(axis=1)[:, None]
    d = np.abs(xs - rm[:, None])
    D = d + e0
    mD = D.mean(axis=1)[:, None]
    ev = (K + 6) * U * (D * D).mean(axis=1)[:, None] + 2 * (K + 4) * U * mD * (e0 + K * U * mD)
    v = (d * d).mean(axis=1)[:, None]
    er = ev / (2 * (v + e32)) + 3 * U
    M.assert_within(m, rm, (U * np.abs(rm) + (K + 3) * U * mD[:, 0]) * 1.01, "mean")
    M.assert_within(r, rr, 1.05 * (er * rr[:, None])[:, 0], "rstd")
    ef = U * (2 * D + (K + 3) * mD)
    h = d * rr[:, None]
    bound = np.abs(gm) * (1.05 * rr[:, None] * ef + h * (1.05 * er + 4 * U)) + 4 * U * (np.abs(gm) * h + np.abs(ry))
    M.assert_within(y, ry, bound, "y")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", [77, 256, 2600])
def test_infinities_keep_the_mean_they_had(api, C, dtype):
    """An infinity is the row's mean; both signs or a NaN leave none; neighbours keep their bits."""
    g = torch.Generator(device="cuda").manual_seed(C)
    x = torch.randn((6, C), generator=g, device="cuda").to(M.DT[dtype])
    gamma, beta = _vec(C, 1, 1.0), _vec(C, 2)
    good = api.layer_norm_fwd(x, gamma, beta)
    bad = x.clone()
    bad[1, 3], bad[2, 5], bad[3, 0], bad[3, 1], bad[4, C - 1] = float("inf"), float("-inf"), float("inf"), float("-inf"), float("nan")
    y, m, r = api.layer_norm_fwd(bad, gamma, beta)
    assert m[1] == float("inf") and m[2] == float("-inf") and torch.isnan(m[3:5]).all()
    assert torch.isnan(y[1:5]).all() and torch.isnan(r[1:5]).all()
    for a, b in zip((y, m, r), good):
        assert torch.equal(a[0], b[0]) and torch.equal(a[5], b[5])
