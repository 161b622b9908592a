"""Pins of the fp64 oracle of layer norm and dropout: published answers of the generator, hand examples, torch's float64
routines with autograd, finite differences, and statistics of the mask."""
import numpy as np
import pytest
import torch

from oracle import norm as N


def test_generator_known_answers():
    """The published known answers of Philox4x32-10 (Random123 distribution, kat_vectors)."""
    full = 0xFFFFFFFF
    for ctr, key, want in [((0,) * 4, (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
                           ((full,) * 4, (full, full), (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
                           ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
                            (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]:
        assert tuple(int(v) for v in N.philox4x32_10(np.array(ctr, dtype=np.uint64), key)) == want


def test_mask_layout_by_hand():
    """Element i takes field i % 8 of block i / 8: the first block under a zero key and counter, p set on either side of a field."""
    fields = [w >> s & 0xFFFF for w in (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8) for s in (0, 16)]
    for e, f in enumerate(fields):
        assert N.keep_mask(8, f / 65536, 0, 0)[e] and not N.keep_mask(8, (f + 1) / 65536, 0, 0)[e]
    whole = N.keep_mask(100, 0.3, 7, 9)
    assert np.array_equal(N.keep_mask(41, 0.3, 7, 9, first=37), whole[37:78])
    # beyond 2^32 blocks the second word of the counter counts
    a = N.keep_mask(64, 0.5, 1, 2, first=1 << 35)
    assert not np.array_equal(a, N.keep_mask(64, 0.5, 1, 2)) and a.any() and not a.all()


def test_mask_frequency_and_independence():
    """The kept share of 2^20 elements lies within 5 deviations of 1 - p; masks of another offset, seed or neighbouring field
    agree as often as independent ones."""
    n = 1 << 20
    for p in (0.1, 0.2, 0.5):
        q = 1 - N.threshold(p) / 65536
        a, b, c = N.keep_mask(n, p, 11, 0), N.keep_mask(n, p, 11, 1), N.keep_mask(n, p, 12, 0)
        assert abs(a.mean() - q) < 5 * np.sqrt(q * (1 - q) / n)
        same = q * q + (1 - q) ** 2
        for other in (b, c, np.roll(a, 1), np.roll(a, 8)):
            assert abs((a == other).mean() - same) < 6 * np.sqrt(same * (1 - same) / n)


def test_dropout_limits_and_scale():
    x = np.arange(1.0, 33.0)
    assert np.array_equal(N.dropout(x, 0.0, 3, 4), x) and not N.dropout(x, 1.0, 3, 4).any()
    y = N.dropout(x, 0.25, 3, 4, residual=-x)
    k = N.keep_mask(32, 0.25, 3, 4)
    assert np.allclose(y[k], x[k] / 3) and np.array_equal(y[~k], -x[~k])


@pytest.mark.parametrize("n,C", [(1, 1), (3, 2), (5, 7), (4, 64)])
def test_layer_norm_against_torch(n, C):
    g = torch.Generator().manual_seed(n * 100 + C)
    x = torch.randn(n, C, generator=g, dtype=torch.float64, requires_grad=True)
    w = torch.randn(C, generator=g, dtype=torch.float64, requires_grad=True)
    b = torch.randn(C, generator=g, dtype=torch.float64, requires_grad=True)
    dy = torch.randn(n, C, generator=g, dtype=torch.float64)
    y = torch.nn.functional.layer_norm(x, (C,), w, b, 1e-5)
    y.backward(dy)
    got, m, r = N.layer_norm(x.detach().numpy(), w.detach().numpy(), b.detach().numpy(), 1e-5)
    assert np.allclose(got, y.detach().numpy(), atol=1e-12)
    dx, dw, db = N.layer_norm_bwd(dy.numpy(), x.detach().numpy(), w.detach().numpy(), m, r)
    # r reaches 1/sqrt(eps) = 316 where a row has one value: 1e-10 is 1e-16 times r^3 / 1e-5, less than that in every case
    assert np.allclose(dx, x.grad.numpy(), atol=1e-10) and np.allclose(dw, w.grad.numpy(), atol=1e-10)
    assert np.allclose(db, b.grad.numpy(), atol=1e-12)


def test_layer_norm_by_hand():
    y, m, r = N.layer_norm([[1.0, 3.0], [5.0, 5.0]], None, None, 0.0 + 1.0)
    assert np.allclose(m, [2, 5]) and np.allclose(r, [1 / np.sqrt(2), 1]) and np.allclose(y, [[-1 / np.sqrt(2), 1 / np.sqrt(2)], [0, 0]])


def test_joined_gradient_against_differences():
    """d/dx and d/dresidual of <y, dy> + <s, ds> by central differences of the joined forward pass."""
    g = np.random.default_rng(5)
    n, C, p, seed, off = 3, 5, 0.3, 21, 6
    x, res, dy, ds = (g.normal(size=(n, C)) for _ in range(4))
    gamma, beta = g.normal(size=C), g.normal(size=C)

    def value(x, res, gamma=gamma, beta=beta):
        s = N.dropout(x, p, seed, off, residual=res)
        return (N.layer_norm(s, gamma, beta, 1e-3)[0] * dy).sum() + (s * ds).sum()
    s = N.dropout(x, p, seed, off, residual=res)
    _, m, r = N.layer_norm(s, gamma, beta, 1e-3)
    dres, dx, dgamma, dbeta = N.joined_bwd(dy, ds, s, p, seed, off, gamma, m, r)
    h = 1e-5

    def numeric(f, a):
        out = np.empty_like(a)
        for i in np.ndindex(*a.shape):
            hi, lo = a.copy(), a.copy()
            hi[i] += h
            lo[i] -= h
            out[i] = (f(hi) - f(lo)) / (2 * h)
        return out
    # the third derivative times h^2 / 6 and 1e-16 / h: both below 1e-7 here
    assert np.allclose(numeric(lambda a: value(a, res), x), dx, atol=1e-7)
    assert np.allclose(numeric(lambda a: value(x, a), res), dres, atol=1e-7)
    assert np.allclose(numeric(lambda a: value(x, res, gamma=a), gamma), dgamma, atol=1e-7)
    assert np.allclose(numeric(lambda a: value(x, res, beta=a), beta), dbeta, atol=1e-7)
