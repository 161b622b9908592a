"""GPU: layer norm forward and backward, alone and behind a residual add with dropout, against the fp64 oracle, with error bounds
counted from the roundings."""
import numpy as np
import pytest
import torch

from oracle import norm as N

import gpu_util as U
import norm_util as M

pytestmark = pytest.mark.gpu
DTYPES = ["f16", "bf16", "f32"]


@pytest.fixture(scope="module")
def api():
    from paper_1810_01993_amd import api as _api
    assert torch.cuda.is_available()
    return _api


def _rand(shape, dtype, seed, mean=0.0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * spread + mean).to(M.DT[dtype])


def _vec(C, seed, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return mean + 0.3 * torch.randn(C, generator=g, device="cuda")


def _alone(api, n, C, dtype, eps=1e-5, mean=0.5, spread=1.0, affine=True, params=True, x=None):
    print(f"[case] layer_norm n={n} C={C} {dtype} affine={affine} params={params}", flush=True)
    x = _rand((n, C), dtype, n + C, mean, spread) if x is None else x
    dy = _rand((n, C), dtype, n + C + 1)
    gamma, beta = (_vec(C, 1, 1.0), _vec(C, 2)) if affine else (None, None)
    yb, y = U.guarded((n, C), M.DT[dtype])
    mb, m = U.guarded((n,), torch.float32)
    rb, r = U.guarded((n,), torch.float32)
    api.layer_norm_fwd(x, gamma, beta, eps, y=y, mean=m, rstd=r)
    torch.cuda.synchronize()
    assert U.guards_intact(yb) and U.guards_intact(mb) and U.guards_intact(rb)
    M.check_forward(x, gamma, beta, eps, y, m, r, dtype)
    db_, dx = U.guarded((n, C), M.DT[dtype])
    gb, dg = U.guarded((C,), torch.float32)
    bb, dbeta = U.guarded((C,), torch.float32)
    need = api.dl_layer_norm_bwd_workspace_bytes(n, C)
    wb, ws = U.guarded_workspace(need)
    if params:
        api.layer_norm_bwd(dy, x, gamma, m, r, dx=dx, dgamma=dg, dbeta=dbeta, workspace=ws)
    else:
        assert api.layer_norm_bwd(dy, x, gamma, m, r, dx=dx, want_params=False)[1:] == (None, None)
    torch.cuda.synchronize()
    assert U.guards_intact(db_) and U.guards_intact(gb) and U.guards_intact(bb) and U.workspace_guards_intact(wb, need)
    M.check_backward(dy, x, gamma, m, r, dx, dg if params else None, dbeta if params else None, dtype)
    return x, dy, gamma, beta, y, m, r, dx, dg, dbeta


def _joined(api, n, C, dtype, p=0.2, residual=True, stream=True, affine=True):
    print(f"[case] joined n={n} C={C} {dtype} p={p} residual={residual} ds={stream}", flush=True)
    seed, off = (n << 34) + C, 7
    d = None if p is None else api.DropoutDesc(p, seed, off)
    x = _rand((n, C), dtype, n + C)
    res = _rand((n, C), dtype, n + C + 1, 0.5) if residual else None
    gamma, beta = (_vec(C, 1, 1.0), _vec(C, 2)) if affine else (None, None)
    outs = [U.guarded((n, C), M.DT[dtype]) for _ in range(4)]
    (_, s), (_, y), (_, dres), (_, dx) = outs
    mb, m = U.guarded((n,), torch.float32)
    rb, r = U.guarded((n,), torch.float32)
    api.dropout_add_layer_norm_fwd(x, res, d, gamma, beta, 1e-5, s=s, y=y, mean=m, rstd=r)
    torch.cuda.synchronize()
    M.check_dropout(x, 0.0 if p is None else p, seed, off, res, s, dtype)
    M.check_forward(s, gamma, beta, 1e-5, y, m, r, dtype)
    # the bits of the two calls one after the other
    s2 = api.dropout_fwd(x, d if d else api.DropoutDesc(0.0, 0), residual=res)
    y2, m2, r2 = api.layer_norm_fwd(s2, gamma, beta, 1e-5)
    assert torch.equal(s, s2) and torch.equal(y, y2) and torch.equal(m, m2) and torch.equal(r, r2)
    dy = _rand((n, C), dtype, n + C + 2)
    ds = _rand((n, C), dtype, n + C + 3) if stream else None
    dresidual, dxo, dg, db = api.dropout_add_layer_norm_bwd(dy, ds, s, d, gamma, m, r, dresidual=dres, dx=dx)
    torch.cuda.synchronize()
    assert all(U.guards_intact(b) for b, _ in outs) and U.guards_intact(mb) and U.guards_intact(rb)
    M.check_backward(dy, s, gamma, m, r, dres, dg, db, dtype, ds, dx, (0.0 if p is None else p, seed, off))
    _, dg2, db2 = api.layer_norm_bwd(dy, s, gamma, m, r)
    assert torch.equal(dg, dg2) and torch.equal(db, db2)


# one channel; fewer than a piece; either side of whole pieces; of a wave's row, a workgroup's row and the longest row kept in
# registers; rows from one to several workgroups' worth, odd ones among them
SHAPES = [(1, 1), (3, 2), (9, 3), (700, 5), (1, 7), (5, 8), (33, 9), (257, 16), (64, 24), (101, 31), (77, 33), (66, 48), (130, 64),
          (19, 65), (4099, 77), (31, 100), (9, 127), (8, 255), (2, 256), (1031, 256), (4, 257), (999, 304), (35, 511), (3, 512),
          (5, 513), (61, 771), (130, 1024), (7, 1025), (17, 2047), (21, 2048), (6, 2049), (3, 2056), (2, 3001), (5, 4096),
          (3, 4097), (4, 8192), (2, 8193), (3, 8200), (1, 12345), (2, 12289), (2, 16384), (2, 16385), (1, 40000),
          (40, 768), (41, 769), (20, 1536), (21, 1537), (700, 2057)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,C", SHAPES, ids=[f"{n}x{C}" for n, C in SHAPES])
def test_alone(api, n, C, dtype):
    _alone(api, n, C, dtype, affine=(n + C) % 5 != 0, params=(n + C) % 7 != 0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,C", SHAPES, ids=[f"{n}x{C}" for n, C in SHAPES])
def test_joined(api, n, C, dtype):
    _joined(api, n, C, dtype, p=(0.2, 0.5, None, 0.05)[n % 4], residual=C % 6 != 0, stream=(n + C) % 4 != 0, affine=n % 5 != 0)


# many rows: several rows a workgroup, slabs of unequal length
MANY = [(20011, 8), (30011, 24), (100003, 3), (25013, 40), (65537, 64), (20001, 128), (9001, 304), (40007, 256), (3001, 1024),
        (1025, 2048), (2051, 771), (600, 4104), (300, 8192), (77, 20000), (300001, 16)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,C", MANY, ids=[f"{n}x{C}" for n, C in MANY])
def test_many_rows(api, n, C, dtype):
    _alone(api, n, C, dtype)
    _joined(api, n, C, dtype)


@pytest.mark.parametrize("dtype,C", [("f16", 1544), ("f32", 772)])
def test_many_rows_of_one_piece_a_lane(api, dtype, C):
    """A workgroup per row with one piece a lane, either side of the row count from which more workgroups share the rows."""
    for n in (16383, 16384):
        _alone(api, n, C, dtype)


@pytest.mark.parametrize("n,C", [(2 * 48 * 72, 1024), (2 * 192 * 288, 304)])
def test_framework_sized_maps(api, n, C):
    _alone(api, n, C, "bf16")
    _joined(api, n, C, "f16", p=0.1)


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_of_equal_values_and_far_means(api, dtype):
    """No spread: y is beta, and 1/sqrt(eps) stays finite; a mean far above the spread costs the digits that the bound counts."""
    for C in (1, 8, 77, 256, 2048, 9000):
        x = _rand((5, 1), dtype, C).expand(5, C).contiguous()
        beta = _vec(C, 3)
        y, m, r = api.layer_norm_fwd(x, torch.ones_like(beta), beta, 1e-5)
        K = M.chain(C) * M.U32
        # x - m is off by the mean's error alone, and the deviation's square by its square
        e = K * M.f64(x)[:, :1].__abs__() * 1e-5 ** -0.5 * 1.01
        ref = np.broadcast_to(M.f64(beta), (5, C))
        M.assert_within(y, ref, e + (M.HALF[dtype] * 1.01 + 4 * M.U32) * np.abs(ref) + e * M.HALF[dtype] * 1.01 + M.TINY[dtype], "y")
        _alone(api, 6, C, dtype, mean=300.0, spread=1.0) if C > 1 else None
        _alone(api, 6, C, dtype, spread=1e-3)


def test_zero_eps_and_large_eps(api):
    _alone(api, 50, 256, "f32", eps=0.0)
    _alone(api, 50, 77, "f16", eps=3.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("C", [7, 64, 77, 1024, 4100, 9000])
def test_a_bad_row_stays_alone(api, C, dtype):
    """NaN or an infinity in one row: that row's outputs are NaN, every other row keeps its bits."""
    n = 37
    x, dy = _rand((n, C), dtype, C), _rand((n, C), dtype, C + 1)
    gamma, beta = _vec(C, 1, 1.0), _vec(C, 2)
    y, m, r = api.layer_norm_fwd(x, gamma, beta)
    dx, _, _ = api.layer_norm_bwd(dy, x, gamma, m, r)
    bad = x.clone()
    bad[5, C // 2], bad[20, 0], bad[36, C - 1] = float("nan"), float("inf"), float("-inf")
    y2, m2, r2 = api.layer_norm_fwd(bad, gamma, beta)
    dx2, dg2, db2 = api.layer_norm_bwd(dy, bad, gamma, m2, r2)
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[[5, 20, 36]] = False
    for a, b in ((y, y2), (m, m2), (r, r2), (dx, dx2)):
        assert torch.equal(a[keep], b[keep])
    assert torch.isnan(y2[~keep]).all() and torch.isnan(dx2[~keep]).all()
    assert torch.isnan(dg2).all() and torch.isfinite(db2).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,C", [(65, 48), (65, 77), (300, 256), (9, 2048), (5, 4100), (3, 9001), (2, 20001), (900, 1801), (700, 4099)])
def test_in_place_and_repeatable(api, n, C, dtype):
    """Outputs over inputs, as the header allows, and the same bits from the same call."""
    x, res, dy, ds = (_rand((n, C), dtype, C + k) for k in range(4))
    gamma, beta = _vec(C, 1, 1.0), _vec(C, 2)
    d = api.DropoutDesc(0.25, 3, 4)
    y, m, r = api.layer_norm_fwd(x, gamma, beta)
    a = x.clone()
    assert torch.equal(api.layer_norm_fwd(a, gamma, beta, y=a)[0], y)
    assert torch.equal(api.layer_norm_fwd(x, gamma, beta, want_stats=False)[0], y)
    want = api.layer_norm_bwd(dy, x, gamma, m, r)
    for over in ("dy", "x"):
        a, b = dy.clone(), x.clone()
        got = api.layer_norm_bwd(a, b, gamma, m, r, dx=a if over == "dy" else b)
        assert all(torch.equal(p, q) for p, q in zip(got, want)), over
    fwd = api.dropout_add_layer_norm_fwd(x, res, d, gamma, beta)
    for s_over, y_over in (("x", "res"), ("res", "x"), ("x", None), (None, "res")):
        a, b = x.clone(), res.clone()
        pick = {"x": a, "res": b, None: None}
        got = api.dropout_add_layer_norm_fwd(a, b, d, gamma, beta, s=pick[s_over], y=pick[y_over])
        assert all(torch.equal(p, q) for p, q in zip(got, fwd)), (s_over, y_over)
    s, _, m, r = fwd
    bwd = api.dropout_add_layer_norm_bwd(dy, ds, s, d, gamma, m, r)
    for one, two in (("dy", "ds"), ("ds", "s"), ("s", "dy"), ("dy", None), (None, "ds")):
        v = {"dy": dy.clone(), "ds": ds.clone(), "s": s.clone(), None: None}
        got = api.dropout_add_layer_norm_bwd(v["dy"], v["ds"], v["s"], d, gamma, m, r, dresidual=v[one], dx=v[two])
        assert all(torch.equal(p, q) for p, q in zip(got, bwd)), (one, two)
    # one tensor given twice as input
    both = api.dropout_add_layer_norm_fwd(x, x, d, gamma, beta)
    assert all(torch.equal(p, q) for p, q in zip(both, api.dropout_add_layer_norm_fwd(x, x.clone(), d, gamma, beta)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,C", [(40, 200), (300, 77), (6, 2600), (3, 20001)])
def test_least_alignment(api, n, C, dtype):
    """Tensors that begin 16 bytes into a line, float arrays 4 bytes: the same bits as from a fresh allocation."""
    step = 16 // M.DT[dtype].itemsize

    def moved(t, by):
        buf = torch.zeros(t.numel() + by, dtype=t.dtype, device="cuda")
        buf[by:] = t.reshape(-1)
        return buf[by:].view(t.shape)
    x, res, dy, ds = (_rand((n, C), dtype, C + k) for k in range(4))
    gamma, beta, d = _vec(C, 1, 1.0), _vec(C, 2), api.DropoutDesc(0.25, 3, 4)
    want = api.dropout_add_layer_norm_fwd(x, res, d, gamma, beta)
    outs = [moved(t, by) for t, by in zip(want, (step, 3 * step, 1, 3))]
    got = api.dropout_add_layer_norm_fwd(moved(x, step), moved(res, 5 * step), d, moved(gamma, 1), moved(beta, 3), s=outs[0], y=outs[1],
                                         mean=outs[2], rstd=outs[3])
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    s, _, m, r = want
    want = api.dropout_add_layer_norm_bwd(dy, ds, s, d, gamma, m, r)
    outs = [moved(t, by) for t, by in zip(want, (step, 7 * step, 1, 2))]
    ws = torch.empty(api.dl_layer_norm_bwd_workspace_bytes(n, C) + 16, dtype=torch.uint8, device="cuda")[16:]
    got = api.dropout_add_layer_norm_bwd(moved(dy, step), moved(ds, 3 * step), moved(s, step), d, moved(gamma, 1), moved(m, 1), moved(r, 3),
                                         dresidual=outs[0], dx=outs[1], dgamma=outs[2], dbeta=outs[3], workspace=ws)
    assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_outputs_left_out(api):
    """The C boundary writes only what it is given: dx or dresidual alone, statistics left out."""
    n, C = 70, 77
    x, res, dy = (_rand((n, C), "f16", k) for k in range(3))
    gamma, beta, d = _vec(C, 1, 1.0), _vec(C, 2), api.DropoutDesc(0.4, 8)
    s, y, m, r = api.dropout_add_layer_norm_fwd(x, res, d, gamma, beta)
    dres, dx, _, _ = api.dropout_add_layer_norm_bwd(dy, None, s, d, gamma, m, r)
    for only in (0, 1):
        outs = [torch.full_like(dy, 5.0) for _ in range(2)]
        ptr = [o.data_ptr() if i == only else None for i, o in enumerate(outs)]
        rc = api._lib.dropout_add_layer_norm_bwd(dy.data_ptr(), None, s.data_ptr(), d._kept, gamma.data_ptr(), m.data_ptr(), r.data_ptr(),
                                                 0, n, C, *ptr, None, None, None, 0, api._stream())
        torch.cuda.synchronize()
        assert rc == 0 and torch.equal(outs[only], (dres, dx)[only]) and bool((outs[1 - only] == 5).all())
    y2 = torch.empty_like(y)
    assert api._lib.layer_norm_fwd(s.data_ptr(), gamma.data_ptr(), beta.data_ptr(), 0, n, C, 1e-5, y2.data_ptr(), None, None, api._stream()) == 0
    torch.cuda.synchronize()
    assert torch.equal(y2, y)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,C", [(33, 77), (5, 2048)])
def test_everything_dropped(api, n, C, dtype):
    """p = 1 over infinities and NaN: without a residual every row of s is empty (zero), y is beta and no gradient reaches x."""
    x = torch.full((n, C), float("nan"), device="cuda").to(M.DT[dtype])
    x[::2] = float("inf")
    gamma, beta, d = _vec(C, 1, 1.0), _vec(C, 2), api.DropoutDesc(1.0, 7)
    s, y, m, r = api.dropout_add_layer_norm_fwd(x, None, d, gamma, beta)
    assert not s.any() and not m.any() and torch.equal(y, beta.to(M.DT[dtype]).expand(n, C))
    M.assert_within(r, np.full(n, float(np.float32(1e-5)) ** -0.5), np.full(n, 4 * M.U32 * 317), "rstd")     # a square root and a division
    dy, ds = _rand((n, C), dtype, 1), _rand((n, C), dtype, 2)
    dres, dx, dg, db = api.dropout_add_layer_norm_bwd(dy, ds, s, d, gamma, m, r)
    assert not dx.any() and not dg.any()
    M.check_backward(dy, s, gamma, m, r, dres, dg, db, dtype, ds)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_gradients_against_differences(api, dtype):
    """dx, dgamma and dbeta against central differences of the oracle's forward pass at the stored inputs."""
    n, C, eps = 4, 11, 1e-2
    x, dy = _rand((n, C), dtype, 1), _rand((n, C), dtype, 2)
    gamma, beta = _vec(C, 1, 1.0), _vec(C, 2)
    _, m, r = api.layer_norm_fwd(x, gamma, beta, eps)
    dx, dg, db = api.layer_norm_bwd(dy, x, gamma, m, r)
    a = [M.f64(x), M.f64(gamma), M.f64(beta)]
    up, h = M.f64(dy), 1e-5

    def value(v):
        return (N.layer_norm(v[0], v[1], v[2], eps)[0] * up).sum()
    # half a step of dx's type, the fp32 roundings (some tens of 2^-24 of terms of a few units), h^2 and 1e-16 / h of the quotient
    for k, got in enumerate((dx, dg, db)):
        num = np.empty_like(a[k])
        for i in np.ndindex(*num.shape):
            hi, lo = [v.copy() for v in a], [v.copy() for v in a]
            hi[k][i] += h
            lo[k][i] -= h
            num[i] = (value(hi) - value(lo)) / (2 * h)
        tol = 5e-6 + (1.01 * M.HALF[dtype] * np.abs(num) if k == 0 else 0)
        assert (np.abs(M.f64(got) - num) <= tol).all(), k


def test_captured_step(api):
    """Joined forward and backward in one graph: each replay, with other inputs and another mask, gives the eager bits; two graphs
    that share a workspace are replayed in turn."""
    n, C = 500, 200
    x, res, dy, ds = (_rand((n, C), "bf16", k) for k in range(4))
    gamma, beta = _vec(C, 1, 1.0), _vec(C, 2)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    ws = torch.empty(api.dl_layer_norm_bwd_workspace_bytes(n, C), dtype=torch.uint8, device="cuda")

    def buffers():
        return [torch.empty_like(x) for _ in range(4)] + [torch.empty(n, device="cuda") for _ in range(2)] + [torch.empty(C, device="cuda") for _ in range(2)]

    def go(d, b, work):
        s, y, dres, dx, m, r, dg, db = b
        api.dropout_add_layer_norm_fwd(x, res, d, gamma, beta, s=s, y=y, mean=m, rstd=r)
        api.dropout_add_layer_norm_bwd(dy, ds, s, d, gamma, m, r, dresidual=dres, dx=dx, dgamma=dg, dbeta=db, workspace=work)
    graphs = []
    for k in range(2):
        b, d = buffers(), api.DropoutDesc(0.3, 17, 1000 * k, step)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            go(d, b, ws)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            go(d, b, ws)
        graphs.append((g, b))
    for t in range(4):
        step.fill_(t)
        x.mul_(0.75)
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for k, (_, b) in enumerate(graphs):
            e = buffers()
            go(api.DropoutDesc(0.3, 17, 1000 * k + t), e, None)
            assert all(torch.equal(p, q) for p, q in zip(b, e)), (t, k)


def test_calls_on_two_streams(api):
    """Two backward calls at once, each with a workspace of its own."""
    n, C = 30000, 256
    x, dy = _rand((n, C), "f16", 1), _rand((n, C), "f16", 2)
    gamma, beta = _vec(C, 1, 1.0), _vec(C, 2)
    _, m, r = api.layer_norm_fwd(x, gamma, beta)
    want = api.layer_norm_bwd(dy, x, gamma, m, r)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append([api.layer_norm_bwd(dy, x, gamma, m, r) for _ in range(3)])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for per in got for out in per for a, b in zip(out, want))


def test_offsets_beyond_32_bits(api):
    """More than 2^32 elements: the last rows are as the same rows alone, forward and backward."""
    C = 264
    n = (1 << 32) // C + 1001
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.empty((n, C), dtype=torch.bfloat16, device="cuda")
    rows = [slice(0, 40), slice((1 << 31) // C - 20, (1 << 31) // C + 20), slice(n - 40, n)]
    x.zero_()
    for k in rows:
        x[k] = torch.randn((40, C), generator=g, device="cuda").to(torch.bfloat16)
    gamma, beta = _vec(C, 1, 1.0), _vec(C, 2)
    y, m, r = api.layer_norm_fwd(x, gamma, beta)
    torch.cuda.synchronize()
    for k in rows:
        ya, ma, ra = api.layer_norm_fwd(x[k].clone(), gamma, beta)
        assert torch.equal(y[k], ya) and torch.equal(m[k], ma) and torch.equal(r[k], ra)
    dx, dg, db = api.layer_norm_bwd(x, x, gamma, m, r, dx=y)
    # the rows of zeros add nothing to either sum: what the three runs of rows give is all
    part = torch.cat([x[k] for k in rows])
    pm, pr = torch.cat([m[k] for k in rows]), torch.cat([r[k] for k in rows])
    da, _, _ = api.layer_norm_bwd(part, part, gamma, pm, pr)
    assert torch.equal(torch.cat([dx[k] for k in rows]), da)
    M.check_backward(part, part, gamma, pm, pr, None, dg, db, "bf16")


def test_empty(api):
    x = torch.empty((0, 24), dtype=torch.float16, device="cuda")
    gamma, beta = _vec(24, 1, 1.0), _vec(24, 2)
    y, m, r = api.layer_norm_fwd(x, gamma, beta)
    dx, dg, db = api.layer_norm_bwd(x, x, gamma, m, r)
    torch.cuda.synchronize()
    assert y.shape == dx.shape == (0, 24) and m.shape == (0,) and not dg.any() and not db.any()


def test_refusals_on_the_device(api):
    x, v = torch.zeros((6, 8), dtype=torch.float16, device="cuda"), torch.zeros(8, device="cuda")
    m = torch.zeros(6, device="cuda")
    for call in (lambda: api.layer_norm_fwd(x.t(), v[:6], v[:6]), lambda: api.layer_norm_fwd(x, v, v[:4]), lambda: api.layer_norm_fwd(x, v, None),
                 lambda: api.layer_norm_fwd(x, v.half(), v.half()), lambda: api.layer_norm_fwd(x, v, v, y=x.float()), lambda: api.layer_norm_fwd(x, v, v, y=x[:3]),
                 lambda: api.layer_norm_fwd(x, v, v, y=x.cpu()), lambda: api.layer_norm_fwd(x, v, v, y=x.view(2, 24)),
                 lambda: api.layer_norm_fwd(x, v.cpu(), v.cpu()), lambda: api.layer_norm_bwd(x, x, v, m[:5], m),
                 lambda: api.layer_norm_bwd(x, x.float(), v, m, m), lambda: api.dropout_fwd(x, api.DropoutDesc(0.1, 1), residual=x[:3]),
                 lambda: api.layer_norm_fwd(x[:, :4], v[:4], v[:4])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: api.layer_norm_fwd(x, v, v, eps=-1.0), lambda: api.layer_norm_bwd(x, x, v, m, m, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")),
                 lambda: api.dropout_add_layer_norm_fwd(x, x, None, v, v, s=x, y=x), lambda: api.layer_norm_fwd(x.view(-1)[4:44].view(5, 8), v, v)):
        with pytest.raises(api.DlError):
            call()


def test_residual_blocks_run_together(api):
    """Two residual blocks as a program would run them, forward and backward: norm, 1x1 convolution with bias and ReLU, dropout
    joined to the residual add and the next norm, a 3x3 convolution.  Every stage is held to the oracle at its stored inputs, and
    the whole chain's weight gradient to the change of <output, upstream> along it."""
    N_, H, W, C = 2, 9, 13, 48
    shape = (N_, H, W, C)
    c1 = api.ConvDesc(N_, H, W, C, C, 1, 1, dtype=api.DL_F16)
    c3 = api.ConvDesc(N_, H, W, C, C, 3, 3, 1, 1, 1, 1, dtype=api.DL_F16)
    x = _rand(shape, "f16", 1)
    w1, w3 = _rand((C, 1, 1, C), "f16", 2, spread=C ** -0.5), _rand((C, 3, 3, C), "f16", 3, spread=(9 * C) ** -0.5)
    g1, b1, g2, b2, bias = _vec(C, 4, 1.0), _vec(C, 5), _vec(C, 6, 1.0), _vec(C, 7), _vec(C, 8)
    drop = api.DropoutDesc(0.2, 99, 12)
    y1, m1, r1 = api.layer_norm_fwd(x, g1, b1)
    u = api.conv2d_fwd_bias_relu(c1, y1, w1, bias, True)
    s, y2, m2, r2 = api.dropout_add_layer_norm_fwd(u, x, drop, g2, b2)
    z = api.conv2d_fwd(c3, y2, w3)
    up = _rand(shape, "f16", 9)
    dy2 = api.conv2d_bwd_data(c3, up, w3)
    dres, du, dg2, db2 = api.dropout_add_layer_norm_bwd(dy2, None, s, drop, g2, m2, r2)
    dpre, dbias = api.bias_relu_bwd(du, u, True)
    dy1 = api.conv2d_bwd_data(c1, dpre, w1)
    dw1 = api.conv2d_bwd_filter(c1, y1, dpre)
    dx1, dg1, db1 = api.layer_norm_bwd(dy1, x, g1, m1, r1)
    torch.cuda.synchronize()
    f = lambda t: t.reshape(-1, C)                                                                      # noqa: E731
    M.check_forward(f(x), g1, b1, 1e-5, f(y1), m1.reshape(-1), r1.reshape(-1), "f16")
    M.check_dropout(u, 0.2, 99, 12, x, s, "f16")
    M.check_forward(f(s), g2, b2, 1e-5, f(y2), m2.reshape(-1), r2.reshape(-1), "f16")
    M.check_backward(f(dy2), f(s), g2, m2, r2, f(dres), dg2, db2, "f16", None, f(du), (0.2, 99, 12))
    M.check_backward(f(dy1), f(x), g1, m1, r1, f(dx1), dg1, db1, "f16")
    # The whole chain in float64 on the host, differentiated by torch; every stored tensor is rounded once to fp16 (half a step,
    # 2^-11 of its value), about ten of them lie on the way to a gradient: 2^-7 of the gradient's largest value covers each adding up.
    keep = torch.from_numpy(N.keep_mask(x.numel(), 0.2, 99, 12).reshape(shape))
    X, W1, W3 = (t.double().cpu().requires_grad_() for t in (x, w1, w3))
    P = [t.double().cpu().requires_grad_() for t in (g1, b1, g2, b2, bias)]
    n1 = torch.nn.functional.layer_norm(X, (C,), P[0], P[1], 1e-5)
    U_ = (n1 @ W1.reshape(C, C).T + P[4]) * (u > 0).double().cpu()         # the branch of the ReLU that the program took
    S = X + torch.where(keep, U_ * (65536 / (65536 - N.threshold(0.2))), 0.0)
    n2 = torch.nn.functional.layer_norm(S, (C,), P[2], P[3], 1e-5)
    Z = torch.nn.functional.conv2d(n2.permute(0, 3, 1, 2), W3.permute(0, 3, 1, 2), padding=1).permute(0, 2, 3, 1)
    (Z * up.double().cpu()).sum().backward()
    pairs = [(z, Z), (dres.double() + dx1.double(), X.grad), (dw1, W1.grad), (dg1, P[0].grad), (db1, P[1].grad), (dg2, P[2].grad), (db2, P[3].grad),
             (dbias, P[4].grad)]
    for k, (got, ref) in enumerate(pairs):
        assert U.rel_err(M.f64(got), ref.detach().numpy()) <= 2.0 ** -7, k
