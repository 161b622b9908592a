"""GPU: dropout from the counter-based generator against the fp64 oracle: masks bit for bit, values to a rounding."""
import numpy as np
import pytest
import torch

from oracle import norm as N

import gpu_util as U
import norm_util as M

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_1810_01993_amd import api as _api
    assert torch.cuda.is_available()
    return _api


def _rand(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(M.DT[dtype])


# single elements, either side of a generator block, of a piece and of a workgroup; odd counts; several workgroups
COUNTS = [1, 2, 7, 8, 9, 15, 17, 255, 2048, 2049, 4095, 16384, 16391, 99991, 1 << 20, (1 << 20) + 13]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("n", COUNTS)
def test_forward_and_backward(api, n, dtype):
    p, seed, off = (0.1, 0.2, 0.5, 0.93)[n % 4], (0xDEADBEEF << 32) + n, (n << 33) + 5
    print(f"[case] dropout n={n} {dtype} p={p}", flush=True)
    d = api.DropoutDesc(p, seed, off)
    x, res = _rand(n, dtype, n), _rand(n, dtype, n + 1)
    for residual in (None, res):
        buf, y = U.guarded((n,), M.DT[dtype])
        out = api.dropout_fwd(x, d, residual=residual, y=y)
        torch.cuda.synchronize()
        assert out is y and U.guards_intact(buf)
        M.check_dropout(x, p, seed, off, residual, y, dtype)
    buf, dx = U.guarded((n,), M.DT[dtype])
    api.dropout_bwd(x, d, dx=dx)
    torch.cuda.synchronize()
    assert U.guards_intact(buf)
    M.check_dropout(x, p, seed, off, None, dx, dtype)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_all_none_and_steps_of_p(api, dtype):
    n = 4099
    x = _rand(n, dtype, 3)
    assert torch.equal(api.dropout_fwd(x, api.DropoutDesc(0.0, 9)), x)
    assert torch.equal(api.dropout_fwd(x, api.DropoutDesc(2.0 ** -18, 9)), x)          # less than half a step of p
    assert not api.dropout_fwd(x, api.DropoutDesc(1.0, 9)).any()
    assert torch.equal(api.dropout_fwd(x, api.DropoutDesc(1.0, 9), residual=x), x)
    wide = _rand(1 << 18, "f32", 4)                                     # the largest scale, 65536, on the few that are kept
    M.check_dropout(wide, 1 - 2.0 ** -16, 9, 0, None, api.dropout_fwd(wide, api.DropoutDesc(1 - 2.0 ** -16, 9)), "f32")


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_infinities_and_nan_where_dropped(api, dtype):
    """What is dropped does not reach the output, whatever it is; what is kept does."""
    n, p, seed, off = 8 * 600 + 3, 0.5, 77, 1
    keep = torch.from_numpy(N.keep_mask(n, p, seed, off)).cuda()
    x, res = _rand(n, dtype, 4), _rand(n, dtype, 5)
    lowest = torch.finfo(M.DT[dtype]).min
    bad = torch.tensor([float("nan"), float("inf"), float("-inf"), lowest], device="cuda").to(M.DT[dtype]).repeat(n // 4 + 1)[:n]
    y = api.dropout_fwd(torch.where(keep, x, bad), api.DropoutDesc(p, seed, off), residual=res)
    assert torch.equal(y, api.dropout_fwd(x, api.DropoutDesc(p, seed, off), residual=res))
    dx = api.dropout_bwd(torch.where(keep, bad, x), api.DropoutDesc(p, seed, off))
    assert not dx[~keep].any()
    assert torch.equal(torch.isnan(dx), torch.isnan(bad) & keep)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_in_place_shapes_and_repeats(api, dtype):
    """y over x or over the residual; the mask follows the flat index whatever the shape; the same call gives the same bits."""
    d = api.DropoutDesc(0.3, 5, 6)
    x, res = _rand((3, 5, 7, 11), dtype, 6), _rand((3, 5, 7, 11), dtype, 7)
    y = api.dropout_fwd(x, d, residual=res)
    assert torch.equal(y, api.dropout_fwd(x, d, residual=res))
    assert torch.equal(y.view(-1), api.dropout_fwd(x.view(-1), d, residual=res.view(-1)))
    a, b = x.clone(), res.clone()
    api.dropout_fwd(a, d, residual=res, y=a)
    api.dropout_fwd(x, d, residual=b, y=b)
    assert torch.equal(a, y) and torch.equal(b, y)
    g = x.clone()
    api.dropout_bwd(g, d, dx=g)
    assert torch.equal(g, api.dropout_fwd(x, d))
    assert torch.equal(api.dropout_fwd(x, d, residual=x), api.dropout_fwd(x, d, residual=x.clone()))     # one tensor twice


def test_gradient_is_the_transpose(api):
    """<dropout(x), dy> = <x, dropout_bwd(dy)> with whole numbers, where nothing rounds."""
    n, d = 65537, api.DropoutDesc(0.5, 1 << 40, 3)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randint(-8, 9, (n,), generator=g, device="cuda").float()
    dy = torch.randint(-8, 9, (n,), generator=g, device="cuda").float()
    assert (api.dropout_fwd(x, d).double() * dy).sum() == (x.double() * api.dropout_bwd(dy, d)).sum()


def test_step_on_the_device(api):
    """offset + *step names the mask: an eager call, and a captured one whose replays follow the counter."""
    n, p, seed = 5000, 0.2, 31
    x, res = _rand(n, "f16", 8), _rand(n, "f16", 9)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    d = api.DropoutDesc(p, seed, 100, step)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    step.fill_(4)
    assert torch.equal(api.dropout_fwd(x, d), api.dropout_fwd(x, api.DropoutDesc(p, seed, 104)))
    step.fill_(-1)                                                      # 2^64 - 1: the sum wraps round
    assert torch.equal(api.dropout_fwd(x, d), api.dropout_fwd(x, api.DropoutDesc(p, seed, 99)))
    step.fill_(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        api.dropout_fwd(x, d, residual=res, y=y)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.dropout_fwd(x, d, residual=res, y=y)
        api.dropout_bwd(y, d, dx=dx)
    for k in range(5):
        step.fill_(k)
        x.add_(0.25)
        graph.replay()
        torch.cuda.synchronize()
        e = api.DropoutDesc(p, seed, 100 + k)
        want = api.dropout_fwd(x, e, residual=res)
        assert torch.equal(y, want) and torch.equal(dx, api.dropout_bwd(want, e)), k


def test_on_another_stream(api):
    x = _rand(1 << 20, "bf16", 10)
    d = api.DropoutDesc(0.1, 2)
    want = api.dropout_fwd(x, d)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = api.dropout_fwd(x, d)
    s.synchronize()
    assert torch.equal(got, want)


def test_offsets_beyond_32_bits(api):
    """2^35 + 21 elements (68.7 GB, in place): the element index, its byte offset and the block number all pass 32 bits."""
    n = (1 << 35) + 21
    x = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    p, seed, off = 0.5, 3, 4
    starts = [0, (1 << 31) - 40, (1 << 32) - 40, (1 << 34) - 40, n - 61]
    for a in starts:
        x[a:a + 61] = _rand(61, "bf16", a % 1000)
    before = {a: x[a:a + 61].clone() for a in starts}
    api.dropout_fwd(x, api.DropoutDesc(p, seed, off), y=x)
    torch.cuda.synchronize()
    for a in starts:
        M.check_dropout(before[a], p, seed, off, None, x[a:a + 61], "bf16", first=a)


def test_empty(api):
    x = torch.empty((0, 5), dtype=torch.float16, device="cuda")
    assert api.dropout_fwd(x, api.DropoutDesc(0.5, 1), residual=x.clone()).shape == (0, 5)
    assert api.dropout_bwd(x, api.DropoutDesc(0.5, 1)).shape == (0, 5)
