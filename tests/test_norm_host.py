"""Host-only checks of layer norm and dropout: every refusal comes back as its status before anything is launched, workspace
queries, and what the Python wrapper refuses."""
import copy
import ctypes
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED, VALUE = 0, 1, 2, 3, 4, 5, 6, 8


@pytest.fixture(scope="module")
def api():
    from paper_1810_01993_amd import api as _api
    return _api


def _drop(api, p=0.1, step=None):
    return ctypes.byref(api._Dropout(p, 1, 2, step))


def test_dropout_refusals(api):
    fwd, bwd, d = api._lib.dropout_fwd, api._lib.dropout_bwd, _drop(api)
    assert fwd(None, None, d, 0, 8, 16, None) == NULL and fwd(16, None, d, 0, 8, None, None) == NULL
    assert fwd(16, None, None, 0, 8, 16, None) == NULL and bwd(None, d, 0, 8, 16, None) == NULL
    assert fwd(16, None, d, 0, -1, 16, None) == SHAPE and bwd(16, d, 0, 1 << 46, 16, None) == SHAPE
    assert fwd(16, None, d, 3, 8, 16, None) == DTYPE and bwd(16, d, -1, 8, 16, None) == DTYPE
    for p in (-0.1, 1.001, float("nan"), float("inf")):
        assert fwd(16, None, _drop(api, p), 0, 8, 16, None) == VALUE
    assert fwd(24, None, d, 0, 8, 16, None) == ALIGN and fwd(16, 8, d, 0, 8, 16, None) == ALIGN
    assert bwd(16, d, 0, 8, 18, None) == ALIGN and fwd(16, None, _drop(api, 0.1, 12), 0, 8, 16, None) == ALIGN
    assert fwd(None, None, d, 0, 0, None, None) == OK                   # nothing to do: nothing is launched
    assert b"range" in api._lib.dl_status_string(VALUE)


def test_layer_norm_forward_refusals(api):
    f = api._lib.layer_norm_fwd
    assert f(None, 16, 16, 0, 4, 8, 1e-5, 16, 16, 16, None) == NULL
    assert f(16, 16, None, 0, 4, 8, 1e-5, 16, 16, 16, None) == NULL     # gamma without beta
    assert f(16, 16, 16, 0, 4, 8, 1e-5, None, 16, 16, None) == NULL
    for n, C in ((-1, 8), (4, 0), (4, -3), (4, (1 << 20) + 1), (1 << 45, 2), (1 << 62, 1 << 20)):
        assert f(16, 16, 16, 0, n, C, 1e-5, 16, 16, 16, None) == SHAPE, (n, C)
    assert f(16, 16, 16, 4, 4, 8, 1e-5, 16, 16, 16, None) == DTYPE
    for eps in (-1e-9, float("nan"), float("inf")):
        assert f(16, 16, 16, 0, 4, 8, eps, 16, 16, 16, None) == VALUE
    for i, bad in ((0, 8), (1, 18), (2, 6), (7, 4), (8, 2), (9, 3)):
        a = [16, 16, 16, 0, 4, 8, 1e-5, 16, 16, 16, None]
        a[i] = bad
        assert f(*a) == ALIGN, i
    assert f(None, None, None, 0, 0, 8, 1e-5, None, None, None, None) == OK


def test_layer_norm_backward_refusals(api):
    f = api._lib.layer_norm_bwd
    need = api.dl_layer_norm_bwd_workspace_bytes(4, 8)
    ok = [16, 16, 16, 16, 16, 0, 4, 8, 16, 16, 16, 16, need, None]

    def code(**change):
        a = list(ok)
        for i, v in change.items():
            a[int(i[1:])] = v
        return f(*a)
    for i in (0, 1, 3, 4, 8, 9, 10):                                    # dy, x, mean, rstd, dx; dgamma or dbeta alone
        assert code(**{f"_{i}": None}) == NULL, i
    assert code(_6=-1) == SHAPE and code(_7=0) == SHAPE and code(_5=9) == DTYPE
    for i, bad in ((0, 2), (1, 8), (2, 2), (3, 1), (4, 6), (8, 8), (9, 2), (10, 7), (11, 8)):
        assert code(**{f"_{i}": bad}) == ALIGN, i
    assert code(_11=None) == WORKSPACE and code(_12=need - 1) == WORKSPACE
    with pytest.raises(api.DlError):
        api.dl_layer_norm_bwd_workspace_bytes(4, 0)
    assert api._lib.dl_layer_norm_bwd_workspace_bytes(4, 8, None) == NULL
    assert f(None, None, None, None, None, 0, 0, 8, None, None, None, None, 0, None) == OK


def test_joined_refusals(api):
    fwd, bwd, d = api._lib.dropout_add_layer_norm_fwd, api._lib.dropout_add_layer_norm_bwd, _drop(api)
    assert fwd(16, 16, d, 16, 16, 0, 4, 8, 1e-5, None, 32, 16, 16, None) == NULL
    assert fwd(16, 16, d, 16, 16, 0, 4, 8, 1e-5, 48, 48, 16, 16, None) == UNSUPPORTED        # s and y are one tensor
    assert fwd(16, 16, _drop(api, 2.0), 16, 16, 0, 4, 8, 1e-5, 48, 64, 16, 16, None) == VALUE
    assert fwd(16, 24, d, 16, 16, 0, 4, 8, 1e-5, 48, 64, 16, 16, None) == ALIGN
    assert fwd(16, 16, d, 16, 16, 0, 4, 8, 1e-5, 40, 64, 16, 16, None) == ALIGN
    assert fwd(16, 16, d, 16, 16, 0, -4, 8, 1e-5, 48, 64, 16, 16, None) == SHAPE
    assert fwd(16, 16, d, 16, 16, 7, 4, 8, 1e-5, 48, 64, 16, 16, None) == DTYPE
    need = api.dl_layer_norm_bwd_workspace_bytes(4, 8)
    assert bwd(16, 16, 16, d, 16, 16, 16, 0, 4, 8, None, None, 16, 16, 16, need, None) == NULL
    assert bwd(16, 16, 16, d, 16, 16, 16, 0, 4, 8, 32, 32, 16, 16, 16, need, None) == UNSUPPORTED
    assert bwd(16, 8, 16, d, 16, 16, 16, 0, 4, 8, 32, 48, 16, 16, 16, need, None) == ALIGN
    assert bwd(16, 16, 16, d, 16, 16, 16, 0, 4, 8, 32, 48, 16, 16, 16, need - 1, None) == WORKSPACE
    assert bwd(16, 16, 16, _drop(api, -1.0), 16, 16, 16, 0, 4, 8, 32, 48, 16, 16, 16, need, None) == VALUE


def test_workspace_query_stays_small(api):
    """The sums' workspace: a slab per row at most on small maps, at most a third of a 16-bit tensor on large ones, never empty."""
    for n, C in ((1, 1), (0, 256), (2, 256), (6912, 1024), (110592, 304), (1769472, 256), (208297, 77), (50, 8192), (7, 1 << 20)):
        b = api.dl_layer_norm_bwd_workspace_bytes(n, C)
        assert b >= 8 * C and b % (8 * C) == 0, (n, C)
        assert b <= max(8 * C * min(max(n, 1), 768), 0.35 * 2 * n * C), (n, C, b)


def test_descriptor(api):
    for bad in (dict(p=-0.1, seed=0), dict(p=1.5, seed=0), dict(p=float("nan"), seed=0), dict(p=0.1, seed=-1), dict(p=0.1, seed=1 << 64),
                dict(p=0.1, seed=0, offset=1 << 64), dict(p=0.1, seed=0, step=torch.zeros(1, dtype=torch.int64))):
        with pytest.raises(ValueError):
            api.DropoutDesc(**bad)
    d = copy.deepcopy(api.DropoutDesc(0.25, (1 << 64) - 1, 5))
    c = d._kept._obj
    assert (c.p, c.seed, c.offset, c.step) == (0.25, (1 << 64) - 1, 5, None)


def test_wrapper_refusals(api):
    x, v = torch.zeros(4, 8, dtype=torch.float16), torch.zeros(8)
    d = api.DropoutDesc(0.1, 1)
    for call in (lambda: api.dropout_fwd(x, d), lambda: api.dropout_bwd(x, d), lambda: api.layer_norm_fwd(x, v, v),
                 lambda: api.layer_norm_bwd(x, x, v, v[:4], v[:4]), lambda: api.dropout_add_layer_norm_fwd(x, x, d, v, v),
                 lambda: api.dropout_add_layer_norm_bwd(x, x, x, d, v, v[:4], v[:4])):
        with pytest.raises(ValueError):                                 # host tensors
            call()
    with pytest.raises(TypeError):
        api.layer_norm_fwd(x.double(), v, v)
    for t in (torch.zeros(()), torch.zeros(3, 0)):
        with pytest.raises(ValueError):
            api._rows(t, t.shape)
    assert api._rows(x, x.shape) == (4, 8)
    for bad in (v.half(), v[:7], torch.zeros(16)[::2]):
        with pytest.raises(ValueError):
            api._vectors("gamma", -1, 8, bad)
    assert api._vectors("gamma beta", -1, 8, v, None) == [v.data_ptr(), None]
    with pytest.raises(ValueError):
        api._affine(v, None, -1, 8)


def test_host_path_under_sanitizers(tmp_path):
    from test_sanitizers import ENV, SAN, _build_sanitized_host_library
    lib = _build_sanitized_host_library()
    exe = str(tmp_path / "norm_san")
    subprocess.run(["amdclang", "-O1", "-g", *SAN, "-std=c11", "-Wall", "-o", exe, os.path.join(ROOT, "tests", "norm_sanitize_driver.c"),
                    lib, f"-Wl,-rpath,{os.path.dirname(lib)}"], check=True)
    r = subprocess.run([exe], env=ENV, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "0 wrong status codes" in r.stdout
