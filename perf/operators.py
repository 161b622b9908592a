"""Timed workloads of the normalisation and dropout operators on [pixels, channels] tensors.

  layer_norm              y = (x - mean) * rstd * gamma + beta over the channels of each pixel, and its backward pass
                          with the gradients of gamma and beta
  dropout                 elements dropped by a counter-based generator (no mask is stored), with a residual added or not,
                          and its backward pass
  dropout_add_layer_norm  s = residual + dropout(x), y = layer_norm(s) in one pass, and its backward pass

``listed()`` holds the fixed cases, ``draw(rng)`` makes one more of the same ranges, ``prepare(case, seed)`` builds what a
program has in hand before the call, ``run(state)`` makes one pass: in plain 32-bit torch operations where ``own`` is false,
through ``paper_1810_01993_amd.api`` where it is true.  ``work(case)`` counts the bytes and operations that a pass cannot do
without, ``exact(case, seed)`` gives the outputs in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
SIZES = {"f16": 2, "bf16": 2, "f32": 4}
EPS = 1e-5


# ---- the cases ---------------------------------------------------------------
def _case(op, rows, C, dtype, p=0.0, residual=False):
    return {"op": op, "rows": rows, "C": C, "dtype": dtype, "p": p, "residual": residual}


def listed():
    return [
        # inference, the image-pool branch of the atrous pyramid: one pooled pixel of each of two images; latency alone
        dict(_case("layer_norm_fwd", 2, 256, "f16"), name="ln_fwd_pool"),
        # a residual block at output stride 16, two images: the shape most of an encoder's norms have
        dict(_case("layer_norm_fwd", 2 * 48 * 72, 1024, "bf16"), name="ln_fwd_os16"),
        # a decoder layer at full resolution, two images: 906 MB in, 906 MB out, beyond every cache
        dict(_case("layer_norm_fwd", 2 * 768 * 1152, 256, "f16"), name="ln_fwd_fullres"),
        # the decoder's concatenated channels at output stride 4: rows that are not whole 128-byte lines
        dict(_case("layer_norm_bwd", 2 * 192 * 288, 304, "f16"), name="ln_bwd_concat"),
        # the encoder's widest norm, trained in fp32: a wide gradient of gamma over few rows
        dict(_case("layer_norm_bwd", 2 * 48 * 72, 2048, "f32"), name="ln_bwd_os16"),
        # an odd-sized region with an odd channel count: nothing is aligned
        dict(_case("layer_norm_bwd", 361 * 577, 77, "bf16"), name="ln_bwd_odd"),
        # dropout after a dense layer of the second network (32 new channels at full resolution)
        dict(_case("dropout_fwd", 2 * 768 * 1152, 32, "f16", 0.2), name="dropout_fwd_dense"),
        # the way back through dropout in fp32, an odd number of elements
        dict(_case("dropout_bwd", 361 * 577, 77, "f32", 0.1), name="dropout_bwd_odd"),
        # a pooled map through a residual block's tail with dropout: a small call
        dict(_case("dropout_fwd", 24 * 36, 256, "bf16", 0.1, True), name="dropout_fwd_small"),
        # the tail of a residual block and the next one's norm, output stride 4
        dict(_case("dropout_add_layer_norm_fwd", 2 * 192 * 288, 256, "bf16", 0.1, True), name="daln_fwd_os4"),
        # inference-sized map of a tile through the same, small
        dict(_case("dropout_add_layer_norm_bwd", 45 * 67, 512, "f16", 0.1, True), name="daln_bwd_small"),
        # backward of the same at output stride 2, two images
        dict(_case("dropout_add_layer_norm_bwd", 2 * 384 * 576, 256, "bf16", 0.1, True), name="daln_bwd_os2"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


OPS = ("layer_norm_fwd", "layer_norm_bwd", "dropout_fwd", "dropout_bwd", "dropout_add_layer_norm_fwd",
       "dropout_add_layer_norm_bwd")


def draw(rng):
    """One pixel to a full-resolution map, 8 to 8192 channels, half of the counts as they come and half multiples of 8."""
    op = rng.choice(OPS)
    C = _log(rng, 8, 8192)
    if rng.random() < 0.5:
        C = C // 8 * 8
    dtype = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
    cap = 1 << (27 if op.startswith("layer_norm") else 26)
    rows = _log(rng, 1, min(2 * 768 * 1152, cap // C))
    p = 0.0 if op.startswith("layer_norm") else rng.choice([0.05, 0.1, 0.2, 0.35, 0.5])
    residual = op.startswith("dropout_add") or (op == "dropout_fwd" and rng.random() < 0.5)
    return _case(op, rows, C, dtype, p, residual)


# ---- inputs ------------------------------------------------------------------
def _inputs(case, seed):
    op, n, C, dt = case["op"], case["rows"], case["C"], DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, dtype=dt):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype)
    st = {"op": op, "n": n, "C": C, "p": case["p"], "seed": (1810019930 << 20) + seed, "offset": 3 + seed % 1000}
    if op.endswith("fwd"):
        st["x"] = normal((n, C))
    else:
        st["dy"] = normal((n, C))
    if op.startswith("layer_norm") or op.startswith("dropout_add"):
        st["gamma"] = 1 + 0.1 * normal(C, torch.float32)
        st["beta"] = 0.1 * normal(C, torch.float32)
        centre = (0.5 * normal(C, torch.float32)).to(dt)
        if op == "layer_norm_fwd":
            st["x"] += centre
        if op.endswith("bwd"):
            name = "x" if op.startswith("layer_norm") else "s"
            st[name] = normal((n, C)) + centre
            st["mean"], st["rstd"] = _stats(st[name])
    if case["residual"] and op.endswith("fwd"):
        st["residual"] = normal((n, C))
        if op.startswith("dropout_add"):
            st["residual"] += centre
    if op == "dropout_add_layer_norm_bwd":
        st["ds"] = normal((n, C))
    return st


def prepare(case, seed):
    """Activations of unit spread round a mean of their own per channel, upstream gradients N(0, 1), gamma near 1 and beta near
    0 in fp32 as an optimizer keeps them; the mean and 1/deviation of each row that the forward pass has left for the backward
    pass; the generator's seed and the number of the call.  The kernels' outputs and workspace are the program's own, made
    once."""
    st = _inputs(case, seed)
    if own:
        op, n, C, dt = case["op"], case["rows"], case["C"], DTYPES[case["dtype"]]
        from paper_1810_01993_amd import api
        st["api"] = api
        new = lambda: torch.empty((n, C), device="cuda", dtype=dt)                                   # noqa: E731
        vec = lambda k: torch.empty(k, device="cuda", dtype=torch.float32)                           # noqa: E731
        if case["p"] > 0:
            st["drop"] = api.DropoutDesc(case["p"], st["seed"], st["offset"])
        if op.endswith("layer_norm_fwd"):
            st["out"] = dict(y=new(), mean=vec(n), rstd=vec(n))
            if op.startswith("dropout"):
                st["out"]["s"] = new()
        elif op.endswith("layer_norm_bwd"):
            st["out"] = dict(dgamma=vec(C), dbeta=vec(C), dx=new())
            if op.startswith("dropout"):
                st["out"]["dresidual"] = new()
            nb = api.dl_layer_norm_bwd_workspace_bytes(n, C)
            st["out"]["workspace"] = torch.empty(max(nb, 16), device="cuda", dtype=torch.uint8)
        else:
            st["out"] = dict(y=new()) if op == "dropout_fwd" else dict(dx=new())
    return st


def _stats(x):
    f = x.float()
    mean = f.mean(-1)
    f -= mean[:, None]
    return mean, torch.rsqrt((f * f).mean(-1) + EPS)


# ---- the plain form ----------------------------------------------------------
_M32 = 0xFFFFFFFF


def _keep(st, n, device):
    """keep[i] for the flat elements 0..n-1: Philox4x32-10 keyed by the seed on counter (i // 8, offset); element i owns the
    16-bit field i % 8 of the 128 bits, kept where that is at least 65536 * p."""
    i = torch.arange((n + 7) // 8, device=device, dtype=torch.int64)
    c = [i & _M32, i >> 32, torch.full_like(i, st["offset"] & _M32), torch.full_like(i, st["offset"] >> 32)]
    k0, k1 = st["seed"] & _M32, st["seed"] >> 32
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57                       # 64-bit products, the sign bit included
        c = [((b >> 32) & _M32) ^ c[1] ^ k0, b & _M32, ((a >> 32) & _M32) ^ c[3] ^ k1, a & _M32]
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    u = torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], dim=1).reshape(-1)[:n]
    return u >= round(st["p"] * 65536)


def _dropped(st, v):
    t = round(st["p"] * 65536)
    keep = _keep(st, v.numel(), v.device).reshape(v.shape)
    return torch.where(keep, v * (65536 / (65536 - t)), torch.zeros((), device=v.device))


def _norm(x, gamma, beta):
    f = x.float()
    mean = f.mean(-1, keepdim=True)
    d = f - mean
    rstd = torch.rsqrt((d * d).mean(-1, keepdim=True) + EPS)
    return (d * rstd * gamma + beta).to(x.dtype), mean[:, 0], rstd[:, 0]


def _norm_bwd(dy, x, gamma, mean, rstd):
    g, r = dy.float(), rstd[:, None]
    h = (x.float() - mean[:, None]) * r
    dgamma, dbeta = (g * h).sum(0), g.sum(0)
    g = g * gamma
    dx = r * (g - g.mean(-1, keepdim=True) - h * (g * h).mean(-1, keepdim=True))
    return dx, dgamma, dbeta


def _plain(st):
    op = st["op"]
    if op == "layer_norm_fwd":
        return _norm(st["x"], st["gamma"], st["beta"])
    if op == "layer_norm_bwd":
        dx, dgamma, dbeta = _norm_bwd(st["dy"], st["x"], st["gamma"], st["mean"], st["rstd"])
        return dx.to(st["dy"].dtype), dgamma, dbeta
    if op == "dropout_fwd":
        v = _dropped(st, st["x"].float())
        return (v + st["residual"].float() if "residual" in st else v).to(st["x"].dtype)
    if op == "dropout_bwd":
        return _dropped(st, st["dy"].float()).to(st["dy"].dtype)
    if op == "dropout_add_layer_norm_fwd":
        s = (st["residual"].float() + _dropped(st, st["x"].float())).to(st["x"].dtype)
        return (s, *_norm(s, st["gamma"], st["beta"]))
    ds, dgamma, dbeta = _norm_bwd(st["dy"], st["s"], st["gamma"], st["mean"], st["rstd"])
    ds = st["ds"].float() + ds
    return ds.to(st["dy"].dtype), _dropped(st, ds).to(st["dy"].dtype), dgamma, dbeta


# ---- one pass ----------------------------------------------------------------
def run(st):
    """One pass.  Outputs: forward of a norm (s, if joined,) y, mean, rstd; backward (dresidual, if joined,) dx, dgamma, dbeta;
    dropout y or dx."""
    if not own:
        return _plain(st)
    op, api, out = st["op"], st["api"], st["out"]
    if op == "layer_norm_fwd":
        return api.layer_norm_fwd(st["x"], st["gamma"], st["beta"], EPS, **out)
    if op == "layer_norm_bwd":
        return api.layer_norm_bwd(st["dy"], st["x"], st["gamma"], st["mean"], st["rstd"], **out)
    if op == "dropout_fwd":
        return api.dropout_fwd(st["x"], st["drop"], residual=st.get("residual"), **out)
    if op == "dropout_bwd":
        return api.dropout_bwd(st["dy"], st["drop"], **out)
    if op == "dropout_add_layer_norm_fwd":
        return api.dropout_add_layer_norm_fwd(st["x"], st["residual"], st["drop"], st["gamma"], st["beta"], EPS, **out)
    return api.dropout_add_layer_norm_bwd(st["dy"], st["ds"], st["s"], st["drop"], st["gamma"], st["mean"], st["rstd"], **out)


def work(case):
    """Each tensor once; 4-byte statistics per row and parameters per channel; 32-bit operations on the elements (the
    generator's integer operations are not counted)."""
    op, n, C = case["op"], case["rows"], case["C"]
    tensors, rows, channels, ops = {"layer_norm_fwd": (2, 2, 2, 8), "layer_norm_bwd": (3, 2, 3, 15), "dropout_fwd": (2, 0, 0, 1),
                                    "dropout_bwd": (2, 0, 0, 1), "dropout_add_layer_norm_fwd": (4, 2, 2, 10),
                                    "dropout_add_layer_norm_bwd": (5, 2, 3, 17)}[op]
    if op == "dropout_fwd" and case["residual"]:
        tensors, ops = 3, 2
    return {"bytes": n * C * tensors * SIZES[case["dtype"]] + 4 * n * rows + 4 * C * channels, "flops": n * C * ops}


# ---- the definition in 64 bits ------------------------------------------------
def _exact_keep(seed, offset, p, n):
    """As above, on the host in unsigned 64-bit numbers, one round written out on arrays of words."""
    lo = np.uint64(_M32)
    s32 = np.uint64(32)
    block = np.arange((n + 7) // 8, dtype=np.uint64)
    x0, x1 = block & lo, block >> s32
    x2, x3 = np.full_like(block, offset & _M32), np.full_like(block, offset >> 32)
    for r in range(10):
        ka = np.uint64(((seed & _M32) + r * 0x9E3779B9) & _M32)
        kb = np.uint64(((seed >> 32) + r * 0xBB67AE85) & _M32)
        pa, pb = np.uint64(0xD2511F53) * x0, np.uint64(0xCD9E8D57) * x2
        x0, x1, x2, x3 = (pb >> s32) ^ x1 ^ ka, pb & lo, (pa >> s32) ^ x3 ^ kb, pa & lo
    words = np.stack([x0, x1, x2, x3], axis=1).astype("<u4")
    return np.ascontiguousarray(words).view("<u2").reshape(-1)[:n] >= int(np.rint(p * 65536))


def exact(case, seed):
    op, n, C, p = case["op"], case["rows"], case["C"], case["p"]
    if p > 0 and n * C > 120_000_000:                  # the generator runs on the host: seconds
        return None
    st = _inputs(case, seed)
    if p > 0:
        keep = torch.from_numpy(_exact_keep(st["seed"], st["offset"], p, n * C)).cuda().reshape(n, C)
        scale = 1.0 / (1.0 - float(np.rint(p * 65536)) / 65536.0)
    outs, sums = [], [torch.zeros(C, dtype=torch.float64, device="cuda") for _ in range(2)]
    step = max(1, (1 << 25) // C)                      # rows at a time
    for a in range(0, n, step):
        part = slice(a, min(n, a + step))

        def wide(name):
            return st[name][part].double()
        if op == "dropout_bwd":
            outs.append([torch.where(keep[part], scale * wide("dy"), 0.0)])
            continue
        if op == "layer_norm_fwd":
            s = wide("x")
            row = []
        elif op.endswith("fwd"):
            s = torch.where(keep[part], scale * wide("x"), 0.0)
            if "residual" in st:
                s = s + wide("residual")
            row = [s]
            s = s.to(DTYPES[case["dtype"]]).double()   # the norm is that of the stored sum
        if op == "dropout_fwd":
            outs.append(row)
            continue
        if op.endswith("fwd"):
            mean = s.sum(1) / C
            rstd = 1.0 / torch.sqrt(((s - mean[:, None]) ** 2).sum(1) / C + EPS)
            y = (s - mean[:, None]) * rstd[:, None] * st["gamma"].double() + st["beta"].double()
            outs.append(row + [y, mean, rstd])
            continue
        hat = (wide("x" if op == "layer_norm_bwd" else "s") - st["mean"][part].double()[:, None]) * wide("rstd")[:, None]
        up = wide("dy")
        sums[0] += (up * hat).sum(0)
        sums[1] += up.sum(0)
        up = up * st["gamma"].double()
        down = (up - (up.sum(1)[:, None] + hat * (up * hat).sum(1)[:, None]) / C) * st["rstd"][part].double()[:, None]
        if op == "layer_norm_bwd":
            outs.append([down])
        else:
            down = down + wide("ds")
            outs.append([down, torch.where(keep[part], scale * down, 0.0)])
    res = [torch.cat(t) for t in zip(*outs)]
    if op.endswith("layer_norm_bwd"):
        res += sums
    return res[0] if len(res) == 1 else tuple(res)
