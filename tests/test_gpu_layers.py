"""Parity of layer norm and the linear layers, forward and backward, with the fp64 oracle.

Bounds, from the arithmetic (u = 2^-24; a sum of n terms in any order is within n u of the sum of its terms' magnitudes, to
first order; a result is rounded by at most half a step of its type, 2^-8 of the value in bf16):
  * mean: (n + 2) u mean|x| = m.  A deviation d = x - mean is off by m + u |d|, the variance by 2 m mean|d| + m^2 + (n + 6) u
    var, so rstd by r = half of that over (var + eps), and 4 u (root, reciprocal), relative.  y: |gamma| rstd (|d| (r + 4 u)
    + m) + u (|y| + |beta|) and its rounding.
  * the norm's gradient takes mean and rstd as given: xh is within 3 u |xh|, g within u |g|; mean(g) within (n + 3) u mean|g|,
    mean(g xh) within (n + 7) u mean|g xh|.
  * products: (K + 8) u sum |a| |b|.  tanh is within 4e-7, its slope within 1e-6, Phi within 1.5e-7 + 4 u, so gelu within
    |z| (1.5e-7 + 8 u), its slope within 1e-6 (Phi, and z phi(z) <= 0.25 to some u (z^2 + 4)); the slopes of all of them are
    at most 1.13.  dz enters its products rounded to the layer's type.
"""
import numpy as np
import pytest

from oracle import block as OB
from paper_1702_02181_amd import fold as F
from tests.block_common import HALF, U, dev, host, ld, pads_are_zero, rounded, torch_type, vec, within

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "tanh", "gelu"]


# ---- layer norm -----------------------------------------------------------------------------------------------------

NORMS = [(1, 1, "f32"), (1, 4096, "bf16"), (3, 64, "bf16"), (33, 300, "bf16"), (7, 75, "f32"), (130, 129, "f32"),
         (257, 320, "bf16"), (65, 448, "f32"), (18, 513, "bf16"), (50, 1000, "f32"), (40, 1024, "bf16"), (9, 1537, "f32"),
         (19, 2048, "bf16"), (5, 2300, "bf16"), (6, 4095, "f32"), (2100, 64, "f32"), (3000, 190, "bf16"),
         (70000, 70, "bf16"), (20000, 128, "f32")]


def _norm_case(M, n, dtype, seed=0, shift=3.0):
    rng = np.random.default_rng(seed + M + n)
    x = rounded(rng.standard_normal((M, n)) * np.exp(rng.uniform(-2, 2, (M, 1))) + shift * rng.standard_normal((M, 1)), dtype)
    return x, (1 + 0.3 * rng.standard_normal(n)).astype(np.float32), (0.3 * rng.standard_normal(n)).astype(np.float32), rng


def _norm_bounds(x, gamma, beta, eps, y, rstd, dtype):
    n = x.shape[1]
    x = x.astype(np.float64)
    m = (n + 2) * U * np.abs(x).mean(1)
    d = np.abs(x - x.mean(1, keepdims=True))
    var = (d ** 2).mean(1)
    r = 0.5 * (2 * m * d.mean(1) + m * m + (n + 6) * U * var) / (var + eps) + 4 * U
    g, b = np.abs(1.0 if gamma is None else gamma), np.abs(0.0 if beta is None else beta)
    by = g * rstd[:, None] * (d * (r + 4 * U)[:, None] + m[:, None]) + U * (np.abs(y) + b) + HALF[dtype] * np.abs(y)
    return by, m + U * np.abs(x.mean(1)), rstd * r


@pytest.mark.parametrize("M,n,dtype", NORMS)
def test_layer_norm(M, n, dtype):
    x, gamma, beta, _ = _norm_case(M, n, dtype)
    for g, b, eps in ((gamma, beta, 1e-5), (None, None, 1e-2)):
        want = OB.layer_norm(x, g, b, eps)
        got = F.layer_norm(dev(x, dtype, fill=7.0), n, vec(g), vec(b), eps)
        for what, a, w, bound in zip(("y", "mean", "rstd"), (host(got[0], n), host(got[1]), host(got[2])), want,
                                     _norm_bounds(x, g, b, eps, want[0], want[2], dtype)):
            within(a, w, bound, what)
        pads_are_zero(got[0], n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_norm_in_place_and_without_stats(dtype):
    import torch
    x, gamma, beta, _ = _norm_case(37, 300, dtype)
    want = F.layer_norm(dev(x, dtype), 300, vec(gamma), vec(beta))[0]
    t = dev(x, dtype)
    got = F.layer_norm(t, 300, vec(gamma), vec(beta), stats=False, out=t)
    assert got[0] is t and got[1] is None and got[2] is None and torch.equal(t, want)


def test_layer_norm_of_constant_and_bad_rows():
    """A constant row has no deviation (y = beta); NaN and infinities stay in their own row."""
    import torch
    x = np.random.default_rng(1).standard_normal((6, 100)).astype(np.float32)
    x[1], x[3, 5], x[4, 9] = 2.5, np.nan, np.inf
    beta = np.arange(100, dtype=np.float32)
    y = host(F.layer_norm(dev(x), 100, None, vec(beta))[0], 100)
    assert np.array_equal(y[1], beta) and np.isnan(y[3]).all() and np.isnan(y[4]).all()
    clean = host(F.layer_norm(dev(x[[0, 2, 5]]), 100, None, vec(beta))[0], 100)
    assert np.array_equal(y[[0, 2, 5]], clean)
    assert torch.cuda.is_available()


def _norm_back_bounds(x, dy, gamma, mean, rstd, res, dx, dtype):
    n, M = x.shape[1], x.shape[0]
    xh = np.abs((x.astype(np.float64) - mean[:, None]) * rstd[:, None])
    # the deviation itself is rounded: u |x - mean| against a mean that may be far larger is exact in the subtraction
    g = np.abs(dy * (1.0 if gamma is None else gamma)).astype(np.float64)
    m1, m2 = g.mean(1, keepdims=True), (g * xh).mean(1, keepdims=True)
    b = (n + 3) * U * m1 + xh * (n + 7) * U * m2 + 8 * U * (g + m1 + xh * m2)
    bdx = rstd[:, None] * b + (0 if res is None else 2 * U * np.abs(res)) + (HALF[dtype] + U) * np.abs(dx)
    return bdx, (M + 8) * U * np.abs(dy * xh).sum(0), (M + 8) * U * np.abs(dy).sum(0)


@pytest.mark.parametrize("M,n,dtype", NORMS)
def test_layer_norm_backward(M, n, dtype):
    x, gamma, beta, rng = _norm_case(M, n, dtype, 1)
    _, mean, rstd = OB.layer_norm(x)
    mean, rstd = mean.astype(np.float32), rstd.astype(np.float32)
    for k, (up, down, res) in enumerate([(dtype, dtype, True), ("f32", "f32", False), ("f32", dtype, True)]):
        dy = rounded(rng.standard_normal((M, n)), up)
        r = rounded(rng.standard_normal((M, n)), down) if res else None
        g = None if k == 1 else gamma
        dx, dg, db = OB.layer_norm_backward(x, dy, g, mean=mean, rstd=rstd)
        dx = dx if r is None else dx + r
        got = F.layer_norm_backward(dev(x, dtype, 3.0), n, dev(dy, up, -2.0), vec(mean), vec(rstd), vec(g),
                                    residual=None if r is None else dev(r, down, 5.0), dtype=torch_type(down))
        bounds = _norm_back_bounds(x, dy, g, mean.astype(np.float64), rstd.astype(np.float64), r, dx, down)
        for what, a, w, bound in zip(("dx", "dgamma", "dbeta"), (host(got[0], n), host(got[1]), host(got[2])), (dx, dg, db),
                                     bounds):
            within(a, w, bound, (what, up, down))
        pads_are_zero(got[0], n)


def test_layer_norm_backward_parts():
    """Outputs left out, added to and in place."""
    import torch
    M, n = 77, 200
    x, gamma, _, rng = _norm_case(M, n, "bf16", 2)
    xd, dy = dev(x, "bf16"), dev(rounded(rng.standard_normal((M, n)), "bf16"), "bf16")
    _, mean, rstd = F.layer_norm(xd, n)
    dx, dg, db = F.layer_norm_backward(xd, n, dy, mean, rstd, vec(gamma))
    assert torch.equal(F.layer_norm_backward(xd, n, dy, mean, rstd, vec(gamma), dgamma=None, dbeta=None)[0], dx)
    assert torch.equal(F.layer_norm_backward(xd, n, dy, mean, rstd, vec(gamma), dx=None, dgamma=None)[2], db)
    base = torch.full((n,), 0.5, device="cuda")
    more = base.clone()
    F.layer_norm_backward(xd, n, dy, mean, rstd, vec(gamma), dx=None, dgamma=more, dbeta=None, accumulate=True)
    assert torch.equal(more, base + dg)
    t = dy.clone()
    assert torch.equal(F.layer_norm_backward(xd, n, t, mean, rstd, vec(gamma), dx=t)[0], dx)
    r = dev(rounded(rng.standard_normal((M, n)), "bf16"), "bf16")
    want = F.layer_norm_backward(xd, n, dy, mean, rstd, vec(gamma), residual=r)[0]
    full = F.layer_norm_backward(xd, n, dy, mean, rstd, vec(gamma), residual=r, dtype=torch.float32)[0]
    assert full.dtype == torch.float32 and torch.equal(full.bfloat16(), want)  # one rounding, at the end
    other = F.layer_norm_backward(xd, n, dy, mean, rstd, vec(gamma), residual=r.float(), dtype=torch.bfloat16)[0]
    assert torch.equal(other, want)
    assert torch.equal(F.layer_norm_backward(xd, n, dy, mean, rstd, vec(gamma), residual=r, dx=r)[0], want)


@pytest.mark.parametrize("n", [5, 70])
def test_layer_norm_against_differences(n):
    """The gradient against central differences of the forward pass, both in fp32.  The step h leaves h^2 / 6 times the third
    derivative along the direction (at most 24 rstd^3 |dy|_2 |gamma|_max |d|_2^3, the derivatives of (x - mean) rstd) and
    32 u of the forward's values, over h."""
    rng = np.random.default_rng(n)
    x, dy = rng.standard_normal((4, n)).astype(np.float32), rng.standard_normal((4, n)).astype(np.float32)
    gamma, beta = rng.standard_normal(n).astype(np.float32), rng.standard_normal(n).astype(np.float32)
    d = rng.standard_normal((4, n)).astype(np.float32)
    d /= np.linalg.norm(d, axis=1, keepdims=True)
    h = 2.0 ** -6
    up, down = (host(F.layer_norm(dev(x + s * h * d), n, vec(gamma), vec(beta))[0], n) for s in (1, -1))
    _, mean, rstd = F.layer_norm(dev(x), n)
    dx = host(F.layer_norm_backward(dev(x), n, dev(dy), mean, rstd, vec(gamma))[0], n)
    slope, want = ((up - down) * dy).sum(1) / (2 * h), (dx * d).sum(1)
    r, size = host(rstd), np.linalg.norm(dy, axis=1) * np.abs(gamma).max()
    bound = h * h / 6 * 24 * r ** 3 * size + 32 * U * (np.abs(up) * np.abs(dy)).sum(1) / h
    assert (np.abs(slope - want) <= bound).all(), (slope - want, bound)


# ---- linear layers --------------------------------------------------------------------------------------------------

LAYERS = [(1, 1, 1, "f32"), (1, 1024, 4096, "bf16"), (1, 300, 70, "bf16"), (2, 64, 65, "f32"), (16, 1000, 333, "bf16"),
          (17, 320, 640, "f32"), (33, 75, 1200, "bf16"), (64, 4096, 100, "bf16"), (65, 300, 130, "bf16"), (130, 65, 257, "f32"),
          (257, 512, 300, "bf16"), (300, 1300, 96, "f32"), (1000, 128, 512, "bf16"), (2049, 300, 200, "f32"),
          (4100, 256, 1024, "bf16"), (3, 16384, 40, "bf16"), (70, 40, 16384, "f32"), (16640, 256, 1280, "bf16"),
          (1, 4200, 70, "bf16"), (1, 4096, 130, "f32"), (33, 2100, 200, "f32"), (64, 1088, 130, "bf16"), (17, 2048, 64, "bf16")]


def _layer_case(M, K, N, dtype, seed=0):
    rng = np.random.default_rng(seed + M + 3 * K + 7 * N)
    x = rounded(rng.standard_normal((M, K)), dtype)
    W = rounded(rng.standard_normal((N, K)) / np.sqrt(K), dtype)
    return x, W, (0.3 * rng.standard_normal(N)).astype(np.float32), rng


def _out_error(act, z):
    return {"none": 0.0, "relu": 0.0, "tanh": 4e-7}.get(act, np.abs(z) * (1.5e-7 + 8 * U))


@pytest.mark.parametrize("M,K,N,dtype", LAYERS)
def test_linear(M, K, N, dtype):
    x, W, b, rng = _layer_case(M, K, N, dtype)
    r = rounded(rng.standard_normal((M, N)), dtype)
    size = np.abs(x.astype(np.float64)) @ np.abs(W.astype(np.float64)).T
    for k, act in enumerate(ACTS):
        bias, res = (None if k == 3 else b), (r if k % 2 == 0 else None)
        want, z = OB.linear(x, W, bias, act, res)
        layer = F.Linear(dev(W, dtype), vec(bias), K, act)
        rd = None if res is None else dev(res, dtype, 9.0)
        out, pre = layer.forward(dev(x, dtype, 4.0), rd, pre=True)
        bz = (K + 8) * U * (size + (0 if bias is None else np.abs(bias)))
        within(host(pre, N), z, bz + HALF[dtype] * np.abs(z), ("pre", act))
        bound = 1.13 * bz + _out_error(act, z) + (HALF[dtype] + 2 * U) * (np.abs(want) + bz)
        within(host(out, N), want, bound, ("out", act))
        pads_are_zero(out, N)
        pads_are_zero(pre, N)
        alone = layer.forward(dev(x, dtype, 4.0), rd)
        assert (alone == out).all()


@pytest.mark.parametrize("M", [5, 300])
def test_linear_residual_in_place(M):
    import torch
    x, W, b, rng = _layer_case(M, 128, 200, "bf16")
    r = dev(rounded(rng.standard_normal((M, 200)), "bf16"), "bf16")
    layer = F.Linear(dev(W, "bf16"), vec(b), 128, "gelu")
    want = layer.forward(dev(x, "bf16"), r)
    assert torch.equal(layer.forward(dev(x, "bf16"), r, out=r), want)


def _slope_error(act):
    return 0.0 if act in ("none", "relu") else 1e-6


@pytest.mark.parametrize("M,K,N,dtype", LAYERS)
def test_linear_backward(M, K, N, dtype):
    x, W, _, rng = _layer_case(M, K, N, dtype, 1)
    dout = rounded(rng.standard_normal((M, N)), dtype)
    z = rounded(1.5 * rng.standard_normal((M, N)), dtype)
    ax, aw = np.abs(x.astype(np.float64)), np.abs(W.astype(np.float64))
    for k, act in enumerate(ACTS):
        dx, dw, db, dz = OB.linear_backward(x, W, dout, act, z)
        bent = act != "none"
        tx, tw = (dtype, "f32") if k % 2 else ("f32", dtype)
        layer = F.Linear(dev(W, dtype), None, K, act)
        dpre = dev(np.zeros((M, N)), dtype) if bent else None
        got = layer.backward(dev(x, dtype), dev(dout, dtype), dev(z, dtype, 2.0) if bent else None, dpre=dpre,
                             dx_dtype=torch_type(tx), dw_dtype=torch_type(tw))
        e = np.abs(dout) * _slope_error(act) + (2 * U * np.abs(dz) if bent else 0)  # before its rounding
        ez = e + (HALF[dtype] * np.abs(dz) if bent else 0)
        if bent:
            within(host(dpre, N), dz, ez, ("dpre", act))
            pads_are_zero(dpre, N)
        s = np.abs(dz) + ez
        within(host(got[0], K), dx, ez @ aw + (N + 8) * U * (s @ aw) + HALF[tx] * (np.abs(dx) + ez @ aw), ("dx", act))
        eW = ez.T @ ax
        within(host(got[1], K), dw, eW + (M + 8) * U * (s.T @ ax) + HALF[tw] * (np.abs(dw) + eW), ("dW", act))
        within(host(got[2]), db, e.sum(0) + (M + 8) * U * s.sum(0), ("db", act))
        pads_are_zero(got[0], K)
        pads_are_zero(got[1], K)


@pytest.mark.parametrize("M,dtype", [(20, "f32"), (700, "bf16")])
def test_linear_backward_parts(M, dtype):
    """Outputs left out, added to, and the gradient before the activation written over its inputs."""
    import torch
    x, W, _, rng = _layer_case(M, 100, 200, dtype, 2)
    xd, z = dev(x, dtype), dev(rounded(rng.standard_normal((M, 200)), dtype), dtype)
    dout = dev(rounded(rng.standard_normal((M, 200)), dtype), dtype)
    layer = F.Linear(dev(W, dtype), None, 100, "tanh")
    dx, dW, db = layer.backward(xd, dout, z)
    assert torch.equal(layer.backward(xd, dout, z, dW=None, dbias=None)[0], dx)
    assert torch.equal(layer.backward(xd, dout, z, dx=None, dbias=None)[1], dW)
    assert torch.equal(layer.backward(xd, dout, z, dx=None, dW=None)[2], db)
    for over in (z, dout):
        zz, dd = z.clone(), dout.clone()
        got = layer.backward(xd, dd, zz, dpre=zz if over is z else dd)
        assert all(torch.equal(a, b) for a, b in zip(got, (dx, dW, db)))
    w0, b0 = torch.ones_like(dW), torch.full_like(db, 2.0)
    _, dW2, db2 = layer.backward(xd, dout, z, dW=w0.clone(), dbias=b0.clone(), accumulate=True)
    assert torch.equal(db2, b0 + db) and torch.allclose(dW2[:, :100], (w0 + dW)[:, :100], rtol=0, atol=0)


def test_linear_against_differences():
    """dx, dW and db against central differences of the forward pass in fp32 (tanh: third derivative at most 2, gelu: 2.5; the
    direction moves every z by at most what |d| gives)."""
    M, K, N = 7, 40, 30
    x, W, b, rng = _layer_case(M, K, N, "f32", 3)
    dout = rng.standard_normal((M, N)).astype(np.float32)
    dx_, dW_, db_ = (rng.standard_normal(s).astype(np.float32) for s in ((M, K), (N, K), (N,)))
    dW_ /= np.sqrt(K)
    h = 2.0 ** -7
    for act in ("tanh", "gelu"):
        layer = F.Linear(dev(W), vec(b), K, act)
        _, pre = layer.forward(dev(x), pre=True)
        got = [host(t) for t in layer.backward(dev(x), dev(dout), pre)]
        for what, (ex, ew, eb), want in (("dx", (dx_, 0, 0), (got[0][:, :K] * dx_).sum()),
                                         ("dW", (0, dW_, 0), (got[1][:, :K] * dW_).sum()),
                                         ("db", (0, 0, db_), (got[2] * db_).sum())):
            ends = [host(F.Linear(dev(W + s * h * ew), vec(b + s * h * eb), K, act).forward(dev(x + s * h * ex)), N)
                    for s in (1, -1)]
            dzd = np.abs(ex @ W.T if np.ndim(ex) else 0) + np.abs(x @ dW_.T if np.ndim(ew) else 0) + np.abs(eb)
            slope = ((ends[0] - ends[1]) * dout).sum() / (2 * h)
            noise = (K + 16) * U * (np.abs(x) @ np.abs(W).T + 1) + 1e-6
            bound = h * h / 6 * 2.5 * (np.abs(dout) * dzd ** 3).sum() + (np.abs(dout) * noise).sum() / h
            assert abs(slope - want) <= bound, (act, what, slope, want, bound)


def test_empty_batches():
    import torch
    layer = F.Linear(torch.zeros((40, 64), device="cuda"), None, 33, "relu")
    x, d = torch.zeros((0, 64), device="cuda"), torch.zeros((0, 64), device="cuda")
    assert layer.forward(x).shape == (0, 64)
    dx, dW, db = layer.backward(x, d, d)
    assert dx.shape == (0, 64) and not dW.any() and not db.any()
    y, mean, rstd = F.layer_norm(x, 33)
    assert y.shape == (0, 64) and mean.shape == (0,)
    dx, dg, db = F.layer_norm_backward(x, 33, d, mean, rstd)
    assert dx.shape == (0, 64) and not dg.any() and not db.any()


def test_layer_wrappers_refuse():
    import torch
    W, x = torch.zeros((10, 64), device="cuda"), torch.zeros((4, 64), device="cuda")
    z, v = torch.zeros((4, 64), device="cuda"), torch.zeros(33, device="cuda")
    layer, plain = F.Linear(W, None, 33, "tanh"), F.Linear(W, None, 33)
    for bad in (lambda: F.Linear(W, None, 33, "swish"), lambda: F.Linear(W.half()), lambda: F.Linear(W[:, :32]),
                lambda: F.Linear(W, torch.zeros(9, device="cuda")), lambda: layer.forward(x.bfloat16()),
                lambda: layer.forward(x[:, :48].contiguous()), lambda: layer.forward(x, z[:3]),
                lambda: layer.backward(x, z), lambda: plain.backward(x, z, z), lambda: plain.backward(x, z, dpre=z),
                lambda: layer.backward(x, z, z, accumulate=True), lambda: layer.backward(x, z[:3], z),
                lambda: F.layer_norm(x, 100), lambda: F.layer_norm(x, 33, v[:30]), lambda: F.layer_norm(x.half(), 33),
                lambda: F.layer_norm_backward(x, 33, z, v[:4], v[:3]),
                lambda: F.layer_norm_backward(x, 33, z, v[:4].contiguous(), v[:4].contiguous(), accumulate=True)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: layer.forward(x, out=x), lambda: F.layer_norm(x, 33, eps=0.0),
                lambda: plain.backward(x, z, dW=W, accumulate=True, dbias=None)):
        with pytest.raises(F.FoldError):
            bad()


def _layers(x, up, n, gamma, beta, first, second, stream=None):
    y, mean, rstd = F.layer_norm(x, n, gamma, beta, stream=stream)
    a, pre = first.forward(y, pre=True, stream=stream)
    out = second.forward(a, residual=x, stream=stream)
    da, dW2, db2 = second.backward(a, up, dx_dtype=up.dtype, stream=stream)
    dy, dW1, db1 = first.backward(y, da, pre, dx_dtype=up.dtype, stream=stream)
    dx, dg, db = F.layer_norm_backward(x, n, dy, mean, rstd, gamma, residual=up, stream=stream)
    return [out, dx, dg, db, dW1, db1, dW2, db2]


@pytest.mark.parametrize("M,n,wide,dtype", [(9, 96, 300, "bf16"), (700, 64, 250, "f32"), (3000, 256, 1024, "bf16")])
def test_layers_on_streams_and_in_graphs(M, n, wide, dtype):
    """A norm and a two-layer branch, forward and backward, on a stream of its own and captured: every replay, with eager work
    between, equals the eager results of the inputs it finds."""
    import gc

    import torch
    x, gamma, beta, rng = _norm_case(M, n, dtype, 5)
    first = F.Linear(dev(_layer_case(1, n, wide, dtype)[1], dtype), vec(np.zeros(wide)), n, "gelu")
    second = F.Linear(dev(_layer_case(1, wide, n, dtype)[1], dtype), vec(np.ones(n)), wide)
    xd, up = dev(x, dtype), dev(rounded(rng.standard_normal((M, n)), dtype), dtype)
    a = (up, n, vec(gamma), vec(beta), first, second)
    eager = _layers(xd, *a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = _layers(xd, *a, stream=side)
    side.synchronize()
    assert all(torch.equal(s, t) for s, t in zip(eager, other))
    gc.collect()  # device memory of other tests' garbage, freed by a collection during the recording, would end it
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _layers(xd, *a)
    for it in range(3):
        new = dev(np.roll(x, it, axis=0), dtype)
        want = [t.clone() for t in _layers(new, *a)]
        xd.copy_(new)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(s, t) for s, t in zip(want, out)), it


def test_layers_layout():
    assert ld(300) == F.fold_row_ld(300)
