"""Linear layers whose products go by the largest tiles, 256 x 256: one round of them over the chip, more than that, and few of
them with K in pieces, in both directions; and long K where there would be many.  Sampled rows and columns against fp64, under the bounds of test_gpu_layers.py.
The workspace is full of NaN before every call: a piece that nobody wrote shows."""
import numpy as np
import pytest

from oracle import block as OB
from paper_1702_02181_amd import fold as F
from tests.block_common import HALF, U, host, ld, torch_type, within
from tests.test_gpu_layers import _out_error, _slope_error

pytestmark = pytest.mark.gpu


def _normal(rows, width, dtype, seed, scale=1.0, pad=0.0):
    """[rows, ld(width)] on the GPU, made there."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randn((rows, ld(width)), generator=g, device="cuda") * scale
    t[:, width:] = pad
    return t.to(torch_type(dtype))


def _some(n, seed):
    """The first and the last ones, those around the tiles' borders and some between."""
    rng = np.random.default_rng(seed)
    fixed = [0, 1, 255, 256, n - 257, n - 256, n - 2, n - 1]
    return np.unique(np.clip(np.r_[fixed, rng.integers(0, n, 10)], 0, n - 1))


def _at(t, rows, width):
    return host(t[rows.tolist()], width)


def _forward(x, W, bias, K, N, act, res, pre, dtype):
    import torch
    M = x.shape[0]
    code = F.FOLD_F32 if dtype == "f32" else F.FOLD_BF16
    n, _ = F.fold_linear_workspace_size(code, M, K, N)
    ws = torch.full((max(n // 4, 4),), float("nan"), device="cuda")
    out = torch.full((M, ld(N)), float("nan"), dtype=x.dtype, device="cuda")
    z = torch.full_like(out, float("nan")) if pre else None
    F.fold_linear(code, M, K, N, x, W, bias, F.ACTIVATIONS[act], res, out, z, ws, n)
    return out, z


# long K: whole (two) and in pieces, each with more than 256 tiles; one round of tiles, K in pieces with few of them, the chain of
# more than 256 in fp32 and bf16
FORWARD = [(10300, 8192, 2048, "bf16"), (5000, 16384, 4096, "bf16"), (4200, 16000, 4099, "bf16"), (1844, 1000, 8190, "bf16"),
           (1555, 8000, 2000, "bf16"), (19129, 100, 1424, "f32"), (17000, 520, 4090, "bf16")]


@pytest.mark.parametrize("M,K,N,dtype", FORWARD)
def test_linear_of_large_tiles(M, K, N, dtype):
    import torch
    x, W = _normal(M, K, dtype, 1, pad=3.0), _normal(N, K, dtype, 2, K ** -0.5)
    r = _normal(M, N, dtype, 3, pad=5.0)
    b = torch.linspace(-1, 1, N, device="cuda")
    rows = _some(M, M)
    xs, Ws, rs = _at(x, rows, K), host(W, K), _at(r, rows, N)
    size = np.abs(xs) @ np.abs(Ws).T
    for act, bias, res, pre in (("none", None, None, False), ("none", b, r, False), ("gelu", b, None, True), ("gelu", b, r, True)):
        want, z = OB.linear(xs, Ws, None if bias is None else host(bias), act, None if res is None else rs)
        out, got = _forward(x, W, bias, K, N, act, res, pre, dtype)
        bz = (K + 8) * U * (size + (0 if bias is None else np.abs(host(bias))))
        within(_at(out, rows, N), want, 1.13 * bz + _out_error(act, z) + (HALF[dtype] + 2 * U) * (np.abs(want) + bz),
               ("out", act, res is not None))
        if pre:
            within(_at(got, rows, N), z, bz + HALF[dtype] * np.abs(z), ("pre", act))
        assert torch.isfinite(out).all() and not out[:, N:].any()


# dx in pieces (few tiles), dW in pieces, one round of tiles of either
BACKWARD = [(1633, 2040, 8190, "bf16"), (7119, 2040, 2000, "bf16"), (4090, 4090, 60, "f32"), (70, 4090, 4090, "f32")]


@pytest.mark.parametrize("M,K,N,dtype", BACKWARD)
def test_linear_backward_of_large_tiles(M, K, N, dtype):
    import torch
    code = F.FOLD_F32 if dtype == "f32" else F.FOLD_BF16
    x, W = _normal(M, K, dtype, 4), _normal(N, K, dtype, 5, K ** -0.5)
    dout, z = _normal(M, N, dtype, 6), _normal(M, N, dtype, 7, 1.5)
    rows, outs = _some(M, M), _some(N, N)
    ax, aw = np.abs(host(x, K)), np.abs(host(W, K))
    _, n = F.fold_linear_workspace_size(code, M, K, N)
    for act, tx, tw in (("none", dtype, dtype), ("gelu", "f32", dtype), ("relu", dtype, "f32")):
        bent = act != "none"
        ws = torch.full((max(n // 4, 4),), float("nan"), device="cuda")
        dx = torch.full((M, ld(K)), float("nan"), dtype=torch_type(tx), device="cuda")
        dW = torch.full((N, ld(K)), float("nan"), dtype=torch_type(tw), device="cuda")
        db, dpre = torch.full((N,), float("nan"), device="cuda"), torch.full_like(z, float("nan")) if bent else None
        F.fold_linear_backward(code, M, K, N, x, W, F.ACTIVATIONS[act], z if bent else None, dout, dpre,
                               F._code(dx.dtype), dx, F._code(dW.dtype), dW, db, 0, ws, n)
        # the rows' part of dx, the outputs' part of dW and db
        want, _, _, dz = OB.linear_backward(_at(x, rows, K), host(W, K), _at(dout, rows, N), act, _at(z, rows, N))
        e = np.abs(_at(dout, rows, N)) * _slope_error(act) + (2 * U + HALF[dtype] if bent else 0) * np.abs(dz)
        s = np.abs(dz) + e
        within(_at(dx, rows, K), want, e @ aw + (N + 8) * U * (s @ aw) + HALF[tx] * (np.abs(want) + e @ aw), ("dx", act))
        do, zo = host(dout)[:, outs], host(z)[:, outs]
        _, want, wantb, dz = OB.linear_backward(host(x, K), _at(W, outs, K), do, act, zo)
        eb = np.abs(do) * _slope_error(act) + (2 * U * np.abs(dz) if bent else 0)
        e = eb + (HALF[dtype] * np.abs(dz) if bent else 0)
        s = np.abs(dz) + e
        eW = e.T @ ax
        within(_at(dW, outs, K), want, eW + (M + 8) * U * (s.T @ ax) + HALF[tw] * (np.abs(want) + eW), ("dW", act))
        within(host(db)[outs], wantb, eb.sum(0) + (M + 8) * U * s.sum(0), ("db", act))
        assert torch.isfinite(dx).all() and torch.isfinite(dW).all() and not dx[:, K:].any() and not dW[:, K:].any()
