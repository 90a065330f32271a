"""The attention block where element offsets pass 2^31, and the largest plans."""
import numpy as np
import pytest

from paper_1702_02181_amd import fold as F
from tests.block_common import HALF, U, host, within

pytestmark = pytest.mark.gpu


def _ends(rows, tail, width, seed, dtype):
    """([rows, width] of zeros but for its last `tail` rows, those rows alone)."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    part = torch.randn((tail, width), generator=g, device="cuda").to(dtype)
    full = torch.zeros((rows, width), dtype=dtype, device="cuda")
    full[-tail:] = part
    return full, part


def test_layer_norm_rows_far_out():
    """A row's result depends on nothing but the row: the last rows of a matrix of more than 2^31 elements come out as alone."""
    import torch
    rows, n, tail = 2 ** 21 + 40, 1024, 40
    x, px = _ends(rows, tail, n, 1, torch.bfloat16)
    gamma = torch.linspace(0.5, 2.0, n, device="cuda")
    y, mean, rstd = F.layer_norm(x, n, gamma)
    want = F.layer_norm(px, n, gamma)
    assert all(torch.equal(a[-tail:], b) for a, b in zip((y, mean, rstd), want))
    assert not y[:-tail].any()
    dy, pdy = _ends(rows, tail, n, 2, torch.bfloat16)
    dx, dgamma, dbeta = F.layer_norm_backward(x, n, dy, mean, rstd, gamma, dx=dy)
    w = F.layer_norm_backward(px, n, pdy, want[1], want[2], gamma)
    assert torch.equal(dx[-tail:], w[0]) and not dx[:-tail].any()
    # the zero rows add nothing; the others' sums, in another order: within 2 (40 + 8) u of the terms' magnitudes
    for a, b, t in ((dgamma, w[1], pdy.float() * ((px.float() - want[1][:, None]) * want[2][:, None])), (dbeta, w[2], pdy.float())):
        within(host(a), host(b), 2 * (tail + 8) * U * host(t.abs().sum(0)), "sums")


def test_linear_rows_far_out():
    import torch
    rows, n_in, n_out, tail = 2 ** 21 + 70, 64, 1024, 70
    x, px = _ends(rows, tail, n_in, 3, torch.bfloat16)
    W = torch.randn((n_out, n_in), device="cuda").bfloat16()
    layer = F.Linear(W, torch.full((n_out,), 0.25, device="cuda"), n_in)
    out = layer.forward(x)
    hx, hW = host(px), host(W)
    want = hx @ hW.T + 0.25
    size = np.abs(hx) @ np.abs(hW).T + 0.25
    within(host(out[-tail:]), want, (n_in + 8) * U * size + HALF["bf16"] * np.abs(want) * (1 + U), "out")
    assert (out[:-tail] == 0.25).all()
    del out
    dout, pdo = _ends(rows, tail, n_out, 4, torch.bfloat16)
    dx, dW, db = layer.backward(x, dout)
    hd = host(pdo)
    within(host(dx[-tail:]), hd @ hW, (n_out + 8) * U * (np.abs(hd) @ np.abs(hW)), "dx")
    within(host(dW), hd.T @ hx, (tail + 8) * U * (np.abs(hd).T @ np.abs(hx)), "dW")  # (the zero rows add nothing)
    within(host(db), hd.sum(0), (tail + 8) * U * np.abs(hd).sum(0), "db")
    assert not dx[:-tail].any()


@pytest.mark.parametrize("width", [64, 60])
def test_cross_rows_far_out(width):
    """Columns of a matrix of more than 2^31 elements, its last rows listed: as compact matrices, bit for bit."""
    import torch
    ptr = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    rows, ld, nq, nk = 4200, 2 ** 19, 50, 90
    wide = torch.zeros((rows, ld), dtype=torch.bfloat16, device="cuda")
    at = torch.arange(rows - 100, rows, device="cuda")
    q, k, v, do, out, dq, dk, dv = (wide[:, 1024 * i + ld // 2:1024 * i + ld // 2 + 2 * width] for i in range(8))
    compact = []
    for m in (q, k, v, do):
        part = torch.randn((100, 2 * width), device="cuda").bfloat16()
        m[at] = part
        compact.append(torch.nn.functional.pad(part, (0, 128 - 2 * width)))
    near = F.CrossAttention(2, width, ptr(0, nq), ptr(0, nk), ptr(*range(100 - nq, 100)), ptr(*range(100 - nk, 100)), 100, 100)
    far = F.CrossAttention(2, width, ptr(0, nq), ptr(0, nk), at[-nq:].int(), at[-nk:].int(), rows, rows)
    wo, wl = near.forward(*compact[:3])
    wg = near.backward(*compact[:3], wo, wl, compact[3])
    _, lse = far.forward(q, k, v, out=out)
    far.backward(q, k, v, out, lse, do, dq=dq, dk=dk, dv=dv)
    assert torch.equal(lse[at[-nq:]], wl[-nq:])
    for got, want in zip((out, dq, dk, dv), (wo, *wg)):
        assert torch.equal(got[at], want[:, :2 * width])


def test_plans_of_too_many_tiles_are_refused():
    import torch
    n = 2 ** 24
    ptr = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    with pytest.raises(F.FoldError) as e:
        F.CrossAttention(1, 32, ptr, one, source=torch.zeros(n, dtype=torch.int32, device="cuda"))
    assert e.value.code == F.FOLD_E_INVALID and "tiles" in str(e.value)
