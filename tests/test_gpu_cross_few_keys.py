"""Gradients of cross attention beside few keys, where dp - delta is far smaller than dp and delta.

delta = sum_j p_j dp_j is summed in fp32 from the first key's dp on.  With u = 2^-24, H half a step of the type, es a score's bound,
rp p's relative one (test_gpu_cross.py): delta is within sum_j p_j (rp |dp_j - base| + (d + 4) u |do|.|v_j|) + (n + 8) u sum_j p_j
(|dp_j| + |base|) + |1 - sum p| |delta - base|, where sum p is 1 but for the largest rp of the row.  The rest is as there: nothing of
out's rounding is left in it."""
import numpy as np
import pytest

from oracle import block as OB
from tests.block_common import HALF, U, host, vec, within
from tests.test_gpu_cross import TINY, Case

pytestmark = pytest.mark.gpu


def _bounds(c):
    """(dq, dk) bounds; every source is read by one sequence."""
    H = HALF[c.dtype] if c.dtype == "bf16" else 0.0
    d, f64 = c.d, np.float64
    q, k, v, do = (a.astype(f64) for a in (c.q, c.k, c.v, c.dout))
    bq, bk, dq, dk = np.zeros_like(q), np.zeros_like(k), np.zeros_like(q), np.zeros_like(k)
    for rows, keys, h, qc, kc in c.pairs():
        n, m = len(keys), len(rows) * (c.heads // c.kv) + 64
        qa, ka, va, da = np.abs(q[rows, qc]), np.abs(k[keys, kc]), np.abs(v[keys, kc]), np.abs(do[rows, qc])
        s = c.scale * (q[rows, qc] @ k[keys, kc].T)
        ref = np.abs(s).max(1, keepdims=True) * 1.4427 + 8
        ep = c.scale * (d + 4) * U * (qa @ ka.T) + U * (4 * np.abs(s) * 1.4427 + 4 * ref + 16)
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        lse = s.max(1, keepdims=True) + np.log(np.exp(s - s.max(1, keepdims=True)).sum(1, keepdims=True))
        rp = ep + (p * ep).sum(1, keepdims=True) + (n + 8) * U + 4 * U * (np.abs(lse) + 1)
        dp, edp = do[rows, qc] @ v[keys, kc].T, (d + 4) * U * (da @ va.T)
        delta, base = (p * dp).sum(1, keepdims=True), dp[:, :1]
        ed = (p * (rp * np.abs(dp - base) + edp + (n + 8) * U * (np.abs(dp) + np.abs(base)))).sum(1, keepdims=True)
        ed = ed + rp.max(1, keepdims=True) * np.abs(delta - base)
        if n == 1:
            ed = edp = np.zeros_like(dp)  # the same number
        ds = c.scale * p * (dp - delta)
        e = c.scale * p * (rp * np.abs(dp - delta) + edp + ed + 4 * U * (np.abs(dp) + np.abs(delta)) * (n > 1))
        e = e + H * (np.abs(ds) + e) + 2 * U * np.abs(ds) + (TINY * (np.abs(dp - delta) + 1) if n > 1 else 0)
        big = np.abs(ds) + e
        cols = np.ix_(keys, range(kc.start, kc.stop))
        bq[rows, qc] += e @ ka + (n + 8) * U * (big @ ka) + n * TINY * (n > 1)
        bk[cols] += e.T @ qa + m * U * (big.T @ qa) + m * TINY * (n > 1)
        dq[rows, qc] += ds @ k[keys, kc]
        dk[cols] += ds.T @ q[rows, qc]
    return tuple(b + (H + 2 * U) * (np.abs(x) + b) for b, x in ((bq, dq), (bk, dk)))


def _run(c):
    plan, (q, k, v), mask = c.plan(), c.tensors(), c.mask_tensor()
    from tests.block_common import dev
    out, lse = plan.forward(q, k, v, mask, c.scale)
    dq, dk, _ = plan.backward(q, k, v, out, lse, dev(c.dout, c.dtype), mask, c.scale)
    return host(dq, c.heads * c.d), host(dk, c.kv * c.d)


# a few lengths each, rows of 32-row tiles that end inside a sequence, groups of heads, longer sources beside them
CASES = [("bf16", 2, 2, 64, [40, 33, 1, 70], [2, 3, 4, 1], 0.0), ("bf16", 6, 2, 50, [35, 9, 64], [5, 31, 64], 0.0),
         ("bf16", 4, 1, 128, [20, 50, 3], [32, 33, 2], 0.0), ("bf16", 1, 1, 16, [300], [17], 0.0),
         ("bf16", 3, 3, 75, [12, 40, 31, 5], [31, 32, 6, 200], 0.4), ("bf16", 8, 8, 60, [8] * 40, [1, 2, 3, 9] * 10, 0.3),
         ("f32", 2, 1, 60, [40, 7, 5], [1, 2, 30], 0.0), ("f32", 4, 4, 128, [33, 2], [1, 1], 0.0)]


@pytest.mark.parametrize("dtype,heads,kv,d,ql,kl,mask", CASES)
def test_gradients_beside_few_keys(dtype, heads, kv, d, ql, kl, mask):
    c = Case(dtype, heads, kv, d, ql, kl, mask=mask, seed=len(ql) + d)
    want = OB.attend_backward(c.q, c.k, c.v, c.dout, c.heads, c.kv, c.d, mask=c.mask, scale=c.scale, **c.lists())
    for what, got, w, b, rows in zip(("dq", "dk"), _run(c), want, _bounds(c), (c.q_rows, c.k_rows)):
        short = {}  # rows whose source has up to 32 keys (fp32: one); the others' bounds are test_gpu_cross.py's
        for i, n in enumerate(kl):
            if n <= (32 if dtype == "bf16" else 1):
                p = c.q_ptr if what == "dq" else c.k_ptr
                short.update(dict.fromkeys(rows[p[i]:p[i + 1]]))
        at = list(short)
        # a single key: w is 0 but for fp64's own rounding
        within(got[at], w[at], b[at] + 1e-13, what)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d,group", [(64, 1), (50, 4), (128, 2), (16, 1)])
def test_one_key_has_no_gradient(dtype, d, group):
    """p = 1 whatever the score: dq and dk are exactly 0, dv is not."""
    import torch
    from tests.block_common import dev
    c = Case(dtype, 2 * group, 2, d, [37, 5, 130], [1, 1, 1], seed=d, spread=3.0)
    plan, (q, k, v) = c.plan(), c.tensors()
    out, lse = plan.forward(q, k, v, None, c.scale)
    dq, dk, dv = plan.backward(q, k, v, out, lse, dev(c.dout, dtype), None, c.scale)
    assert not dq.any() and not dk.any() and dv.any()
    if dtype == "bf16":  # and where the mask leaves one of up to 32
        c = Case(dtype, 2 * group, 2, d, [37, 5, 130], [32, 7, 19], seed=d, spread=3.0)
        c.mask = np.zeros(58, np.uint8)
        c.mask[[31, 32 + 2, 39 + 18]] = 1
        plan, (q, k, v) = c.plan(), c.tensors()
        out, lse = plan.forward(q, k, v, vec(c.mask, np.uint8), c.scale)
        dq, dk, dv = plan.backward(q, k, v, out, lse, dev(c.dout, dtype), vec(c.mask, np.uint8), c.scale)
        assert not dq.any() and not dk.any() and dv.any()
        assert torch.isfinite(lse[torch.from_numpy(c.q_rows).long().cuda()]).all()


def test_masked_rows_beside_few_keys():
    """NaN and infinities in masked keys, and in rows that no key is left for, reach no gradient."""
    import torch
    from tests.block_common import dev
    c = Case("bf16", 2, 2, 64, [20, 6, 9], [6, 3, 30], seed=3)
    c.mask = (np.arange(39) % 3 != 0).astype(np.uint8)
    c.mask[6:9] = 0
    plan, mask, at = c.plan(), vec(c.mask, np.uint8), torch.from_numpy(c.k_rows).long().cuda()
    q, k, v = c.tensors()
    do = dev(c.dout, "bf16")
    out, lse = plan.forward(q, k, v, mask, c.scale)
    want = plan.backward(q, k, v, out, lse, do, mask, c.scale)
    gone = at[torch.from_numpy(c.mask == 0).cuda()]
    k[gone], v[gone] = float("nan"), float("inf")
    lost = torch.from_numpy(c.q_rows[20:26]).long().cuda()
    do[lost], q[lost] = float("nan"), float("-inf")
    got = plan.backward(q, k, v, out, lse, do, mask, c.scale)
    assert all(torch.isfinite(t).all() for t in got)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 50), ("f32", 60)])
def test_workspaces_hold_nothing(dtype, d):
    """Short, long, empty and unread sources and rows without one: a workspace full of NaN changes no bit."""
    import torch
    from paper_1702_02181_amd import fold as F
    from tests.block_common import dev
    c = Case(dtype, 4, 2, d, [40, 7, 600, 1, 33, 90], [5, 0, 400, 32, 1], source=[0, 2, 3, -1, 1, 4], mask=0.2, seed=8)
    plan, (q, k, v), mask, do = c.plan(), c.tensors(), c.mask_tensor(), dev(c.dout, dtype)
    out, lse = plan.forward(q, k, v, mask, c.scale)
    want = [t.clone() for t in (out, lse, *plan.backward(q, k, v, out, lse, do, mask, c.scale))]
    got = [torch.zeros_like(t) for t in want]
    ws = [torch.full((max(n // 4, 4),), float("nan"), device="cuda") for n in plan.ws_bytes]
    ld = lambda t: t.stride(0)  # noqa: E731
    F.fold_cross_attend(plan.handle, q, ld(q), k, ld(k), v, ld(v), mask, c.scale, got[0], ld(got[0]), got[1], ws[0], plan.ws_bytes[0])
    F.fold_cross_backward(plan.handle, q, ld(q), k, ld(k), v, ld(v), mask, c.scale, got[0], ld(got[0]), got[1], do, ld(do), got[2],
                          ld(got[2]), got[3], ld(got[3]), got[4], ld(got[4]), ws[1], plan.ws_bytes[1])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert not any(torch.isnan(t).any() for t in got)
