"""Parity of cross attention, forward and backward, with the fp64 oracle.

Bounds, from the arithmetic (u = 2^-24; H half a step of the type, 2^-8 in bf16; sums of n terms within n u of the sum of their
magnitudes, to first order).  Per pair of a query and a key:
  * the score is within es = scale (d + 4) u |q|.|k|; its exponent, one fma against the row's reference m in base 2, adds
    u (4 |s| + 4 |m| + 16) (the exponential's two ulp among it): ep in all.  A row's sum of n terms adds (n + 8) u.
  * p is rounded to bf16 before it meets v: r = ep + sum p ep + (n + 8) u (+ H).  o: sum p |v| (r + (n + 2) u) and its rounding;
    lse: sum p ep + (n + 8) u + 4 u |lse|.
  * the gradient starts from lse and the rounded o: p is within rp = ep + the lse's bound, delta within |do|.(o's bound) + (d + 4)
    u |do|.|o|, dp within (d + 4) u |do|.|v|; ds = scale p (dp - delta) within scale p (rp |dp - delta| + those + 4 u (|dp| +
    |delta|)), and H of it where it meets k and q; sums of n terms and the result's rounding as above.
  * below fp32's smallest normal value, t = 2^-126, a result may be 0: p and each product of the sums within t on top.
"""
import numpy as np
import pytest

from oracle import block as OB
from paper_1702_02181_amd import fold as F
from tests.block_common import HALF, U, dev, host, ld, rounded, torch_type, vec, within

pytestmark = pytest.mark.gpu

TINY = 2.0 ** -126


class Case:
    """Sequences of the given lengths; rows of larger matrices in random order (listed) or as they come."""

    def __init__(self, dtype, heads, kv_heads, d, ql, kl, source=None, mask=0.0, listed=True, packed=False, seed=0, scale=None,
                 spread=1.0):
        rng = self.rng = np.random.default_rng(seed)
        self.dtype, self.heads, self.kv, self.d, self.packed = dtype, heads, kv_heads, d, packed
        self.q_ptr, self.k_ptr = np.r_[0, np.cumsum(ql)].astype(np.int32), np.r_[0, np.cumsum(kl)].astype(np.int32)
        nq, nk = int(self.q_ptr[-1]), int(self.k_ptr[-1])
        self.nq, self.nk = nq, nk
        self.NQ, self.NK = (nq + 5, nk + 3) if listed else (nq, nk)
        self.q_rows = rng.permutation(self.NQ)[:nq].astype(np.int32) if listed else None
        self.k_rows = rng.permutation(self.NK)[:nk].astype(np.int32) if listed else None
        self.source = None if source is None else np.asarray(source, np.int32)
        self.mask = (rng.random(nk) >= mask).astype(np.uint8) if mask > 0 else None
        self.scale = d ** -0.5 if scale is None else scale
        self.q = rounded(spread * rng.standard_normal((self.NQ, heads * d)), dtype)
        self.k, self.v = (rounded(rng.standard_normal((self.NK, kv_heads * d)), dtype) for _ in range(2))
        self.dout = rounded(rng.standard_normal((self.NQ, heads * d)), dtype)

    def lists(self):
        return dict(q_ptr=self.q_ptr, k_ptr=self.k_ptr, q_rows=self.q_rows, k_rows=self.k_rows, source=self.source)

    def plan(self):
        return F.CrossAttention(self.heads, self.d, vec(self.q_ptr, np.int32), vec(self.k_ptr, np.int32),
                                vec(self.q_rows, np.int32), vec(self.k_rows, np.int32), self.NQ, self.NK,
                                vec(self.source, np.int32), self.kv, torch_type(self.dtype))

    def tensors(self, fill=0.0):
        q, w = dev(self.q, self.dtype, fill), self.kv * self.d
        if self.packed:
            both = dev(np.concatenate([self.k, self.v], 1), self.dtype, fill)
            return q, both[:, :w], both[:, w:2 * w]
        return q, dev(self.k, self.dtype, fill), dev(self.v, self.dtype, fill)

    def mask_tensor(self):
        return vec(self.mask, np.uint8)

    def pairs(self):
        """Per query sequence with keys, per head: rows, keys, columns of q and of k."""
        for rows, keys in OB._pairs(self.q_ptr, self.k_ptr, self.q_rows, self.k_rows, self.source, self.mask):
            if len(keys) == 0 or len(rows) == 0:
                continue
            for h in range(self.heads):
                g = h // (self.heads // self.kv)
                yield rows, keys, h, slice(h * self.d, (h + 1) * self.d), slice(g * self.d, (g + 1) * self.d)

    def bounds(self):
        """(out, lse, dq, dk, dv) bounds of the listed rows and keys."""
        H = HALF[self.dtype] if self.dtype == "bf16" else 0.0
        d, f64 = self.d, np.float64
        q, k, v, do = (a.astype(f64) for a in (self.q, self.k, self.v, self.dout))
        bo, bl = np.zeros_like(q), np.zeros((self.NQ, self.heads))
        bq, bk, bv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
        dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
        reads = {}
        for rows, keys, h, c, g in self.pairs():
            n = len(keys)
            reads[int(keys[0])] = reads.get(int(keys[0]), 0) + len(rows)
        for rows, keys, h, c, g in self.pairs():
            n, m = len(keys), reads[int(keys[0])] + 64
            qa, ka, va, da = np.abs(q[rows, c]), np.abs(k[keys, g]), np.abs(v[keys, g]), np.abs(do[rows, c])
            s = self.scale * (q[rows, c] @ k[keys, g].T)
            ref = np.abs(s).max(1, keepdims=True) * 1.4427 + 8
            ep = self.scale * (d + 4) * U * (qa @ ka.T) + U * (4 * np.abs(s) * 1.4427 + 4 * ref + 16)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            o = p @ v[keys, g]
            mean = (p * ep).sum(1, keepdims=True)
            r = ep + mean + (n + 8) * U + H
            b = (p * (r + (n + 2) * U) + TINY) @ va + n * TINY
            bo[rows, c] = b + (H + U) * (np.abs(o) + b)
            lse = s.max(1) + np.log(np.exp(s - s.max(1, keepdims=True)).sum(1))
            bl[rows, h] = mean[:, 0] + (n + 8) * U + 4 * U * (np.abs(lse) + 1)
            rp = ep + bl[rows, h][:, None]
            dp, delta = do[rows, c] @ v[keys, g].T, (do[rows, c] * o).sum(1, keepdims=True)
            ed = (da * bo[rows, c]).sum(1, keepdims=True) + (d + 4) * U * (da * np.abs(o)).sum(1, keepdims=True)
            size = np.abs(dp - delta)
            e = self.scale * p * (rp * size + (d + 4) * U * (da @ va.T) + ed + 4 * U * (np.abs(dp) + np.abs(delta)))
            ds = self.scale * p * (dp - delta)
            e = e + H * (np.abs(ds) + e) + 2 * U * np.abs(ds) + TINY * (self.scale * size + 1)
            big = np.abs(ds) + e
            bq[rows, c] += e @ ka + (n + 8) * U * (big @ ka) + n * TINY
            cols = np.ix_(keys, range(g.start, g.stop))
            bk[cols] += e.T @ qa + m * U * (big.T @ qa) + m * TINY
            bv[cols] += (p * (rp + H) + TINY).T @ da + m * U * (p.T @ da) + m * TINY
            dq[rows, c] += ds @ k[keys, g]
            dk[cols] += ds.T @ q[rows, c]
            dv[cols] += p.T @ do[rows, c]
        return bo, bl, *(b + (H + 2 * U) * (np.abs(x) + b) for b, x in ((bq, dq), (bk, dk), (bv, dv)))


def check(case):
    import torch
    c = case
    kw = dict(mask=c.mask, scale=c.scale, **c.lists())
    want, wl = OB.attend(c.q, c.k, c.v, c.heads, c.kv, c.d, **kw)
    grads = OB.attend_backward(c.q, c.k, c.v, c.dout, c.heads, c.kv, c.d, **kw)
    bounds = c.bounds()
    plan, (q, k, v), mask = c.plan(), c.tensors(fill=11.0), c.mask_tensor()
    out, lse = plan.forward(q, k, v, mask, c.scale)
    at = slice(None) if c.q_rows is None else c.q_rows
    wq, wk = c.heads * c.d, c.kv * c.d
    within(host(out, wq)[at], want[at], bounds[0][at], "out")
    within(host(lse)[at], wl[at], bounds[1][at], "lse")
    if c.q_rows is not None:
        rest = np.setdiff1d(np.arange(c.NQ), c.q_rows)
        assert not host(out)[rest].any()
    assert not host(out)[:, wq:].any()
    dout = dev(c.dout, c.dtype, fill=-7.0)
    got = plan.backward(q, k, v, out, lse, dout, mask, c.scale)
    kat = slice(None) if c.k_rows is None else c.k_rows
    for what, t, w, b, rows, width in zip(("dq", "dk", "dv"), got, grads, bounds[2:], (at, kat, kat), (wq, wk, wk)):
        within(host(t, width)[rows], w[rows], b[rows], what)
        assert not host(t)[:, width:].any()
    # parts of the gradient, alone
    assert torch.equal(plan.backward(q, k, v, out, lse, dout, mask, c.scale, dk=None, dv=None)[0], got[0])
    _, dk, dv = plan.backward(q, k, v, out, lse, dout, mask, c.scale, dq=None)
    assert torch.equal(dk, got[1]) and torch.equal(dv, got[2])
    assert torch.equal(plan.backward(q, k, v, out, lse, dout, mask, c.scale, dq=None, dv=None)[1], got[1])
    return plan, out, lse, got


DIMS = [(1, 1, 1), (2, 1, 16), (4, 2, 32), (3, 3, 50), (5, 5, 60), (4, 1, 64), (2, 2, 75), (6, 2, 96), (1, 1, 100), (2, 1, 128)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv,d", DIMS)
def test_shapes_of_heads(dtype, heads, kv, d):
    """Ragged sequences of a batch, some without queries, some without keys, listed rows in any order."""
    check(Case(dtype, heads, kv, d, [5, 0, 33, 1, 70, 2], [17, 9, 0, 1, 130, 65], mask=0.2, seed=d))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("packed,listed", [(False, False), (True, True), (True, False)])
def test_layouts(dtype, packed, listed):
    check(Case(dtype, 4, 4, 64, [40, 129, 3], [64, 63, 65], listed=listed, packed=packed, seed=3))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_one_query_each(dtype, d):
    """The form for single tokens: a row a sequence, heads in groups, up to thousands of keys, which are cut."""
    check(Case(dtype, 8, 2, d, [1] * 7, [1, 2, 31, 33, 700, 1500, 4099], seed=5))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_short_sequences(dtype):
    """More tiles than the chip holds at once, of a few rows each."""
    check(Case(dtype, 8, 8, 96, [2] * 130, [5, 40] * 65, mask=0.1, seed=16))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_long_sequence(dtype):
    """A single row against many keys, and a single key sequence that many rows read: both sides in pieces."""
    plan, *_ = check(Case(dtype, 1, 1, 32, [1], [9000], seed=6))
    assert plan.ws_bytes[0] > 0
    check(Case(dtype, 2, 1, 64, [2500], [40], seed=7))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_shared_sources(dtype):
    """Several query sequences read one source, one reads none, one source is read by nobody: its gradient is 0."""
    c = Case(dtype, 4, 2, 32, [3, 60, 0, 7, 5], [50, 20, 90], source=[2, 0, 0, 2, -1], mask=0.1, seed=8)
    _, out, lse, (_, dk, dv) = check(c)
    unread = c.k_rows[c.k_ptr[1]:c.k_ptr[2]]
    assert not host(dk)[unread].any() and not host(dv)[unread].any()
    rows = c.q_rows[c.q_ptr[4]:]
    assert not host(out)[rows].any() and np.isneginf(host(lse)[rows]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [4, 150])
def test_masks(dtype, rows):
    """A mask that leaves a sequence nothing, one that leaves a single key, one that begins late; NaN, infinities and the
    type's lowest value where keys do not count."""
    import torch
    c = Case(dtype, 2, 2, 64, [rows] * 4, [100, 100, 300, 5], mask=0.5, seed=9)
    c.mask[:100] = 0
    c.mask[100:200] = 0
    c.mask[163] = 1
    c.mask[200:450] = 0
    c.mask[450:] = 1
    plan, out, lse, grads = check(c)
    empty = c.q_rows[:rows]
    assert not host(out)[empty].any() and np.isneginf(host(lse)[empty]).all() and not host(grads[0])[empty].any()
    lowest = float(torch.finfo(torch_type(dtype)).min)
    for value in (float("nan"), float("inf"), -float("inf"), lowest):
        q, k, v = c.tensors()
        off = torch.from_numpy(c.k_rows[c.mask == 0].astype(np.int64)).cuda()
        k[off], v[off] = value, value
        again = plan.forward(q, k, v, c.mask_tensor())
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)
        got = plan.backward(q, k, v, out, lse, dev(c.dout, dtype), c.mask_tensor())
        assert all(torch.equal(a, b) for a, b in zip(got, grads))
    # rows without a key take no part, whatever they hold
    q, k, v = c.tensors()
    dout = dev(c.dout, dtype)
    at = torch.from_numpy(empty.astype(np.int64)).cuda()
    q[at], dout[at] = float("nan"), float("inf")
    got = plan.backward(q, k, v, out, lse, dout, c.mask_tensor())
    assert all(torch.equal(a, b) for a, b in zip(got, grads))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sharp_softmax(dtype):
    """Large scores: one key takes nearly everything, and the reference has to move from tile to tile."""
    c = Case(dtype, 1, 1, 32, [50, 1], [400, 1000], seed=10, spread=12.0, scale=1.0)
    check(c)
    c = Case(dtype, 2, 2, 64, [40], [300], seed=11, scale=2.0)
    order = np.argsort((c.q[c.q_rows[0], :64] * c.k[c.k_rows, :64]).sum(1))  # ascending scores of the first row
    c.k_rows = c.k_rows[order].copy()
    check(c)


def test_bad_rows_stay_alone():
    """NaN in a query makes its own row and heads NaN; in a key that counts, the rows that read it."""
    c = Case("bf16", 2, 2, 32, [20, 20], [40, 40], seed=12)
    plan, out, _, _ = check(c)
    q, k, v = c.tensors()
    q[int(c.q_rows[3]), 2] = float("nan")
    k[int(c.k_rows[45]), 40] = float("nan")
    got, want = host(plan.forward(q, k, v)[0], 64), host(out, 64)
    bad = np.zeros((c.NQ, 64), bool)
    bad[c.q_rows[3], :32] = True
    bad[c.q_rows[20:], 32:] = True
    assert np.isnan(got[bad]).all() and np.array_equal(got[~bad], want[~bad])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_outputs_in_columns_of_wider_matrices(dtype):
    """Strides of their own, addresses that are no multiple of 16 bytes, and what lies beside the columns left alone."""
    import torch
    c = Case(dtype, 3, 3, 40, [30, 2], [70, 10], seed=13)
    plan, out, lse, grads = check(c)
    q, k, v = c.tensors()
    w, dt = 120, torch_type(dtype)

    def slot(rows, shift):
        wide = torch.full((rows, 2 * w + 17), 5.0, dtype=dt, device="cuda")
        return wide, wide[:, shift:shift + w]
    for shift in (8, 9):
        wo, so = slot(c.NQ, shift)
        wq, sq = slot(c.NQ, shift)
        wkv, sk = slot(c.NK, shift)
        sv = wkv[:, shift + w:shift + 2 * w]
        plan.forward(q, k, v, out=so)
        plan.backward(q, k, v, out, lse, dev(c.dout, dtype), dq=sq, dk=sk, dv=sv)
        for got, want, rows in ((so, out, c.q_rows), (sq, grads[0], c.q_rows), (sk, grads[1], c.k_rows),
                                (sv, grads[2], c.k_rows)):
            at = torch.from_numpy(rows.astype(np.int64)).cuda()
            assert torch.equal(got[at], want[at][:, :w])
        assert (wo[:, :shift] == 5).all() and (wo[:, shift + w:] == 5).all()
        assert (wkv[:, :shift] == 5).all() and (wkv[:, shift + 2 * w:] == 5).all()
        rest = torch.from_numpy(np.setdiff1d(np.arange(c.NQ), c.q_rows)).cuda()
        assert (wo[rest] == 5).all() and (wq[rest] == 5).all()


@pytest.mark.parametrize("shape", ["few", "tall"])
def test_against_differences(shape):
    """The gradient against central differences of the forward pass in fp32.  Along a direction that moves every score by at
    most a and every value by at most b, the third derivative of o is at most 6 a^3 |v| + 6 a^2 b (the softmax's cumulants); the
    forward's bound over h is the rest."""
    c = Case("f32", 2, 1, 16, [2] if shape == "few" else [60], [37], listed=False, seed=14)
    plan, out, lse, (dq, dk, dv) = check(c)
    h, rng = 2.0 ** -7, np.random.default_rng(3)
    noise = (c.bounds()[0] * np.abs(c.dout)).sum() / h
    for i, g in enumerate((dq, dk, dv)):
        x = [c.q, c.k, c.v]
        d = rng.choice([-1.0, 1.0], x[i].shape).astype(np.float32) / 16
        ends = []
        for s in (1, -1):
            y = list(x)
            y[i] = x[i] + s * h * d
            ends.append(host(plan.forward(*(dev(t) for t in y))[0], 32))
        slope = ((ends[0] - ends[1]) * c.dout).sum() / (2 * h)
        want = (host(g, d.shape[1]) * d).sum()
        a = 0.25 * max(np.abs(c.q).max(), np.abs(c.k).max()) if i < 2 else 0.0
        b = 1 / 16 if i == 2 else 0.0
        third = (6 * a ** 3 * np.abs(c.v).max() + 6 * a * a * b) * np.abs(c.dout).sum()
        assert abs(slope - want) <= h * h / 6 * third + noise + 1e-6, (i, slope, want)


def _pass(plan, q, k, v, dout, mask, stream=None):
    out, lse = plan.forward(q, k, v, mask, stream=stream)
    return [out, lse, *plan.backward(q, k, v, out, lse, dout, mask, stream=stream)]


@pytest.mark.parametrize("ql,kl", [([1] * 6, [3000] * 6), ([90, 200, 33], [300, 40, 800])])
def test_streams_and_graphs(ql, kl):
    """On a stream of its own, two calls at once, and captured: every replay, with eager work between, equals the eager results
    of the inputs it finds."""
    import gc

    import torch
    c = Case("bf16", 4, 2, 64, ql, kl, mask=0.1, seed=15)
    plan, (q, k, v), mask, dout = c.plan(), c.tensors(), c.mask_tensor(), dev(c.dout, "bf16")
    eager = _pass(plan, q, k, v, dout, mask)
    sides = [torch.cuda.Stream() for _ in range(2)]
    for s in sides:
        s.wait_stream(torch.cuda.current_stream())
    both = [_pass(plan, q, k, v, dout, mask, stream=s) for s in sides]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for got in both for a, b in zip(eager, got))
    gc.collect()  # device memory of other tests' garbage, freed by a collection during the recording, would end it
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _pass(plan, q, k, v, dout, mask)
    for it in range(3):
        new = torch.roll(q, it + 1, 0)
        want = [t.clone() for t in _pass(plan, new, k, v, dout, mask)]
        q.copy_(new)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), it


def test_plans_are_not_made_while_capturing():
    import gc

    import torch
    ptr = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    x = torch.zeros(8, device="cuda")
    gc.collect()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(F.FoldError) as e:
            F.CrossAttention(1, 32, ptr, ptr, num_queries=4, num_keys=4)
        x += 1
    assert e.value.code == F.FOLD_E_INVALID
    graph.replay()
    torch.cuda.synchronize()
    assert (x == 1).all()


def test_malformed_lists_are_refused():
    """Lists that a kernel would follow out of a matrix, or that name a row twice: refused when the plan is made."""
    import torch
    i = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    ok = dict(query_ptr=i(0, 2, 4), key_ptr=i(0, 3, 5), query_rows=i(0, 1, 2, 3), key_rows=i(4, 3, 2, 1, 0))
    F.CrossAttention(2, 32, **ok)
    for kw in (dict(query_ptr=i(0, 3, 2)), dict(query_ptr=i(1, 2, 4)), dict(query_ptr=i(0, 2, 5)), dict(key_ptr=i(0, 6, 5)),
               dict(query_rows=i(0, 1, 2, 4)), dict(query_rows=i(0, -1, 2, 3)), dict(query_rows=i(0, 1, 1, 3)),
               dict(key_rows=i(4, 3, 2, 1, 5)), dict(key_rows=i(4, 3, 3, 1, 0)), dict(source=i(0, 2)), dict(source=i(-2, 0)),
               dict(num_query_rows=3), dict(key_ptr=i(0, 5))):
        with pytest.raises(F.FoldError) as e:
            F.CrossAttention(2, 32, **dict(ok, **kw))
        assert e.value.code == F.FOLD_E_INVALID, kw
    F.CrossAttention(2, 32, **dict(ok, key_ptr=i(0, 5), source=i(0, 0)))
    for kw in (dict(query_ptr=i(0, 2, 4).long()), dict(source=i(0)), dict(query_rows=ok["query_rows"].cpu())):
        with pytest.raises(ValueError):
            F.CrossAttention(2, 32, **dict(ok, **kw))


def test_wrappers_refuse():
    import torch
    ptr = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    plan = F.CrossAttention(2, 32, ptr, ptr, dtype=torch.float32)
    x, lse = torch.zeros((4, 64), device="cuda"), torch.zeros((4, 2), device="cuda")
    plan.forward(x, x, x)
    for bad in (lambda: plan.forward(x.bfloat16(), x, x), lambda: plan.forward(x[:3], x, x), lambda: plan.forward(x[:, :60], x, x),
                lambda: plan.forward(x.t(), x, x), lambda: plan.forward(x, x, x, key_mask=lse), lambda: plan.forward(x.cpu(), x, x),
                lambda: plan.backward(x, x, x, x, lse[:3], x), lambda: plan.backward(x, x, x, x, lse, x[:, :32])):
        with pytest.raises(ValueError):
            bad()
    y = torch.zeros((4, 128), device="cuda")
    for bad in (lambda: plan.forward(x, x, x, scale=0.0), lambda: plan.forward(x, x, x, scale=float("inf")),
                lambda: plan.forward(x, x, x, out=x), lambda: plan.backward(x, x, x, x, lse, x, dq=y[:, :64], dk=y[:, 32:96]),
                lambda: plan.backward(x, x, x, x, lse, x, dq=x)):
        with pytest.raises(F.FoldError):
            bad()
    plan.backward(x, x, x, x, lse, x, dk=y[:, :64], dv=y[:, 64:])


def test_empty_batches():
    import torch
    i = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    none = torch.zeros((0, 64), device="cuda")
    plan = F.CrossAttention(2, 32, i(0), i(0), dtype=torch.float32)
    out, lse = plan.forward(none, none, none)
    assert out.shape == (0, 64) and lse.shape == (0, 2)
    assert [t.shape[0] for t in plan.backward(none, none, none, out, lse, none)] == [0, 0, 0]
    x = torch.ones((3, 64), device="cuda")
    plan = F.CrossAttention(2, 32, i(0, 3), i(0, 0), dtype=torch.float32)
    out, lse = plan.forward(x, none, none)
    assert not out.any() and torch.isneginf(lse).all()
    assert not plan.backward(x, none, none, out, lse, x)[0].any()
    plan = F.CrossAttention(2, 32, i(0, 0), i(0, 3), dtype=torch.float32)
    out, lse = plan.forward(none, x, x)
    dq, dk, dv = plan.backward(none, x, x, out, lse, none)
    assert not dk.any() and not dv.any()


def test_rows_of_a_schedule():
    """Two batches of graphs, their schedules' rows as lists: a chain batch attends to a tree batch."""
    import torch
    from paper_1702_02181_amd import gen
    from paper_1702_02181_amd.runner import DeviceRun
    trees = DeviceRun(gen.config2(seed=3, num_graphs=5, leaves=9, hidden=64), with_backward=False)
    chains = DeviceRun(gen.config2(seed=4, num_graphs=5, leaves=4, hidden=64), with_backward=False)
    trees.forward()
    chains.forward()
    rows = [F.schedule_rows(r.sched) for r in (chains, trees)]
    assert all(np.array_equal(t.cpu().numpy(), r.sched_arrays()["node_pos"]) for t, r in zip(rows, (chains, trees)))
    plan = F.CrossAttention(2, 32, chains.graph_ptr, trees.graph_ptr, *rows, dtype=torch.float32)
    out, _ = plan.forward(chains.h_pool, trees.h_pool, trees.h_pool)
    q, kv = host(chains.h_pool, 64), host(trees.h_pool, 64)
    want, _ = OB.attend(q, kv, kv, 2, 2, 32, chains.w.graph_ptr, trees.w.graph_ptr, *(t.cpu().numpy() for t in rows))
    assert ld(64) == 64 and np.abs(host(out, 64) - want).max() < 1e-5
