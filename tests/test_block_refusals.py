"""The attention block's refusals, on the CPU: every call fails before it would touch a buffer; and the oracle's gradients
against differences."""
import numpy as np
import pytest

from oracle import block as OB
from tests.test_oracle_vocab import F, NULL_STREAM, _Buf, _refused  # noqa: F401  (F is a fixture)


def test_layer_norm_refuses(F):  # noqa: F811
    x, y, v, m, r, d, ws = (_Buf(1 << (20 + k)) for k in range(7))
    odd = _Buf((1 << 20) + 8)

    def norm(dtype=0, rows=4, width=100, x=x, gamma=v, beta=None, eps=1e-5, y=y, mean=m, rstd=r):
        F.fold_layer_norm(dtype, rows, width, x, gamma, beta, eps, y, mean, rstd, NULL_STREAM)

    for kw in (dict(dtype=2), dict(rows=-1), dict(rows=1 << 31), dict(width=0), dict(width=4097), dict(eps=0.0),
               dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=None), dict(y=None), dict(x=odd),
               dict(y=odd), dict(y=_Buf(x.at + 16)), dict(mean=y), dict(rstd=m), dict(gamma=y), dict(mean=x), dict(beta=r)):
        _refused(F, F.FOLD_E_INVALID, norm, **kw)
    norm(rows=0, x=None, y=None)
    assert F.fold_layer_norm_workspace_size(0, 4, 100) == 0  # few rows: one workgroup
    x, y, d = (_Buf(1 << k) for k in (30, 31, 32))
    n = F.fold_layer_norm_workspace_size(0, 4000, 100)
    assert n > 0

    def back(dtype=0, rows=4000, width=100, x=x, gamma=None, mean=m, rstd=r, dyt=0, dy=d, rt=0, res=None, dxt=0, dx=y, dg=v,
             db=None, flags=0, ws=ws, n=n):
        F.fold_layer_norm_backward(dtype, rows, width, x, gamma, mean, rstd, dyt, dy, rt, res, dxt, dx, dg, db, flags, ws, n,
                                   NULL_STREAM)

    for kw in (dict(dtype=-1), dict(rows=-1), dict(width=0), dict(dyt=1), dict(dxt=1), dict(dyt=2), dict(flags=2),
               dict(x=None), dict(mean=None), dict(rstd=None), dict(dy=None), dict(x=odd), dict(dy=odd), dict(dx=odd),
               dict(res=odd), dict(ws=odd), dict(dx=x), dict(dx=_Buf(d.at + 16)), dict(dg=y), dict(dg=m), dict(db=v),
               dict(ws=x), dict(dtype=1, dyt=0, dxt=1, dx=d),
               dict(rt=1, res=_Buf(1 << 34)), dict(dtype=1, rt=0, dxt=1, res=_Buf(1 << 34), dx=_Buf(1 << 34))):
        _refused(F, F.FOLD_E_INVALID, back, **kw)
    _refused(F, F.FOLD_E_MISMATCH, back, n=n - 1)
    _refused(F, F.FOLD_E_MISMATCH, back, ws=None)
    back(dx=None, dg=None, db=None, ws=None, x=None)
    with pytest.raises(F.FoldError):
        F.fold_layer_norm_workspace_size(0, 4, 5000)


def test_linear_refuses(F):  # noqa: F811
    x, W, out, res, pre, b, d, dx, dw, ws = (_Buf(1 << (20 + k)) for k in range(10))
    odd = _Buf((1 << 20) + 4)

    def fwd(dtype=0, rows=4, k=100, n=70, x=x, W=W, bias=b, act=0, res=None, out=out, pre=None):
        F.fold_linear(dtype, rows, k, n, x, W, bias, act, res, out, pre, None, 0, NULL_STREAM)

    for kw in (dict(dtype=2), dict(rows=-1), dict(rows=1 << 31), dict(k=0), dict(k=16385), dict(n=0), dict(n=16385),
               dict(act=4), dict(act=-1), dict(x=None), dict(W=None), dict(out=None), dict(x=odd), dict(W=odd),
               dict(res=odd), dict(out=odd), dict(pre=odd), dict(out=x), dict(out=W), dict(pre=out), dict(pre=res, res=res),
               dict(res=_Buf(out.at + 16)), dict(out=b), dict(rows=(1 << 31) - 1, n=16384)):
        _refused(F, F.FOLD_E_INVALID, fwd, **kw)
    fwd(rows=0, x=None, W=None, out=None)
    _, n = F.fold_linear_workspace_size(0, 4, 100, 70)

    def back(dtype=0, rows=4, k=100, n=70, x=x, W=W, act=2, pre=pre, dout=d, dpre=pre, dxt=0, dx=dx, dwt=0, dw=dw, db=None,
             flags=0, ws=ws, size=n):
        F.fold_linear_backward(dtype, rows, k, n, x, W, act, pre, dout, dpre, dxt, dx, dwt, dw, db, flags, ws, size,
                               NULL_STREAM)

    for kw in (dict(dtype=2), dict(rows=-1), dict(k=0), dict(n=16385), dict(act=9), dict(dxt=1), dict(dwt=1), dict(flags=2),
               dict(dtype=1, dwt=1, flags=1), dict(x=None), dict(W=None), dict(dout=None), dict(pre=None), dict(dpre=None),
               dict(act=0), dict(act=0, pre=None), dict(x=odd), dict(W=odd), dict(pre=odd), dict(dout=odd), dict(dx=odd),
               dict(dw=odd), dict(dx=d), dict(dx=pre, dpre=d), dict(dw=x), dict(db=dw), dict(dpre=x),
               dict(dpre=_Buf(d.at + 16)), dict(dx=dw)):
        _refused(F, F.FOLD_E_INVALID, back, **kw)
    _refused(F, F.FOLD_E_MISMATCH, fwd, rows=80, k=8192, n=64, x=_Buf(1 << 32), W=_Buf(1 << 33))  # few tiles: K in pieces
    _, big = F.fold_linear_workspace_size(0, 4, 4096, 8192)
    assert big > 0  # few rows: K is cut into pieces
    _refused(F, F.FOLD_E_MISMATCH, back, k=4096, n=8192, act=0, pre=None, dpre=None, x=_Buf(1 << 32), W=_Buf(1 << 33),
             dx=_Buf(1 << 34), dw=_Buf(1 << 35), dout=_Buf(1 << 36), ws=_Buf(1 << 37), size=big - 1)


def _difference(f, x, d, h=1e-5):
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


def test_oracle_gradients_against_differences():
    """fp64 throughout: h = 1e-5 leaves some 1e-9 of the values."""
    rng = np.random.default_rng(0)
    x, dy, gamma = rng.standard_normal((3, 7)), rng.standard_normal((3, 7)), rng.standard_normal(7)
    d = rng.standard_normal((3, 7))
    dx, dg, db = OB.layer_norm_backward(x, dy, gamma)
    assert abs(_difference(lambda t: (OB.layer_norm(t, gamma)[0] * dy).sum(), x, d) - (dx * d).sum()) < 1e-7
    e = rng.standard_normal(7)
    assert abs(_difference(lambda t: (OB.layer_norm(x, t, t)[0] * dy).sum(), gamma, e) - ((dg + db) * e).sum()) < 1e-7
    W, b, dout = rng.standard_normal((5, 7)), rng.standard_normal(5), rng.standard_normal((3, 5))
    for act in ("none", "tanh", "gelu", "relu"):
        _, z = OB.linear(x, W, b, act)
        dx, dw, db, _ = OB.linear_backward(x, W, dout, act, z)
        assert abs(_difference(lambda t: (OB.linear(t, W, b, act)[0] * dout).sum(), x, d) - (dx * d).sum()) < 1e-7
        f = rng.standard_normal((5, 7))
        assert abs(_difference(lambda t: (OB.linear(x, t, b, act)[0] * dout).sum(), W, f) - (dw * f).sum()) < 1e-7
        e = rng.standard_normal(5)
        assert abs(_difference(lambda t: (OB.linear(x, W, t, act)[0] * dout).sum(), b, e) - (db * e).sum()) < 1e-7


def test_oracle_attention_gradients_against_differences():
    rng = np.random.default_rng(1)
    a = dict(heads=4, kv_heads=2, head_dim=3, q_ptr=[0, 2, 2, 5], k_ptr=[0, 4, 4], q_rows=[4, 0, 1, 2, 3], k_rows=[5, 1, 0, 3],
             source=[0, 0, 1], mask=[1, 0, 1, 1])
    q, k, v = rng.standard_normal((5, 12)), rng.standard_normal((6, 6)), rng.standard_normal((6, 6))
    out, lse = OB.attend(q, k, v, **a)
    assert not out[1:4].any() and np.isneginf(lse[1:4]).all() and out[[4, 0]].any()
    dout = rng.standard_normal((5, 12))
    got = OB.attend_backward(q, k, v, dout, **a)
    for i, t in enumerate((q, k, v)):
        d = rng.standard_normal(t.shape)
        args = [q, k, v]

        def f(u):
            return (OB.attend(*[u if j == i else args[j] for j in range(3)], **a)[0] * dout).sum()
        assert abs(_difference(f, t, d) - (got[i] * d).sum()) < 1e-7
    assert not got[1][[1, 2, 4]].any() and not got[2][[1, 2, 4]].any()


def test_cross_refuses(F):  # noqa: F811
    """Sizes that a plan refuses before it looks at a list."""
    ok = dict(dtype=0, heads=4, kv_heads=2, head_dim=64, num_seqs=3, num_sources=3, num_queries=10, num_keys=20,
              num_query_rows=10, num_key_rows=20, query_ptr=4096, query_row=None, key_ptr=8192, key_row=None, source=None)

    def create(**kw):
        F.fold_cross_create(F.fold_cross_batch(**dict(ok, **kw)), NULL_STREAM)

    for kw in (dict(dtype=2), dict(heads=0), dict(heads=1025, kv_heads=1025), dict(kv_heads=0), dict(kv_heads=3), dict(head_dim=0),
               dict(head_dim=129), dict(heads=514, kv_heads=2), dict(num_seqs=-1), dict(num_keys=-1), dict(num_queries=-1), dict(num_sources=2),
               dict(num_query_rows=9), dict(num_key_rows=19), dict(query_ptr=None), dict(key_ptr=None),
               dict(heads=1024, kv_heads=1024, num_queries=1 << 21, num_query_rows=1 << 21)):
        _refused(F, F.FOLD_E_INVALID, create, **kw)
    _refused(F, F.FOLD_E_INVALID, F.fold_cross_attend, None, None, 0, None, 0, None, 0, None, 1.0, None, 0, None, None, 0,
             NULL_STREAM)
    _refused(F, F.FOLD_E_INVALID, F.fold_cross_backward, None, None, 0, None, 0, None, 0, None, 1.0, None, 0, None, None, 0,
             None, 0, None, 0, None, 0, None, 0, NULL_STREAM)
    _refused(F, F.FOLD_E_INVALID, F.fold_cross_workspace_size, None)
    F.fold_cross_free(None)
