"""Pins of the vocabulary head's oracle (oracle.vocab): library routines through automatic differentiation, central
differences, closed forms, and the rows that are no distribution.  Also the host-side argument checks of the library's
entry points, which return before any device work."""
import math
from ctypes import c_void_p

import numpy as np
import pytest
import torch

from oracle import vocab as OV


def _case(seed, M=5, V=17, k=4):
    rng = np.random.default_rng(seed)
    z = 2.0 * rng.standard_normal((M, V))
    tok = rng.integers(0, V, (M, k))
    tok[0, 1] = tok[0, 0]  # the same token twice
    tok[1, 2:] = -1
    tok[2] = V
    t = 3.0 * rng.standard_normal((M, k))
    t[3, 0] = -np.inf
    y = rng.integers(0, V, M)
    y[2], y[4] = -1, V + 3
    return z, tok, t, y


@pytest.mark.parametrize("T,soft,hard", [(1.0, 1.0, 0.0), (2.0, 0.5, 0.5), (0.5, 0.9, 0.1), (3.0, 0.0, 1.0)])
def test_distill_against_automatic_differentiation(T, soft, hard):
    z, tok, t, y = _case(1)
    loss, dz = OV.distill(z, tok, t, y, T, soft, hard, scale=0.3)
    zt = torch.from_numpy(z).requires_grad_()
    total, rows = 0.0, []
    for r in range(z.shape[0]):
        row = torch.zeros((), dtype=torch.float64)
        ok = (tok[r] >= 0) & (tok[r] < z.shape[1]) & np.isfinite(t[r])
        if ok.any():
            q = torch.softmax(torch.from_numpy(t[r][ok]) / T, 0)
            lp = torch.log_softmax(zt[r] / T, 0)[torch.from_numpy(tok[r][ok])]
            row = row + soft * T * T * torch.nn.functional.kl_div(lp, q, reduction="sum")
        if 0 <= y[r] < z.shape[1]:
            row = row + hard * torch.nn.functional.cross_entropy(zt[r][None], torch.tensor([int(y[r])]))
        rows.append(row.item())
        total = total + 0.3 * row
    (g,) = torch.autograd.grad(total, zt)
    np.testing.assert_allclose(loss, rows, rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(dz, g.numpy(), rtol=1e-11, atol=1e-14)


def test_distill_gradient_by_differences():
    z, tok, t, y = _case(2)
    args = dict(T=2.0, soft=0.7, hard=0.4)
    _, dz = OV.distill(z, tok, t, y, scale=1.5, **args)
    rng, h = np.random.default_rng(3), 1e-5
    for _ in range(6):
        d = rng.standard_normal(z.shape)
        up = OV.distill(z + h * d, tok, t, y, **args)[0].sum()
        down = OV.distill(z - h * d, tok, t, y, **args)[0].sum()
        assert abs(1.5 * (up - down) / (2 * h) - (dz * d).sum()) < 1e-8


def test_distill_closed_forms():
    # a teacher with every token and the student's own logits: no loss, no gradient
    z = np.random.default_rng(4).standard_normal((3, 6))
    tok = np.tile(np.arange(6), (3, 1))
    loss, dz = OV.distill(z, tok, z, T=1.7)
    np.testing.assert_allclose(loss, 0, atol=1e-14)
    np.testing.assert_allclose(dz, 0, atol=1e-15)
    # equal logits: the cross entropy of any label is log V
    loss, _ = OV.distill(np.full((1, 8), 3.0), y=np.array([5]), soft=0.0, hard=1.0)
    assert abs(loss[0] - math.log(8)) < 1e-14
    # rows without a target, an empty row and a row with NaN
    zz = np.array([[np.nan] * 3, [-np.inf] * 3, [1.0, np.nan, 0.0]])
    loss, dz = OV.distill(zz, y=np.array([-1, 0, 0]), hard=1.0)
    assert loss[0] == 0 and not dz[0].any() and loss[1] == np.inf and not dz[1].any()
    assert np.isnan(loss[2]) and np.isnan(dz[2]).all()


def test_token_logprobs_against_library_routines():
    rng = np.random.default_rng(5)
    z = 2.0 * rng.standard_normal((4, 33))
    z[1, 5:] = -np.inf
    tok = np.array([[0, 32], [4, -1], [7, 33], [1, 1]])
    logp, ent, top, top_lp = OV.token_logprobs(z, tok, 7)
    lp = torch.log_softmax(torch.from_numpy(z), 1).numpy()
    assert np.allclose(logp, [[lp[0, 0], lp[0, 32]], [lp[1, 4], 0], [lp[2, 7], 0], [lp[3, 1], lp[3, 1]]], rtol=1e-13)
    want = torch.distributions.Categorical(logits=torch.from_numpy(np.where(np.isinf(z), -1e300, z))).entropy().numpy()
    np.testing.assert_allclose(ent, want, rtol=1e-12)
    v, i = torch.from_numpy(lp).topk(7, 1)
    assert np.array_equal(top[[0, 2, 3]], i.numpy()[[0, 2, 3]])
    assert np.array_equal(top[1], [*np.argsort(-z[1, :5]), -1, -1]) and np.isinf(top_lp[1, 5:]).all()
    # ties by the lowest token, an empty row, a row with +inf
    z = np.array([[1.0, 2, 2, 1, 2], [-np.inf] * 5, [0, np.inf, 0, 0, 0]])
    logp, ent, top, top_lp = OV.token_logprobs(z, np.zeros((3, 1), int), 4)
    assert np.array_equal(top, [[1, 2, 4, 0], [-1] * 4, [-1] * 4])
    assert logp[1, 0] == -np.inf and ent[1] == 0 and np.isnan(logp[2, 0]) and np.isnan(ent[2]) and np.isnan(top_lp[2]).all()


def test_head_backward_by_differences():
    rng = np.random.default_rng(6)
    s, W, b, dz = (rng.standard_normal(x) for x in ((3, 4), (5, 4), (5,), (3, 5)))
    f = lambda s, W, b: (OV.head(s, W, b) * dz).sum()  # noqa: E731
    ds, dW, db = OV.head_backward(s, W, dz)
    for x, g, put in ((s, ds, lambda v: f(v, W, b)), (W, dW, lambda v: f(s, v, b)), (b, db, lambda v: f(s, W, v))):
        d = rng.standard_normal(x.shape)
        assert abs((put(x + 1e-6 * d) - put(x - 1e-6 * d)) / 2e-6 - (g * d).sum()) < 1e-8


# ---- argument checks: the calls fail before any device work ---------------------------------------------------------

class _Buf:
    """Stands for a tensor: never dereferenced, the calls fail first."""

    def __init__(self, at=4096):
        self.at = at

    def data_ptr(self):
        return self.at


NULL_STREAM = type("Stream", (), {"cuda_stream": 0})()


@pytest.fixture(scope="module")
def F():
    import os

    from paper_1702_02181_amd import build_lib, fold
    if not os.path.exists(build_lib.LIB):
        build_lib.build()
    return fold


def _refused(F, code, call, *args, **kw):
    with pytest.raises(F.FoldError) as e:
        call(*args, **kw)
    assert e.value.code == code, e.value


def test_refusals_of_the_products(F):
    b, odd = _Buf(), _Buf(4104)

    def logits(dtype=0, rows=4, hidden=8, vocab=16, s=b, W=b, bias=None, out=0, z=b):
        F.fold_vocab_logits(dtype, rows, hidden, vocab, s, W, bias, out, z, NULL_STREAM)

    for kw in (dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(rows=1 << 31), dict(hidden=0), dict(hidden=4097),
               dict(vocab=0), dict(vocab=(1 << 21) + 1), dict(out=1), dict(dtype=1, out=7), dict(s=None), dict(W=None),
               dict(z=None), dict(s=odd), dict(W=odd), dict(z=odd), dict(rows=(1 << 31) - 1, vocab=1 << 20)):
        _refused(F, F.FOLD_E_INVALID, logits, **kw)
    logits(rows=0, s=None, W=None, z=None)

    def back(dtype=0, rows=4, hidden=8, vocab=16, s=b, W=b, dz=b, ds=b, dW=b, db=b, flags=0, ws=None, n=0):
        F.fold_vocab_backward(dtype, rows, hidden, vocab, s, W, dz, ds, dW, db, flags, ws, n, NULL_STREAM)

    for kw in (dict(dtype=3), dict(rows=-2), dict(hidden=-1), dict(vocab=-1), dict(flags=2), dict(flags=-1), dict(dz=None),
               dict(s=None), dict(W=None), dict(s=odd), dict(ds=odd), dict(dW=odd), dict(ws=odd), dict(dz=odd)):
        _refused(F, F.FOLD_E_INVALID, back, **kw)
    n = F.fold_vocab_workspace_size(0, 4, 64, 100000)
    assert n > 0  # few rows: K is cut into pieces
    _refused(F, F.FOLD_E_MISMATCH, back, hidden=64, vocab=100000, ws=b, n=n - 1)
    _refused(F, F.FOLD_E_MISMATCH, back, hidden=64, vocab=100000, ws=None, n=n)
    _refused(F, F.FOLD_E_INVALID, F.fold_vocab_workspace_size, 0, 4, 0, 8)
    back(rows=0, s=None, W=None, dz=None, ds=b, dW=None, db=None)


def test_refusals_of_outputs_that_overlap(F):
    """4 rows, 64 states, a vocabulary of 128, fp32: states and d_states 1 KB, W and dW 32 KB, logits 2 KB, the bias 512
    bytes, each just behind the one before."""
    at, bufs = 1 << 20, {}
    for name, size in dict(s=1024, W=32768, dz=2048, ds=1024, dW=32768, db=512).items():
        bufs[name] = _Buf(at)
        at += size

    def logits(z, bias=None):
        F.fold_vocab_logits(0, 4, 64, 128, bufs["s"], bufs["W"], bias, 0, z, NULL_STREAM)

    for z in (bufs["s"], bufs["W"], _Buf(bufs["s"].at - 2032), _Buf(bufs["dz"].at - 16)):
        _refused(F, F.FOLD_E_INVALID, logits, z)
    _refused(F, F.FOLD_E_INVALID, logits, bufs["dz"], bufs["dz"])

    def back(**kw):
        b = dict(bufs, **kw)
        n = F.fold_vocab_workspace_size(0, 4, 64, 128)
        F.fold_vocab_backward(0, 4, 64, 128, b["s"], b["W"], b["dz"], b["ds"], b["dW"], b["db"], 0,
                              _Buf(1 << 30) if n else None, n, NULL_STREAM)

    for out, other in (("ds", "s"), ("ds", "dz"), ("dW", "W"), ("db", "dW"), ("dW", "ds"), ("db", "dz")):
        _refused(F, F.FOLD_E_INVALID, back, **{out: bufs[other]})


def test_refusals_of_the_distillation_loss(F):
    b, odd = _Buf(), _Buf(4097)
    big = _Buf(1 << 40)

    def call(sched=None, dtype=0, rows=4, vocab=16, z=b, k=2, tok=b, t=b, y=b, T=1.0, soft=1.0, hard=0.0, scale=1.0, loss=b,
             grad=0, dz=big, ws=big, n=1 << 20):
        F.fold_loss_distill(sched, dtype, rows, vocab, z, k, tok, t, y, T, soft, hard, scale, loss, grad, dz, ws, n,
                            NULL_STREAM)

    for kw in (dict(dtype=2), dict(rows=-1), dict(vocab=0), dict(k=-1), dict(k=257), dict(T=0.0), dict(T=1e-4),
               dict(T=2e3), dict(T=math.nan), dict(soft=-1.0), dict(soft=math.inf), dict(hard=math.nan),
               dict(scale=math.inf), dict(z=None), dict(loss=None), dict(tok=None), dict(t=None), dict(grad=2),
               dict(dtype=1, grad=0), dict(z=odd), dict(dz=odd), dict(ws=odd),
               dict(grad=1, dz=b),                     # another type over the same memory
               dict(dz=_Buf(4096 + 256))):             # a row further on
        _refused(F, F.FOLD_E_INVALID, call, **kw)
    n = F.fold_distill_workspace_size(0, 4, 100000, 2)
    assert n > 0  # a row that no workgroup holds
    _refused(F, F.FOLD_E_MISMATCH, call, vocab=100000, n=n - 1)
    _refused(F, F.FOLD_E_MISMATCH, call, vocab=100000, ws=None)
    _refused(F, F.FOLD_E_INVALID, F.fold_distill_workspace_size, 0, 4, 16, 300)
    call(rows=0, z=None, loss=None, tok=None, t=None, dz=None, ws=None, n=0)


def test_refusals_of_the_token_log_probabilities(F):
    b, odd = _Buf(), _Buf(4097)

    def call(sched=None, dtype=0, rows=2000, vocab=16, z=b, J=1, tok=b, logp=b, ent=b, K=2, top=b, lp=b, ws=None, n=0):
        F.fold_token_logprobs(sched, dtype, rows, vocab, z, J, tok, logp, ent, K, top, lp, ws, n, NULL_STREAM)

    for kw in (dict(dtype=2), dict(rows=-1), dict(vocab=0), dict(J=-1), dict(K=-1), dict(K=33), dict(z=None),
               dict(tok=None), dict(logp=None), dict(top=None), dict(lp=None), dict(z=odd), dict(ws=odd)):
        _refused(F, F.FOLD_E_INVALID, call, **kw)
    n = F.fold_token_workspace_size(0, 1, 100000, 5)
    assert n > 0  # one long row is cut into segments
    _refused(F, F.FOLD_E_MISMATCH, call, rows=1, vocab=100000, K=5, ws=b, n=n - 1)
    _refused(F, F.FOLD_E_MISMATCH, call, rows=1, vocab=100000, K=5)
    _refused(F, F.FOLD_E_INVALID, F.fold_token_workspace_size, 0, 1, 100000, 64)
    call(J=0, K=0, ent=None, z=None)  # nothing is asked for
    call(rows=0, z=None)


def test_refusals_of_the_tensor_wrappers(F):
    cpu = torch.zeros((4, 64))
    with pytest.raises(ValueError, match="CUDA"):
        F.VocabHead(cpu)
    with pytest.raises(ValueError, match="CUDA"):
        F.distill_loss(cpu, 64)
    with pytest.raises(ValueError, match="CUDA"):
        F.token_logprobs(cpu, 64)
