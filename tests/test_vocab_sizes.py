"""Sizes that the vocabulary head's products take: whatever a launch of fewer than 2^24 tiles covers.  The size checks run
on the host; on the GPU, more rows than fit a bound of 64 pieces for every tile of the states' gradient."""
import random

import numpy as np
import pytest

from tests.test_oracle_vocab import F, NULL_STREAM, _Buf  # noqa: F401  (F is a fixture)

MANY = [(262144, 4096, 33), (1048576, 1024, 1000), (1100000, 1024, 33), (4300000, 256, 33), (8000000, 64, 64),
        (1 << 29, 64, 64), ((1 << 29) - 5, 1, 1), (1 << 23, 4096, 64), (1 << 14, 1, 1 << 21), (16385, 4096, 1 << 21)]


def _logits_fit(F, dtype, rows, hidden, vocab):
    """The size check comes before the buffers': without them the call is refused either way."""
    with pytest.raises(F.FoldError) as e:
        F.fold_vocab_logits(dtype, rows, hidden, vocab, None, None, None, 0, None, NULL_STREAM)
    assert e.value.code == F.FOLD_E_INVALID
    return "NULL buffer" in str(e.value)


@pytest.mark.parametrize("dtype", [0, 1])
def test_many_rows_are_taken(F, dtype):  # noqa: F811
    for rows, hidden, vocab in MANY:
        assert _logits_fit(F, dtype, rows, hidden, vocab), (rows, hidden, vocab)
        if rows * vocab <= 1 << 35:
            assert F.fold_vocab_workspace_size(dtype, rows, hidden, vocab) >= 0


def test_everything_up_to_2_35_fits(F):  # noqa: F811
    rng = random.Random(1)
    for _ in range(4000):
        hidden, vocab = int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 21))
        ld = (max(hidden, vocab) + 63) // 64 * 64
        most = min((1 << 35) // ld, (1 << 31) - 1)
        rows = rng.choice([most, most - rng.randrange(100), int(most ** rng.random())])
        for dtype in (0, 1):
            assert _logits_fit(F, dtype, rows, hidden, vocab), (rows, hidden, vocab)
            F.fold_vocab_workspace_size(dtype, rows, hidden, vocab)


def test_too_many_tiles_are_refused(F):  # noqa: F811
    for rows, hidden, vocab in (((1 << 31) - 1, 64, 1 << 20), ((1 << 31) - 1, 4096, 64), ((1 << 31) - 1, 64, 1 << 21)):
        with pytest.raises(F.FoldError, match="too many tiles") as e:
            F.fold_vocab_workspace_size(0, rows, hidden, vocab)
        assert e.value.code == F.FOLD_E_INVALID
    assert not _logits_fit(F, 0, (1 << 31) - 1, 64, 1 << 20)
    assert not _logits_fit(F, 1, (1 << 31) - 1, 64, 1 << 21)


@pytest.mark.gpu
@pytest.mark.parametrize("M,H,V,dtype", [(1048581, 1024, 40, "bf16"), (262147, 4096, 33, "f32")])
def test_products_of_many_rows(M, H, V, dtype):
    """Every output against fp64 products of the same operands.  Bounds as for fewer rows: (K + 72) u of the sum of the
    terms' magnitudes, but of M terms in a row a sum's rounding is bounded by the root of their number here: M u would be
    6 % of it, and terms of random signs do not add up that way (a factor of 8 covers 10^5 outputs)."""
    import torch
    from paper_1702_02181_amd import fold
    tdt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(M)
    ld, ldv, u = fold.fold_row_ld(H), fold.fold_row_ld(V), 2.0 ** -24
    s = torch.zeros((M, ld), dtype=tdt, device="cuda")
    for lo in range(0, M, 1 << 17):
        n = min(1 << 17, M - lo)
        s[lo:lo + n, :H] = torch.tanh(torch.randn((n, H), generator=g, device="cuda")).to(tdt)
    W = torch.zeros((V, ld), dtype=tdt, device="cuda")
    W[:, :H] = (torch.randn((V, H), generator=g, device="cuda") / H ** 0.5).to(tdt)
    b = torch.randn(V, generator=g, device="cuda")
    dz = torch.zeros((M, ldv), dtype=tdt, device="cuda")
    dz[:, :V] = (torch.randn((M, V), generator=g, device="cuda") / 64).to(tdt)
    head = fold.VocabHead(W, b, H)
    z = head.logits(s, dtype=torch.float32)
    ds, dW, db = head.backward(s, dz)
    Wd, bd = W[:, :H].double(), b.double()
    dW_want = torch.zeros((V, H), dtype=torch.float64, device="cuda")
    db_want = torch.zeros(V, dtype=torch.float64, device="cuda")
    dW_square, db_square = torch.zeros_like(dW_want), torch.zeros_like(db_want)
    for lo in range(0, M, 1 << 15):
        sd, dd = s[lo:lo + (1 << 15), :H].double(), dz[lo:lo + (1 << 15), :V].double()
        mag = sd.abs() @ Wd.abs().t().contiguous() + bd.abs()
        off = (z[lo:lo + (1 << 15), :V].double() - (sd @ Wd.t().contiguous() + bd)).abs()
        assert (off <= (H + 8) * u * mag).all(), lo
        off = (ds[lo:lo + (1 << 15), :H].double() - dd @ Wd).abs()
        assert (off <= (V + 72) * u * (dd.abs() @ Wd.abs())).all(), lo
        dW_want += dd.t().contiguous() @ sd
        dW_square += (dd * dd).t().contiguous() @ (sd * sd)
        db_want += dd.sum(0)
        db_square += (dd * dd).sum(0)
    # after n terms the partial sum is of size sqrt(n) of a term's, so M roundings of half a step add up to at most
    # u sqrt(M) sqrt(sum of squares) in the root mean square
    for got, want, square in ((dW[:, :H], dW_want, dW_square), (db, db_want, db_square)):
        assert ((got.double() - want).abs() <= 8 * u * M ** 0.5 * square.sqrt()).all()
    assert not z[:, V:].any() and not ds[:, H:].any() and not dW[:, H:].any()
