"""Row operators on more rows than one launch takes, and on more than 2^31 logits, against fp64 on the same logits.

Bounds: as for fewer rows (u = 2^-24): rel = u (4 |log p| + V / 256 + 64) with |log p| at most 40 for these logits."""
import pytest

from paper_1702_02181_amd import fold as F

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _logits(M, V):
    import torch
    g = torch.Generator(device="cuda").manual_seed(V)
    z = torch.zeros((M, F.fold_row_ld(V)), dtype=torch.bfloat16, device="cuda")
    for lo in range(0, M, 1 << 19):
        n = min(1 << 19, M - lo)
        z[lo:lo + n, :V] = 2.5 * torch.randn((n, V), generator=g, device="cuda")
    return z, g


def test_token_logprobs_of_many_rows():
    import torch
    M, V = (1 << 23) + 9, 300
    z, g = _logits(M, V)
    tok = torch.randint(0, V, (M, 1), generator=g, device="cuda", dtype=torch.int32)
    r = F.token_logprobs(z, V, tok, 1)
    rel = U * (4 * 40 + V / 256 + 64)
    at = torch.arange(V, device="cuda", dtype=torch.int32)
    for lo in range(0, M, 1 << 18):
        rows = slice(lo, lo + (1 << 18))
        x = z[rows, :V].double()
        lp = torch.log_softmax(x, 1)
        assert ((r.logp[rows].double() - lp.gather(1, tok[rows].long())).abs() <= rel + 80 * U).all(), lo
        ent = -(lp.exp() * lp).sum(1)
        assert ((r.entropy[rows].double() - ent).abs() <= 4 * U * (V / 256 + 64) * (1 + ent) + 16 * U * ent ** 2).all(), lo
        first = torch.where(x == x.amax(1, keepdim=True), at, V).amin(1)
        assert torch.equal(r.top_token[rows, 0], first.int()), lo


def test_distill_of_many_rows():
    import torch
    M, V = (1 << 21) + 7, 1100
    z, g = _logits(M, V)
    y = torch.randint(-1, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    loss, dz = F.distill_loss(z, V, labels=y, soft_weight=0.0, hard_weight=1.0)
    rel = U * (4 * 40 + V / 256 + 64)
    for lo in range(0, M, 1 << 16):
        rows = slice(lo, lo + (1 << 16))
        have = (y[rows] >= 0).double()[:, None]
        lp = torch.log_softmax(z[rows, :V].double(), 1)
        at = y[rows].long().clamp(min=0)[:, None]
        assert ((loss[rows].double() + (have * lp.gather(1, at))[:, 0]).abs() <= rel + 80 * U).all(), lo
        p = lp.exp()
        want = have * p.scatter_add(1, at, torch.full_like(have, -1.0))
        bound = 2 * rel * p
        bound.scatter_add_(1, at, torch.full_like(have, 4 * U))
        off = (dz[rows, :V].double() - want).abs()
        assert (off <= bound * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()).all(), lo
    assert not dz[:, V:].any()
