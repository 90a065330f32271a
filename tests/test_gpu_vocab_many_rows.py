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


def test_longest_rows():
    """Rows of 2^30 logits, the largest vocabulary that the row operators take, in 64 segments: a thread sums
    2^30 / 64 / 256 = 2^16 terms, so rel = u (4 |log p| + 2^16 + 64)."""
    import torch
    M, V, T = 2, 1 << 30, 2.0
    g = torch.Generator(device="cuda").manual_seed(3)
    z = torch.empty((M, V), dtype=torch.bfloat16, device="cuda")
    for r in range(M):
        for lo in range(0, V, 1 << 26):
            z[r, lo:lo + (1 << 26)] = 2.5 * torch.randn(1 << 26, generator=g, device="cuda")
    z[1, V // 2:] = -1e9  # whole segments inside a mask
    z[1, V - 1] = 30.0
    tok = torch.tensor([[0, V - 1, 12345, V], [V // 2 - 1, V - 1, V // 2, -1]], dtype=torch.int32, device="cuda")
    t = torch.tensor([[1.0, 2.0, 0.5, 9.0], [3.0, 1.0, -1.0, 9.0]], device="cuda")
    y = torch.tensor([V - 1, 7], dtype=torch.int32, device="cuda")
    rel = U * (4 * 60 + (1 << 16) + 64)
    want = {}
    for temp in (1.0, T):
        s = torch.zeros(M, dtype=torch.float64, device="cuda")
        ex = torch.zeros_like(s)
        m = z.amax(1).double() / temp
        for lo in range(0, V, 1 << 26):
            x = z[:, lo:lo + (1 << 26)].double() / temp - m[:, None]
            e = x.exp()
            s += e.sum(1)
            ex += (e * x).sum(1)
        want[temp] = m, s, ex
    m, s, ex = want[1.0]
    at = tok.long().clamp(0, V - 1)
    given = z.gather(1, at).double()
    lp = given - m[:, None] - s.log()[:, None]
    lp[0, 3] = lp[1, 3] = 0.0
    r = F.token_logprobs(z, V, tok, 4)
    assert ((r.logp.double() - lp).abs() <= rel + 4 * U * lp.abs()).all()
    ent = s.log() - ex / s
    assert ((r.entropy.double() - ent).abs() <= 4 * rel * (1 + ent)).all()
    for row in range(M):
        top = r.top_token[row].long()
        v = z[row, top].float()
        # in order, equal ones by the lowest token, nothing above the last and nothing before it that equals it
        assert all((v[i] > v[i + 1]) or (v[i] == v[i + 1] and top[i] < top[i + 1]) for i in range(3))
        above = int((z[row] > z[row, top[-1]]).sum())
        assert above + int((z[row, :int(top[-1]) + 1] == z[row, top[-1]]).sum()) == 4
    # the loss and its gradient, in place
    (mT, sT, _), zy = want[T], z.gather(1, y.long()[:, None])[:, 0].double()
    have = torch.tensor([[True, True, True, False]] * 2, device="cuda")
    q = torch.softmax(torch.where(have, t.double() / T, -torch.inf), 1)
    lpT = given / T - mT[:, None] - sT.log()[:, None]
    logq = torch.where(have, q, torch.ones_like(q)).log()
    loss = 0.5 * T * T * torch.where(have, q * (logq - lpT), 0.0).sum(1) - 0.5 * (zy - m - s.log())
    cols = torch.randint(8, V // 2 - 8, (1000,), generator=g, device="cuda")
    old = z[:, cols].double()
    got, dz = F.distill_loss(z, V, tok, t, y, temperature=T, soft_weight=0.5, hard_weight=0.5, dlogits=z)
    assert dz is z
    assert ((got.double() - loss).abs() <= 8 * rel + 16 * U * loss.abs()).all()
    pT = (old / T - mT[:, None]).exp() / sT[:, None]
    p = (old - m[:, None]).exp() / s[:, None]
    target = torch.stack([(cols[:, None] == tok[r].long()).any(1) | (cols == y[r]) for r in range(M)])
    d = 0.5 * T * pT + 0.5 * p
    assert (((dz[:, cols].double() - d).abs() <= 2 * rel * d + 2.0 ** -8 * d * (1 + 2 * rel) + 1e-37) | target).all()
    mass = 0.5 * T * (((given / T - mT[:, None]).exp() / sT[:, None]) - q) + 0.5 * ((given - m[:, None]).exp() / s[:, None])
    mass -= 0.5 * (tok == y[:, None])
    off = (dz.gather(1, at).double() - mass).abs()
    assert ((off <= 4 * rel + 2.0 ** -8 * mass.abs()) | ~have).all()
    assert not dz[1, V // 2 + 1:V - 1].any()
