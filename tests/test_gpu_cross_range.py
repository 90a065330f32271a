"""Cross attention at the ends of its scale and of its scores."""
import numpy as np
import pytest

from paper_1702_02181_amd import fold as F

pytestmark = pytest.mark.gpu


def _case(d=64, nq=40, nk=90):
    import torch
    ptr = lambda n: torch.tensor([0, n], dtype=torch.int32, device="cuda")  # noqa: E731
    plan = F.CrossAttention(1, d, ptr(nq), ptr(nk), dtype=torch.float32)
    g = torch.Generator(device="cuda").manual_seed(1)
    return plan, *(torch.randn((n, d), generator=g, device="cuda") for n in (nq, nk, nk, nq))


def test_scales_by_powers_of_two():
    """2^e in the scale and 2^-e in q and k change no bit: the products and the exponents are the same numbers."""
    import torch
    plan, q, k, v, do = _case()
    out, lse = plan.forward(q, k, v, scale=0.125)
    want = plan.backward(q, k, v, out, lse, do, scale=0.125)
    for e in (100, -100, 120):
        a, b = 2.0 ** -(e // 2), 2.0 ** (e // 2 - e)
        o, ls = plan.forward(q * a, k * b, v, scale=0.125 * 2.0 ** e)
        assert torch.equal(o, out) and torch.equal(ls, lse), e
        dq, dk, dv = plan.backward(q * a, k * b, v, o, ls, do, scale=0.125 * 2.0 ** e)
        assert torch.equal(dq * a, want[0]) and torch.equal(dk * b, want[1]) and torch.equal(dv, want[2]), e


def test_scales_that_are_refused():
    plan, q, k, v, do = _case()
    out, lse = plan.forward(q, k, v)
    for scale in (2.0 ** 127, 3e38, float("inf"), float("nan"), 0.0, -1.0):
        for call in (lambda: plan.forward(q, k, v, scale=scale), lambda: plan.backward(q, k, v, out, lse, do, scale=scale)):
            with pytest.raises(F.FoldError) as e:
                call()
            assert e.value.code == F.FOLD_E_INVALID


@pytest.mark.parametrize("score", [1e3, -3e4, 1e6])
def test_probabilities_of_large_scores(score):
    """One key: o is v whatever its score is, but for p v and 1 / l's roundings and their product's (p = exp2(fma(s, c, -m)) is
    near 1, not 1, and l the same number: 4 u with a reciprocal of one ulp); the gradient's probability is exp(s - lse), off by |lse| 2^-22 (lse is fp32: two
    roundings and a constant's on its way out, the same on its way back, half a step of 2^-24 each)."""
    import torch
    plan, _, _, v, do = _case(32, 3, 1)
    q, k = torch.full((3, 32), 1.0, device="cuda"), torch.full((1, 32), score / 32, device="cuda")
    v, do = v[:, :32].contiguous(), do[:, :32].contiguous()
    q, k, v, do = (torch.nn.functional.pad(t, (0, 32)) for t in (q, k, v, do))
    out, lse = plan.forward(q, k, v, scale=1.0)
    assert ((out[:, :32] - v[:, :32]).abs() <= 2.0 ** -22 * v[:, :32].abs()).all()
    assert (lse.double() - score).abs().max() <= 4 * 2.0 ** -24 * abs(score) * 8  # (32 products and sums: s itself)
    _, _, dv = plan.backward(q, k, v, out, lse, do, scale=1.0)
    want = do[:, :32].double().sum(0)
    size = do[:, :32].double().abs().sum(0)
    assert np.isfinite(score) and ((dv[0, :32].double() - want).abs() <= (1.01 * 2.0 ** -22 * abs(score) + 2.0 ** -20) * size).all()
