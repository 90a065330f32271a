"""The vocabulary head's row operators on logits of any size: masks by a large negative number (-1e4 to -1e30), rows whose
largest logit is large, and large logits that differ by a few of their own steps, against the fp64 oracle.

Bounds, from the arithmetic (u = 2^-24): the exponent of a term is rounded two or three times (the difference to the
reference, the factor log2 e / T and the product: 3 u of it), so p is within rel = u (4 |log p| + V / 256 + 64) of itself
as for logits of ordinary size.  A log probability, (z - m) - log s or ln 2 (z log2 e - m2 - log2 s), is on top of that
rounded four times (two constants, fma or difference, product or sum): 4 u of its value.
"""
import math

import numpy as np
import pytest

from oracle import vocab as OV
from paper_1702_02181_amd import fold as F
from tests.test_gpu_vocab import NAN, U, _check_distill, _dev, _hard_rows, _ints, _logits, _np, _rel, _round, _targets, _within

pytestmark = pytest.mark.gpu

NEAR = 11629079  # 2^24 / log2 e: where a scaled logit's own step reaches 1


def _rows(dtype, V, rng):
    vec = 4 if dtype == "f32" else 8
    cols = np.arange(V)
    lanes = (cols // vec) % 256 < 128  # whole vectors of half the threads of a workgroup
    rows = []

    def row(**at):
        rows.append(_logits(rng, 1, V, dtype)[0])
        return rows[-1]
    for v in (-1e4, -1e9, -1e10, -1e20, -1e30):
        row()[:V // 3] = v
        row()[V // 3:] = v  # whole segments of a long row
        row()[lanes] = v
        one = row()
        one[cols != V // 2] = v
        row()[:] = v
    for v in (1e10, 1e20, 1e30):
        row()[V // 2] = v
        row()[:] = v
        row()[V // 3:] = v
    k = lambda hi: rng.integers(0, hi, V)  # noqa: E731
    half = cols < V // 2
    for z in (1.15e7 + k(20), 1.17e7 + k(20), NEAR - 10 + k(21), -NEAR - 10 + k(21), -1.17e7 - k(20), 3e9 + 256 * k(9),
              -1e8 - 8 * k(9), 1e12 + 65536.0 * k(3),
              np.where(half, NEAR - k(8), NEAR + 1 + k(8)), np.where(half, NEAR + 1 + k(8), NEAR - k(8)),
              np.where(half, -NEAR + k(8), -NEAR - 1 - k(8)), np.where(half, -NEAR - 1 - k(8), -NEAR + k(8)),
              # the same border at T = 0.01
              np.where(half, 116290 - k(8) / 128, 116291 + k(8) / 128), np.where(half, -116291 + k(8) / 128, -116290 - k(8) / 128)):
        row()[:] = z
    return _round(np.stack(rows), dtype)


LONG = {"f32": 70001, "bf16": 120001}  # rows that go in segments


@pytest.mark.parametrize("V", [3, 300, 9000, "long"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_token_logprobs_of_logits_of_any_size(V, dtype):
    V = LONG[dtype] if V == "long" else V
    rng = np.random.default_rng(V)
    z = _rows(dtype, V, rng)
    M = z.shape[0]
    tokens = np.concatenate([rng.integers(0, V, (M, 3)), np.full((M, 1), V // 2), np.full((M, 1), V - 1)], 1)
    r = F.token_logprobs(_dev(z, dtype, NAN), V, _ints(tokens), 8)
    logp, ent, top, top_lp = OV.token_logprobs(z, tokens, 8)
    _within(_np(r.logp), logp, np.take_along_axis(_rel(z, 1.0, V), tokens, 1) + 4 * U * np.abs(logp), "logp")
    _within(_np(r.entropy), ent, 4 * U * (V / 256 + 64) * (1 + ent) + 16 * U * ent ** 2, "entropy")
    assert np.array_equal(r.top_token.cpu().numpy(), top)
    size = np.where(np.isfinite(top_lp), np.abs(top_lp), 0)
    _within(_np(r.top_logp), top_lp, U * (6 * size + V / 256 + 64 + 4 * math.log(V)), "top log probabilities")


@pytest.mark.parametrize("V", [3, 300, 9000, "long"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [0.01, 0.5, 1.0, 2.0, 4.0, 100.0])
def test_distill_of_logits_of_any_size(V, dtype, T):
    V = LONG[dtype] if V == "long" else V
    rng = np.random.default_rng(V)
    z = _rows(dtype, V, rng)
    tok, t, y = _targets(rng, z.shape[0], V, 3)
    _check_distill(z, dtype, dtype, tok, t, y, T, 0.5, 0.5)


@pytest.mark.parametrize("soft,hard", [(1.0, 0.0), (0.0, 1.0)])
def test_one_term_of_logits_of_any_size(soft, hard):
    for V in (300, LONG["f32"]):
        rng = np.random.default_rng(V + 1)
        z = _rows("f32", V, rng)
        tok, t, y = _targets(rng, z.shape[0], V, 3)
        _check_distill(z, "f32", "bf16", tok, t, y, 2.0, soft, hard)


@pytest.mark.parametrize("V", [300, "long"])
@pytest.mark.parametrize("soft,hard", [(0.0, 1.0), (1.0, 0.0), (0.0, 0.0)])
def test_rows_that_are_no_distribution_under_weights_of_zero(V, soft, hard):
    """A target makes the loss of a row with NaN or +inf NaN, and that of a row of -inf alone +inf, also where the only
    target's term has a weight of zero; rows without a target stay at 0."""
    V = LONG["f32"] if V == "long" else V
    rng = np.random.default_rng(V + 2)
    z = np.concatenate([_hard_rows("f32", V, rng)] * 3)
    tok, t, y = _targets(rng, 60, V, 3)
    tok[:20], y[20:40] = -1, -1  # a label alone, a teacher alone, both
    _check_distill(z, "f32", "f32", tok, t, y, 2.0, soft, hard)
