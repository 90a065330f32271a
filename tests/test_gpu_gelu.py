"""gelu and its slope over their whole range, in fp32 the negative tail relative to itself.

fp32: Phi(-|z|) = e Q(t), e = exp(-z^2 / 2), t = 1 / (1 + 0.35 |z|).  With u = 2^-24: Q's fit is within 3.2e-8 < 1 u; t is within 3 u
(a product and sum, a reciprocal of one ulp), which moves t P(t) by at most 1.5 of that; the polynomial's nine steps round by at
most u of the terms' magnitudes, whose sum is at most 2 Q; the last products and exp2's ulp are 4 u: 1 + 4.5 + 18 + 4 < 28 u.  The
exponent -0.7213 z^2 is a rounded constant and two products, 2.5 u of itself, and the logarithm moves by z^2 / 2 of it: 1.25 z^2 u.
So Phi of the negative side is within (28 + 1.25 z^2) u of itself, of the positive side that of Phi(-z) and u.  The value is a
product more.  The slope is Phi + z phi(z): phi(z) within (4 + 1.25 z^2) u of itself, and two products and a sum of the magnitudes.
bf16: Phi is within 1.5e-7 by its formula and 8 u by its rounding, as for the layers."""
import math

import numpy as np
import pytest

from paper_1702_02181_amd import fold as F
from tests.block_common import HALF, U, dev, host, rounded, torch_type, within

pytestmark = pytest.mark.gpu


def _points(dtype):
    z = np.concatenate([np.linspace(-10, 10, 4001), np.linspace(-1, 1, 501), np.random.default_rng(0).standard_normal(2000), [0.0]])
    return np.unique(rounded(z, dtype)).reshape(-1, 1)


def _parts(z, dtype):
    """Phi from erfc, which keeps the tail; phi; the bounds of Phi and of phi."""
    phi = np.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    cdf = 0.5 * np.vectorize(math.erfc)(-z / math.sqrt(2))
    tail = 0.5 * np.vectorize(math.erfc)(np.abs(z) / math.sqrt(2))
    b = (28 + 1.25 * z * z) * U * tail + U * (z >= 0) if dtype == "f32" else 1.5e-7 + 8 * U
    return cdf, phi, b, (4 + 1.25 * z * z) * U * phi


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gelu(dtype):
    z = _points(dtype).astype(np.float64)
    cdf, _, b, _ = _parts(z, dtype)
    want, bound = z * cdf, np.abs(z) * (b + U * cdf)
    bound = bound + HALF[dtype] * (np.abs(want) + bound)
    one = F.Linear(dev([[1.0]], dtype), None, 1, "gelu")
    x = dev(z, dtype)
    within(host(one.forward(x), 1), want, bound, "tiles")
    few = np.concatenate([host(one.forward(part.contiguous()), 1) for part in x.split(60)])
    within(few, want, bound, "few rows")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_slope_of_gelu(dtype):
    import torch
    z = _points(dtype).astype(np.float64)
    cdf, phi, b, bp = _parts(z, dtype)
    want = cdf + z * phi
    bound = b + np.abs(z) * (bp + 3 * U * phi) + U * (cdf + np.abs(z) * phi)
    bound = bound + HALF[dtype] * (np.abs(want) + bound)
    one = F.Linear(dev([[1.0]], dtype), None, 1, "gelu")
    x, got = dev(z, dtype), torch.empty((len(z), 64), dtype=torch_type(dtype), device="cuda")
    one.backward(x, dev(np.ones_like(z), dtype), x.clone(), dx=None, dW=None, dbias=None, dpre=got)
    within(host(got, 1), want, bound, "slope")


def test_gelu_far_out():
    """Past the range of exp: z or 0, slope 1 or 0; NaN stays NaN."""
    z = np.array([[-1e30], [-200.0], [-20.0], [20.0], [200.0], [1e30], [np.inf], [np.nan]], np.float32)
    out = host(F.Linear(dev([[1.0]]), None, 1, "gelu").forward(dev(z)), 1)[:, 0]
    assert np.array_equal(out[3:7], z[3:7, 0]) and np.isnan(out[7]) and (np.abs(out[:3]) < 1e-37).all()
