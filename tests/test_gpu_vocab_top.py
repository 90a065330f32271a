"""Top lists of rows whose large logits crowd in few threads' columns: more of them above the threads' threshold than a
workgroup keeps as candidates, so the list is found digit by digit.  Top tokens have to equal the oracle's."""
import numpy as np
import pytest

from oracle import vocab as OV
from paper_1702_02181_amd import fold as F
from tests.test_gpu_vocab import NAN, _check_tokens, _dev, _ints, _logits, _round

pytestmark = pytest.mark.gpu

THREADS, CAP, K = 256, 1024, 32


def _rows(V, dtype, rng):
    """Crowds in every 256th to (256 + 24)th vector, 24 threads of 256 and K = 32."""
    vec = 4 if dtype == "f32" else 8
    crowd = (np.arange(V) // vec) % THREADS < 24
    n = int(crowd.sum())
    z = _logits(rng, 6, V, dtype)
    z[0, crowd] = _round(20 + rng.standard_normal(n), dtype)                      # one digit decides, or two
    z[1, crowd] = _round(20 + rng.integers(0, 256, n) * 2.0 ** -19, dtype)        # three equal bytes (bf16: all equal)
    z[2, crowd] = 20.0                                                            # by the columns alone
    z[3, crowd] = _round(np.where(rng.random(n) < 10 / n, 20.125, 20.0), dtype)   # a few above many equal ones
    z[4] = _round(-40 + 0.1 * z[4], dtype)                                        # negative ones
    z[4, crowd] = _round(-20 - rng.integers(0, 256, n) * 2.0 ** -19, dtype)
    z[5, crowd] = _round(1e-30 * (1 + rng.random(n)), dtype)                      # small ones over negative ones
    z[5, ~crowd] = -np.abs(z[5, ~crowd])
    return z


def _above(z, lo, hi, vec):
    """Logits above the K-th largest of the threads' maxima, for columns [lo, hi) of a row."""
    part = z[lo:hi].astype(np.float64)
    thread = (np.arange(hi - lo) // vec) % THREADS
    top = np.full(THREADS, -np.inf)
    np.maximum.at(top, thread, part)
    return int((part > np.sort(top)[-K]).sum())


@pytest.mark.parametrize("V,dtype", [(20000, "f32"), (20001, "bf16"), (12345, "f32")])
def test_crowded_rows(V, dtype):
    z = _rows(V, dtype, np.random.default_rng(V))
    assert all(_above(r, 0, V, 4 if dtype == "f32" else 8) > CAP for r in z)
    _check_tokens(z, dtype, np.zeros((6, 1), int), K)


@pytest.mark.parametrize("V,dtype", [(1000003, "f32"), (120001, "bf16")])
def test_crowded_segments(V, dtype):
    """Long rows, cut into segments of whole 64-column blocks that are joined."""
    z = _rows(V, dtype, np.random.default_rng(V))
    size = 4 if dtype == "f32" else 2
    segments = min(-(-V * size // 32768), 64)
    per = -(-V // segments)
    per = -(-per // 64) * 64
    for r in z:
        for lo in range(0, V - per, per):
            assert _above(r, lo, lo + per, 16 // size) > CAP
    _, _, top, _ = OV.token_logprobs(z, np.zeros((6, 1), int), K)
    got = F.token_logprobs(_dev(z, dtype, NAN), V, _ints(np.zeros((6, 1))), K)
    assert np.array_equal(got.top_token.cpu().numpy(), top)


def test_a_crowd_in_one_segment():
    """One segment of a long row holds the list, the others ordinary logits."""
    V, dtype = 120001, "bf16"
    rng = np.random.default_rng(7)
    z = _logits(rng, 3, V, dtype)
    crowd = (np.arange(V) // 8) % THREADS < 24
    crowd &= (np.arange(V) >= 16384) & (np.arange(V) < 31000)
    z[0, crowd] = 20.0
    z[1, crowd] = _round(20 + rng.standard_normal(int(crowd.sum())), dtype)
    z[2, crowd] = -np.inf
    _check_tokens(z, dtype, np.zeros((3, 1), int), K)
