"""The kernel profile of the vocabulary head's backward: every launch lies in a record."""
import pytest

from paper_1702_02181_amd import fold as F
from tests.test_gpu_vocab import _dev, _product_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,H,V,want", [
    (33, 300, 20000, {"vocab_backward", "vocab_dstates_join"}),                                    # one launch for both
    (300, 96, 30000, {"vocab_dstates", "vocab_dstates_join", "vocab_dweights", "vocab_dbias"}),
    (3000, 256, 500, {"vocab_dstates", "vocab_dweights", "vocab_dbias"})])
def test_records_of_the_backward(M, H, V, want):
    import torch
    s, W, _, dz = _product_case(M, H, V, "bf16", 3)
    head = F.VocabHead(_dev(W, "bf16"), None, H)
    s, dz = _dev(s, "bf16"), _dev(dz, "bf16")
    head.backward(s, dz)
    torch.cuda.synchronize()
    F.fold_profile_read()
    F.fold_profile_enable(True)
    try:
        head.backward(s, dz)
        torch.cuda.synchronize()
        got = F.fold_profile_read()
    finally:
        F.fold_profile_enable(False)
    assert set(got) == want and all(n == 1 and ms > 0 for n, ms, _ in got.values()), got
