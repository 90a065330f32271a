"""What a call of the layers' gradients leaves out and what it still writes."""
import numpy as np
import pytest

from paper_1702_02181_amd import fold as F
from tests.block_common import dev, rounded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,dtype,act", [(5, "f32", "tanh"), (700, "bf16", "gelu"), (70, "bf16", "relu")])
def test_gradient_before_the_activation_alone(M, dtype, act):
    import torch
    rng = np.random.default_rng(M)
    x, z, dout = (dev(rounded(rng.standard_normal((M, n)), dtype), dtype) for n in (100, 200, 200))
    layer = F.Linear(dev(rounded(rng.standard_normal((200, 100)), dtype), dtype), None, 100, act)
    want, got = torch.full_like(z, 7.0), torch.full_like(z, 7.0)
    layer.backward(x, dout, z, dpre=want)
    assert layer.backward(x, dout, z, dx=None, dW=None, dbias=None, dpre=got) == (None, None, None)
    assert torch.equal(got, want) and not (got == 7.0).any()
    over = dout.clone()
    layer.backward(x, over, z, dx=None, dW=None, dbias=None, dpre=over)
    assert torch.equal(over, want)
    assert layer.backward(x, dout, z, dx=None, dW=None, dbias=None) == (None, None, None)  # nothing at all
