"""The block between two batches of graphs by itself, with each activation, against the oracle's chain in fp64."""
import numpy as np
import pytest

from oracle import block as OB
from oracle import compare
from paper_1702_02181_amd import gen
from tests.block_common import host

pytestmark = pytest.mark.gpu


def _chain(block, x, s, up, act, lists):
    """out, dx, ds and the parameters' gradients in the order of block.tensors."""
    W = [host(layer[0].weight, layer[0].in_dim) for layer in (block.q, block.kv, block.o, block.first, block.second)]
    a, ma, ra = OB.layer_norm(x)
    q, kv = OB.linear(a, W[0])[0], OB.linear(s, W[1])[0]
    k, v = kv[:, :block.wk], kv[:, block.wk:]
    o, _ = OB.attend(q, k, v, **lists)
    y = OB.linear(o, W[2], residual=x)[0]
    b, mb, rb = OB.layer_norm(y)
    f, pre = OB.linear(b, W[3], act=act)
    z = OB.linear(f, W[4], residual=y)[0]
    out, mz, rz = OB.layer_norm(z)
    dz, dg2, db2 = OB.layer_norm_backward(z, up, mean=mz, rstd=rz)
    df, dW4, d4, _ = OB.linear_backward(f, W[4], dz)
    db_, dW3, d3, _ = OB.linear_backward(b, W[3], df, act, pre)
    dy, dg1, db1 = OB.layer_norm_backward(y, db_, mean=mb, rstd=rb)
    dy = dy + dz
    do, dW2, d2, _ = OB.linear_backward(o, W[2], dy)
    dq, dk, dv = OB.attend_backward(q, k, v, do, **lists)
    ds, dW1, d1, _ = OB.linear_backward(s, W[1], np.concatenate([dk, dv], 1))
    da, dW0, d0, _ = OB.linear_backward(a, W[0], dq)
    dx, dg0, db0 = OB.layer_norm_backward(x, da, mean=ma, rstd=ra)
    return [out, dx + dy, ds, dg0, db0, dg1, db1, dg2, db2, dW0, d0, dW1, d1, dW2, d2, dW3, d3, dW4, d4]


@pytest.mark.parametrize("act", ["none", "relu", "tanh", "gelu"])
def test_block_with_each_activation(act):
    import torch
    from paper_1702_02181_amd.runner import CrossBlock, DeviceRun
    from tests.gpu_common import TOL
    target, source = (DeviceRun(gen.config2(seed=s, num_graphs=6, leaves=n, hidden=64), with_backward=False)
                      for s, n in ((31, 7), (32, 20)))
    target.forward()
    source.forward()
    block = CrossBlock(target, source, 4, 200, kv_heads=2, activation=act, seed=3)
    up = np.random.default_rng(6).standard_normal((target.N, 64)).astype(np.float32)
    out = block.forward()
    dx, ds = block.backward(torch.from_numpy(up).cuda())
    rows = [r.sched_arrays()["node_pos"] for r in (target, source)]
    lists = dict(heads=4, kv_heads=2, head_dim=16, q_ptr=target.w.graph_ptr, k_ptr=source.w.graph_ptr, q_rows=rows[0], k_rows=rows[1])
    want = _chain(block, host(target.h_pool, 64), host(source.h_pool, 64), up, act, lists)
    got = [host(out, 64), host(dx, 64), host(ds, 64)]
    got += [host(g) if g.dim() == 1 else host(g, w.shape[1]) for (_, _, g), w in zip(block.tensors, want[3:])]
    for i, (g, w) in enumerate(zip(got, want)):
        assert g.shape == w.shape, i
        if np.abs(w).max() > 1e-9:  # (the keys' biases move every score of a row alike: a sum of zeros, beside the values' part)
            assert compare.rel_err(g, w, whole=i > 2) <= TOL["f32"], (act, i)
