"""The training step of two batches as a replayed graph whose weights move between the replays, and the direction of its update."""
import numpy as np
import pytest

from tests.test_gpu_cross_step import _build

pytestmark = pytest.mark.gpu


def _own(step):
    """Gradients whose sums have one order: the block's and the head's."""
    return [g for _, _, g in step.block.tensors] + [step.dW, step.db]


def _cells(step):
    return [t for run in (step.target, step.source) for g in run.grad_tensors for t in (*g, run.d_table) if t is not None]


def _update(step, t):
    from paper_1702_02181_amd import fold as F
    lr, b1, b2, eps = step.hyper
    for (master, low, grad), (m, v) in zip(step.tensors, step.moments):
        F.fold_adam_step(master.numel(), master, low, grad, m, v, lr, b1, b2, eps, t)
    for run in (step.target, step.source):
        run.packed.update(run.set_tensors, run.stream)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_replays_follow_the_weights(dtype):
    """Every replay writes all gradients, of the weights that it finds: NaN before it, an eager pass over the same weights after
    it, Adam between one and the next.  The cells' gradients may add in another order: within 1e-4 (fp32, and as much of bf16's
    operands' sums, which are fp32) of their largest."""
    import gc

    import torch
    step, *_ = _build(dtype, lr=1e-2)
    step.gradients()
    step.gradients()
    torch.cuda.synchronize()
    gc.collect()  # device memory of other tests' garbage, freed by a collection during the recording, would end it
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.gradients()
    loss, kept = step.node_loss, (step.target.dh_nodes, step.source.dh_nodes)
    last = None
    for it in range(4):
        for t in (*_own(step), *_cells(step), loss, *kept):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*_own(step), loss, *kept)]
        cells = [t.clone() for t in _cells(step)]
        for t in (*_own(step), *_cells(step)):
            t.fill_(float("nan"))
        step.gradients()
        torch.cuda.synchronize()
        want = [*_own(step), step.node_loss, step.target.dh_nodes, step.source.dh_nodes]
        assert all(torch.isfinite(t).all() for t in got + cells), it
        assert all(torch.equal(a, b) for a, b in zip(got, want)), it
        for a, b in zip(cells, _cells(step)):
            assert (a - b).abs().max() <= 1e-4 * b.abs().max(), it
        assert last is None or not torch.equal(last, got[-3]), it  # other weights, other losses
        last = got[-3]
        _update(step, it + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_update_goes_down(dtype):
    """Adam's first step moves every weight against its gradient: by lr |g| r / (|g| r + eps) with r = (1 - beta2)^1/2 = 0.0316, eps =
    1e-8 (fold_adam_step adds eps to the root of v as it is), which is lr but for a part of eps / (r |g|) <= 3.2e-7 / |g|.  Its
    roundings are below 16 u of lr, the weight's 2^-23 of it."""
    import torch
    step, *_ = _build(dtype, lr=1e-2)
    before = [m.clone() for m, _, _ in step.tensors]
    step.step()
    torch.cuda.synchronize()
    moved = 0
    for (m, low, g), b in zip(step.tensors, before):
        # reshaped: a table's gradient is as wide as the table
        d, g = (m - b).reshape(-1), g.reshape(-1)
        assert not ((d * g) > 0).any()
        large = g.abs() > 1e-5
        d, g, b = d[large].abs(), g[large].abs(), b.reshape(-1)[large].abs()
        assert ((d - 1e-2).abs() <= 1e-2 * (3.2e-7 / g + 2.0 ** -20) + 2.0 ** -23 * (b + 1e-2)).all()
        moved += int(large.sum())
        if low is not None:
            assert torch.equal(low, m.to(low.dtype))
    assert moved > 1000 and np.isfinite(float(step.node_loss.sum()))
