"""Which nodes a vocabulary step counts as having a target: those that fold_loss_distill gives a loss to."""
import numpy as np
import pytest
import torch

from oracle import vocab as OV
from paper_1702_02181_amd import runner


def _targets(N=40, V=11, k=3):
    rng = np.random.default_rng(4)
    tok = rng.integers(-1, V + 2, (N, k))
    t = rng.standard_normal((N, k)).astype(np.float32)
    y = rng.integers(-2, V + 2, N)
    t[::3] = -np.inf        # a teacher that pads by logits: valid tokens, no entry that counts
    t[1::3, 0] = -np.inf
    tok[2::5] = -1
    y[::2] = -1
    y[4] = V
    return V, tok, t, y


@pytest.mark.parametrize("use", ["teacher", "labels", "both", "none"])
def test_nodes_with_a_target(use):
    V, tok, t, y = _targets()
    N = len(y)
    tok, t = (tok, t) if use in ("teacher", "both") else (None, None)
    y = y if use in ("labels", "both") else None
    # by the oracle: logits of one row's NaN make its loss NaN if, and only if, it has a target
    loss, _ = OV.distill(np.full((N, V), np.nan), tok, t, y, soft=1.0, hard=1.0)
    tensors = [None if a is None else torch.from_numpy(a) for a in (y, tok, t)]
    have = runner.nodes_with_target(N, V, *tensors)
    assert have.dtype == torch.bool and np.array_equal(have.numpy(), np.isnan(loss))


@pytest.mark.gpu
def test_the_loss_is_the_mean_over_nodes_with_a_target():
    from tests.test_gpu_vocab import _model
    w = _model("f32")
    N, V = w.num_nodes, 50
    rng = np.random.default_rng(5)
    tok = rng.integers(0, V, (N, 2))
    t = rng.standard_normal((N, 2)).astype(np.float32)
    t[::3] = -np.inf
    step = runner.VocabStep(w, V, None, tok, t)
    step.gradients()
    have = np.isfinite(t).any(1)
    loss = step.node_loss.cpu().numpy()
    assert (loss[have] != 0).all() and not loss[~have].any()
    assert step.scale == 1.0 / have.sum()


@pytest.mark.gpu
@pytest.mark.parametrize("tied", [False, True])
def test_a_batch_without_nodes(tied):
    """Loss rows and score rows of length zero; every gradient and so every step of Adam is zero, as in TrainStep."""
    import dataclasses

    from tests.test_gpu_vocab import _model
    w = _model("bf16")
    none = np.zeros(0, np.int32)
    empty = dataclasses.replace(w, graph_ptr=np.zeros(1, np.int32), node_op=none, child_ptr=np.zeros(1, np.int32),
                                child_idx=none, node_input=none, dh_roots=np.zeros((0, w.hidden), np.float32))
    V = w.leaf_table.shape[0] if tied else 50
    step = runner.VocabStep(empty, V, none, np.zeros((0, 3), np.int32), np.zeros((0, 3), np.float32), tied=tied)
    before = step.W.clone()
    step.step()
    assert step.node_loss.shape == (0,) and torch.equal(step.W, before)
    assert not step.dW.any() and not step.db.any()
    r = step.score(torch.zeros((0, 2), dtype=torch.int32, device="cuda"), 4)
    assert r.logp.shape == (0, 2) and r.top_token.shape == (0, 4)


@pytest.mark.gpu
def test_the_step_as_a_graph():
    """gradients() recorded once; every replay, with eager steps of Adam between, gives the eager gradients of the weights
    that it finds."""
    import gc

    from tests.test_gpu_vocab import _model, _targets
    w = _model("bf16")
    rng = np.random.default_rng(6)
    V = w.leaf_table.shape[0]
    tok, t, y = _targets(rng, w.num_nodes, V, 3)
    step = runner.VocabStep(w, V, y, tok, t, temperature=2.0, soft_weight=0.5, hard_weight=0.5, tied=True)
    tensors = [g for _, _, g in step.tensors]
    step.gradients()
    torch.cuda.synchronize()
    gc.collect()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.gradients()
    loss = step.node_loss
    for _ in range(3):
        step.step()
        step.gradients()
        want = [g.clone() for g in tensors] + [step.node_loss.clone()]
        for g in tensors:
            g.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, tensors + [loss]))
