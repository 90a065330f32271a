"""The operators together, as a model uses them: two batches of graphs, a block of norms, layers and cross attention between
them, a vocabulary head, and the whole backward pass, against the oracle's chain in fp64."""
import numpy as np
import pytest

from oracle import block as OB
from oracle import vocab as OV
from paper_1702_02181_amd import gen
from tests.block_common import host

pytestmark = pytest.mark.gpu


def _models(dtype):
    if dtype == "f32":
        return (gen.config2(seed=21, num_graphs=6, leaves=7, hidden=64), gen.config2(seed=22, num_graphs=6, leaves=20, hidden=64))
    make = lambda seed, n, hi: gen.config3(seed=seed, num_graphs=n, hidden=64, vocab=200, emb_dim=64, leaf_range=(2, hi))  # noqa: E731
    return make(23, 12, 9), make(24, 6, 30)


def _build(dtype, lr=1e-3):
    from paper_1702_02181_amd.runner import CrossStep
    target, source = _models(dtype)
    G, S = len(target.graph_ptr) - 1, len(source.graph_ptr) - 1
    reads = np.arange(G) % S if dtype == "f32" else np.where(np.arange(G) == 3, -1, np.arange(G) // 2)
    rng = np.random.default_rng(5)
    labels = rng.integers(-1, 150, target.num_nodes)
    step = CrossStep(target, source, 150, labels, heads=4, wide=200, kv_heads=2, source_of=reads, seed=7, lr=lr)
    return step, target, source, reads, labels


def _oracle(step, target, source, reads, labels):
    """Losses and gradients by the definitions, with the weights as the step holds them."""
    from oracle import evaluate as EV
    from tests._helpers import oracle_batch, oracle_params
    H, blk = target.hidden, step.block
    fw = []
    for w in (target, source):
        b, P = oracle_batch(w), oracle_params(w)
        fw.append((b, P, EV.forward(b, P, H, w.leaf_table)))
    x, s = (f["h"] for _, _, f in fw)  # node order: lists are the identity
    W = [host(l.weight, l.in_dim) for l in (blk.q[0], blk.kv[0], blk.o[0], blk.first[0], blk.second[0])]
    a, ma, ra = OB.layer_norm(x)
    q, kv = OB.linear(a, W[0])[0], OB.linear(s, W[1])[0]
    k, v = kv[:, :blk.wk], kv[:, blk.wk:]
    lists = dict(heads=4, kv_heads=2, head_dim=H // 4, q_ptr=target.graph_ptr, k_ptr=source.graph_ptr, source=reads)
    o, _ = OB.attend(q, k, v, **lists)
    y = OB.linear(o, W[2], residual=x)[0]
    b, mb, rb = OB.layer_norm(y)
    f, pre = OB.linear(b, W[3], act="gelu")
    z = OB.linear(f, W[4], residual=y)[0]
    n, mz, rz = OB.layer_norm(z)
    head = host(step.W, H)
    loss, dlog = OV.distill(OV.head(n, head, np.zeros(150)), y=labels, soft=0.0, hard=1.0, scale=step.scale)
    dn, dhead, dhead_b = OV.head_backward(n, head, dlog)
    dz, dg2, db2 = OB.layer_norm_backward(z, dn, mean=mz, rstd=rz)
    df, dW4, db4, _ = OB.linear_backward(f, W[4], dz)
    db_, dW3, db3, _ = OB.linear_backward(b, W[3], df, "gelu", pre)
    dy, dg1, db1 = OB.layer_norm_backward(y, db_, mean=mb, rstd=rb)
    dy = dy + dz
    do, dW2, dbo, _ = OB.linear_backward(o, W[2], dy)
    dq, dk, dv = OB.attend_backward(q, k, v, do, **lists)
    dkv = np.concatenate([dk, dv], 1)
    ds, dW1, dbkv, _ = OB.linear_backward(s, W[1], dkv)
    da, dW0, dbq, _ = OB.linear_backward(a, W[0], dq)
    dx, dg0, db0 = OB.layer_norm_backward(x, da, mean=ma, rstd=ra)
    grads = {"dg0": dg0, "db0": db0, "dg1": dg1, "db1": db1, "dg2": dg2, "db2": db2, "Wq": dW0, "bq": dbq, "Wkv": dW1, "bkv": dbkv,
             "Wo": dW2, "bo": dbo, "W1": dW3, "b1": db3, "W2": dW4, "b2": db4, "head": dhead, "head_b": dhead_b}
    for tag, w, (ob, P, fwd), dh in (("target", target, fw[0], dx + dy), ("source", source, fw[1], ds)):
        bw = EV.backward(ob, P, H, w.leaf_table, fwd, np.zeros_like(w.dh_roots, dtype=np.float64), dh, want_table_grad=True)
        grads[tag + ".table"] = bw["d_table"]
        for i, g in enumerate(bw["grads"]):
            grads.update({f"{tag}.{i}.{k}": g[k] for k in ("W_in", "W_rec", "bias") if g.get(k) is not None})
    return n, loss, grads


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_step_against_the_oracle(dtype):
    import torch
    from oracle import compare
    from tests import gpu_common as C
    step, target, source, reads, labels = _build(dtype)
    step.gradients()
    torch.cuda.synchronize()
    n, loss, want = _oracle(step, target, source, reads, labels)
    blk, H = step.block, target.hidden
    got = {"head": host(step.dW, H), "head_b": host(step.db)}
    for i, (_, dg, _, db) in enumerate(blk.norms):
        got[f"dg{i}"], got[f"db{i}"] = host(dg), host(db)
    for name, (lin, dW, db) in (("q", blk.q), ("kv", blk.kv), ("o", blk.o), ("1", blk.first), ("2", blk.second)):
        got["W" + name], got["b" + name] = host(dW, lin.in_dim), host(db)
    for tag, run in (("target", step.target), ("source", step.source)):
        sets, table = run.weight_grads()
        got[tag + ".table"] = table
        for i, g in enumerate(sets):
            got.update({f"{tag}.{i}.{k}": g[k] for k in ("W_in", "W_rec", "bias") if g.get(k) is not None})
    # keys' biases move every score of a row alike: their gradient is a sum of zeros, compared beside the values' part
    errs = {k: compare.rel_err(v, want[k], whole=True) for k, v in got.items() if k in want}
    assert set(got) <= set(want) | {k for k in got if not np.any(got[k])}
    states = host(blk.forward(), H)[step.target.sched_arrays()["node_pos"]]
    errs["states"], errs["loss"] = compare.rel_err(states, n), compare.rel_err(host(step.node_loss), loss)
    assert all(v <= C.TOL[dtype] for v in errs.values()), errs


def test_step_as_a_graph():
    """The launches of gradients() captured: replays with Adam between them equal eager steps bit for bit where no sum is
    taken by atomics (the block's and the head's own gradients and the losses of the first replay)."""
    import gc

    import torch
    step, *_ = _build("bf16")
    step.gradients()
    step.gradients()
    torch.cuda.synchronize()
    eager = [g.clone() for _, _, g in step.block.tensors] + [step.dW.clone(), step.node_loss.clone()]
    gc.collect()  # device memory of other tests' garbage, freed by a collection during the recording, would end it
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.gradients()
    loss = step.node_loss
    for it in range(3):
        graph.replay()
        torch.cuda.synchronize()
        got = [g for _, _, g in step.block.tensors] + [step.dW, loss]
        assert all(torch.equal(a, b) for a, b in zip(got, eager)), it


def test_steps_run():
    import torch
    step, *_ = _build("bf16")
    before = step.logits().clone()
    for _ in range(3):
        step.step()
    after = step.logits()
    assert torch.isfinite(after.float()).all() and not torch.equal(before, after)
