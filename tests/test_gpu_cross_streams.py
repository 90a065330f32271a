"""Cross attention and its block away from the default stream, while the default stream is busy: nothing of a call may wait for
it, or come after it."""
import numpy as np
import pytest

from paper_1702_02181_amd import fold as F
from paper_1702_02181_amd import gen

pytestmark = pytest.mark.gpu

BUSY = 50_000_000  # cycles: some 20 ms and more


def _chains(seed, hidden=64):
    return gen.config3(seed=seed, num_graphs=9, hidden=hidden, vocab=100, emb_dim=64, leaf_range=(2, 20))


def test_rows_of_a_schedule_on_a_stream():
    """The list is there for the stream that it is made on, and for any other, when the call returns."""
    import torch
    from paper_1702_02181_amd.runner import DeviceRun
    run = DeviceRun(_chains(1))
    want = run.sched_arrays()["node_pos"]
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    with torch.cuda.stream(other):
        got = [F.schedule_rows(run.sched, side), F.schedule_rows(run.sched)]
        copies = [t.clone() for t in got]
        other.synchronize()
        assert all(np.array_equal(t.cpu().numpy(), want) for t in copies)
    torch.cuda.synchronize()
    assert np.array_equal(F.schedule_rows(run.sched).cpu().numpy(), want)


def _block(stream, kv_heads, busy=False):
    """out, dx, ds and the parameters' gradients of a block between two runs on `stream`, the current stream busy while the
    block's passes run."""
    import torch
    from paper_1702_02181_amd.runner import CrossBlock, DeviceRun
    target, source = (DeviceRun(_chains(s), stream=stream, with_backward=False) for s in (2, 3))
    torch.cuda.synchronize()  # the runs' own tensors
    rng = np.random.default_rng(4)
    up = torch.from_numpy(rng.standard_normal((target.N, target.ld)).astype(np.float32)).cuda()
    target.forward()
    source.forward()
    block = CrossBlock(target, source, 4, 200, kv_heads, seed=5)
    if busy:
        torch.cuda._sleep(BUSY)
    out = block.forward()
    dx, ds = block.backward(up)
    if stream is None:
        torch.cuda.synchronize()
    else:
        stream.synchronize()
        with torch.cuda.stream(stream):  # read there, not behind the busy stream
            return [t.cpu() for t in (out, dx, ds, *(g for _, _, g in block.tensors))]
    return [t.cpu() for t in (out, dx, ds, *(g for _, _, g in block.tensors))]


@pytest.mark.parametrize("kv_heads", [1, 4])  # of 16 columns each: pad columns behind k and v side by side, and none
def test_block_on_a_stream_of_its_own(kv_heads):
    import torch
    want = _block(None, kv_heads)
    got = _block(torch.cuda.Stream(), kv_heads, busy=True)
    torch.cuda.synchronize()
    assert all(torch.isfinite(t.float()).all() for t in got)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_block_of_runs_on_two_streams_is_refused():
    import torch
    from paper_1702_02181_amd.runner import CrossBlock, DeviceRun
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    runs = [DeviceRun(_chains(2), stream=s, with_backward=False) for s in (a, b, None)]
    torch.cuda.synchronize()
    for target, source in ((runs[0], runs[1]), (runs[0], runs[2]), (runs[2], runs[1])):
        with pytest.raises(ValueError, match="one stream"):
            CrossBlock(target, source, 4, 200)
    CrossBlock(runs[0], runs[0], 4, 200)
    torch.cuda.synchronize()


def test_counts_are_read_on_the_stream():
    """Lists that are written on the plan's stream just before: their ends are read behind that."""
    import torch
    side = torch.cuda.Stream()
    ends = [torch.tensor([0, 3, 7], dtype=torch.int32, device="cuda"), torch.tensor([0, 5, 9], dtype=torch.int32, device="cuda")]
    lists = [torch.zeros_like(e) for e in ends]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
        for t, e in zip(lists, ends):
            t.copy_(e)
    plan = F.CrossAttention(2, 32, *lists, dtype=torch.float32, stream=side)
    assert (plan.num_queries, plan.num_keys) == (7, 9)
    torch.cuda.synchronize()


def test_a_run_on_a_stream_of_its_own():
    """States and gradients of a run whose stream does not wait for the busy one that it was made on."""
    import torch
    from paper_1702_02181_amd.runner import DeviceRun
    w = _chains(2)
    rng = np.random.default_rng(1)
    up = rng.standard_normal((w.num_nodes, 64)).astype(np.float32)

    def states_and_grads(stream):
        run = DeviceRun(w, stream=stream, with_backward=True)
        run.forward()
        run.alloc_grads()
        run.set_upstream(np.zeros_like(w.dh_roots), up)
        run.zero_grads()
        if stream is not None:
            torch.cuda._sleep(BUSY)
        run.zero_grads()
        run.backward()
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            return [t.cpu() for t in (run.h_pool, run.c_pool, *(x for g in run.grad_tensors for x in g if x is not None), run.d_table)]
    want, got = states_and_grads(None), states_and_grads(torch.cuda.Stream())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got[:2], want[:2]))
    for a, b in zip(got[2:], want[2:]):  # (sums by atomics among them)
        assert b.any() and (a - b).abs().max() <= 1e-4 * b.abs().max()
