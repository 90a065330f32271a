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
