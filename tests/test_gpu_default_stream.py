"""A server whose calls are made while the default stream is current (needs a GPU): its work is that
stream's, as it is any other current stream's."""
import ctypes

import pytest
import torch

from paper_2205_11048_gb300 import binding as B

pytestmark = pytest.mark.gpu

ROWS, DIM, DENSE, IDS = 50_000, 64, 1_000_000, 20_000
DELAY = 100_000_000  # cycles: some 50 ms


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


def server():
    adam = B.opt_desc(B.ADAM, 0.01)
    return B.GBA([(ROWS, DIM, B.DIRECT, IDS, adam)], DENSE, adam, 1, 4, seed=3)


def message():
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(0, ROWS, (IDS,), generator=g, device="cuda")
    return ids, torch.randn(IDS, DIM, generator=g, device="cuda"), torch.randn(DENSE, generator=g, device="cuda")


def step(g, ids, rows, dense):
    g.push(0, [ids], [rows], dense, 1)
    assert g.try_apply() == 1


def weights(g):
    """The table's weights as work of the current stream finds them, without waiting for the handle."""
    w = ctypes.c_void_p()
    B.check(g.L.gba_get_table(g.h, 0, ctypes.byref(w), None, None, None), g.h)
    return B._copy_device(w.value, ROWS * DIM, torch.float32)


@pytest.fixture
def want():
    """What a step leaves, every tensor and result waited for."""
    g, made = server(), message()
    torch.cuda.synchronize()
    step(g, *made)
    g.sync()
    table, dense = g.table(0)[0], g.dense()[0]
    torch.cuda.synchronize()
    yield table.view(-1), dense
    g.close()


def test_a_push_reads_what_the_default_stream_wrote_before(want):
    assert torch.cuda.current_stream().cuda_stream == 0
    g, made = server(), message()
    late = [torch.zeros_like(t) for t in made]
    torch.cuda.synchronize()
    torch.cuda._sleep(DELAY)
    for a, b in zip(late, made):
        a.copy_(b)
    step(g, *late)
    g.sync()
    assert torch.equal(g.table(0)[0].view(-1), want[0]) and torch.equal(g.dense()[0], want[1])
    g.close()


def test_the_default_stream_reads_what_a_step_wrote_before(want):
    g, made = server(), message()
    torch.cuda.synchronize()
    torch.cuda._sleep(DELAY)  # so that a step beside the stream would come first, and one on it last
    before = weights(g)
    step(g, *made)
    g.join()
    after = weights(g)
    g.sync()
    torch.cuda.synchronize()
    assert torch.equal(after, want[0]) and not torch.equal(before, after)
    g.close()


def test_a_pull_is_there_for_the_default_stream(want):
    g, made = server(), message()
    ids = torch.arange(ROWS, device="cuda")
    stale = torch.full((ROWS, DIM), float("nan"), device="cuda")
    step(g, *made)
    g.sync()
    torch.cuda.synchronize()
    del stale  # the pull's memory, perhaps
    for _ in range(20):  # work ahead of the pull
        g.push(1, [made[0]], [made[1]], made[2], 1)
        assert g.try_apply() == 1
    got = g.pull(0, ids).clone()
    g.sync()
    torch.cuda.synchronize()
    assert torch.equal(got.view(-1), g.table(0)[0].view(-1))
    g.close()


def test_an_event_of_the_default_stream_covers_the_steps_before_it():
    """Time between events, as a benchmark takes it, is that of the work and not of its enqueueing."""
    g, made = server(), message()
    done, start = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    start.record()
    for k in range(20):
        g.push(k, [made[0]], [made[1]], made[2], 1)
        assert g.try_apply() == 1
    g.join()
    done.record()
    done.synchronize()
    version = weights(g)  # all steps are done: nothing writes any more
    torch.cuda.synchronize()
    g.sync()
    assert torch.equal(version, g.table(0)[0].view(-1)) and start.elapsed_time(done) > 0.0
    g.close()
