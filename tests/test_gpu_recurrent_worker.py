"""A block's operators together, as examples/recurrent_worker.py uses them (needs a GPU)."""
import importlib.util
import math
import os

import pytest
import torch

from paper_2205_11048_gb300 import binding as B

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def E():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)
    at = os.path.join(ROOT, "examples", "recurrent_worker.py")
    spec = importlib.util.spec_from_file_location("recurrent_worker", at)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def rms(x, w):
    return x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w


def plain_loss(m, table, head, weights, ids, lengths, labels):
    """The model by its formulas, in the weights' type."""
    real = torch.arange(ids.shape[1], device="cuda") < lengths[:, None]
    z = table[ids.clamp(min=0)] * math.sqrt(m.dim) * real[..., None]
    first, rest = weights[0], weights[1:]
    y = rms(z, first)
    for i in range(len(m.blocks)):
        into, out, post, pre = rest[4 * i:4 * i + 4]
        x, f, gate = (y @ into).chunk(3, -1)
        a, h, hs = torch.sigmoid(f), torch.zeros_like(x[:, 0]), []
        for t in range(ids.shape[1]):
            h = a[:, t] * h + (1 - a[:, t]) * x[:, t]
            hs.append(h)
        h = torch.stack(hs, 1) * real[..., None]
        z = z + gate * torch.sigmoid(gate) * rms(h @ out, post)
        y = rms(z, pre)
    logp = torch.log_softmax(y @ head, -1).gather(-1, labels.clamp(min=0)[..., None])[..., 0]
    return -(logp * real).sum() / real.sum()


def test_the_gradients_are_those_of_the_loss(E):
    """Against automatic differentiation of the same model in 64 bits.  A float32 gradient is a sum of
    up to n t = 700 terms through a dozen roundings each; products of up to 120 terms round by 120 U.
    700 U + 12 * 120 U < 1.3e-4 of what is summed, taken as ten times the largest element."""
    torch.backends.cuda.matmul.allow_tf32 = False
    with torch.cuda.stream(torch.cuda.Stream()):
        adam = B.opt_desc(B.ADAM, 0.01)
        server = B.GBA([(301, 40, B.DIRECT, 4096, adam)], 40 * 7, adam, 35, 2, seed=3)
        model = E.Recurrent(server, 301, 40, classes=7, seed=1)
        ids, lengths, labels = E.batches(model, 35, 20, torch.Generator(device="cuda").manual_seed(1))
        loss, own, rows_of, rows, dhead = model.gradients(ids, lengths, labels)
        model.ops.sync()
        table = server.table(0)[0].double().requires_grad_()
        head = server.dense()[0].double().view(40, 7).requires_grad_()
        weights = [w.double().requires_grad_() for w in model.weights]
        want = plain_loss(model, table, head, weights, ids, lengths, labels)
        want.backward()
        assert abs(float(loss) - float(want.detach())) <= 1.3e-4 * 10
        got = torch.zeros_like(table).index_add_(0, rows_of, rows.double())
        for a, b in [(got, table.grad), (dhead, head.grad), *zip(own, (w.grad for w in weights))]:
            assert float((a.double() - b).abs().max()) <= 1.3e-3 * float(b.abs().max())
        model.ops.close()
        server.close()


def test_a_sequence_token_by_token_gives_its_last_state(E):
    with torch.cuda.stream(torch.cuda.Stream()):
        adam = B.opt_desc(B.ADAM, 0.01)
        server = B.GBA([(301, 40, B.DIRECT, 4096, adam)], 40 * 7, adam, 35, 2, seed=3)
        model = E.Recurrent(server, 301, 40, classes=7, seed=1)
        ids = torch.randint(0, 301, (6, 30), device="cuda")
        _, last, _ = model.forward(ids, B.sequences(6))
        states = [torch.zeros(6, 40, device="cuda") for _ in model.blocks]
        for t in range(30):
            model.next(ids[:, t], states)
        model.ops.sync()
        # both round what they compute by some hundred U of a value of a few units (see above)
        for a, b in zip(states, last):
            assert float((a - b).abs().max()) <= 1.3e-4 * max(1.0, float(b.abs().max()))
        model.ops.close()
        server.close()


def test_the_example_runs(E):
    losses = E.train(steps=12)
    assert len(losses) == 12 and all(math.isfinite(x) for x in losses)
