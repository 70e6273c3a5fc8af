"""The worker's operators together, as examples/token_worker.py uses them (needs a GPU)."""
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
    spec = importlib.util.spec_from_file_location("token_worker", os.path.join(ROOT, "examples", "token_worker.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("most", [0.05, 0.001])
def test_a_workers_message_is_the_clipped_gradient_of_its_loss(E, most):
    """Against automatic differentiation of the same model in 64 bits.  float32 gradients of this
    size (means of some hundred terms, two of them through a norm) are within about 1e-5 of
    their largest element; 1e-4 leaves room for the products of torch's own float32 head."""
    torch.backends.cuda.matmul.allow_tf32 = False
    with torch.cuda.stream(torch.cuda.Stream()):
        model = E.Model(vocabulary=301, dim=40, classes=5)
        adam = B.opt_desc(B.ADAM, 0.01)
        server = B.GBA([(model.vocabulary, model.dim, B.DIRECT, 4096, adam)], model.dense, adam, 64, 4, seed=3)
        worker = E.TokenWorker(model, server, max_norm=most)
        ids, labels = E.batches(model, 48, 20, torch.Generator(device="cuda").manual_seed(1))
        loss, (token, rows_of, rows, dense) = worker.message(ids, labels)
        worker.ops.sync()
        table = server.table(0)[0].double().requires_grad_()
        flat = server.dense()[0].double().requires_grad_()
        gamma, beta, head = model.split(flat)
        real = ids != E.PAD
        x = table[ids.clamp(min=0)] * math.sqrt(model.dim) * real[..., None]
        mean = x.mean(-1, keepdim=True)
        y = (x - mean) / ((x - mean).square().mean(-1, keepdim=True) + 1e-5).sqrt() * gamma + beta
        share = real.double() / real.sum(1, keepdim=True)
        want = torch.nn.functional.cross_entropy((y * share[..., None]).sum(1) @ head, labels)
        want.backward()
        norm = torch.sqrt(table.grad.square().sum() + flat.grad.square().sum())
        coef = min(1.0, most / (float(norm) + 1e-6))
        assert token == 0 and abs(float(loss) - float(want.detach())) <= 1e-5
        got = torch.zeros_like(table).index_add_(0, rows_of[0], rows[0].double())
        for a, b in ((got, table.grad * coef), (dense.double(), flat.grad * coef)):
            assert float((a - b).abs().max()) <= 1e-4 * float(b.abs().max())
        server.close()


def test_the_example_learns(E):
    losses = E.train(steps=60)
    assert all(math.isfinite(x) for x in losses)
    assert sum(losses[-5:]) / 5 < 0.6 * losses[0]
