"""A block's operators with outputs beside one another, as the gradient of one projection has them
(needs a GPU)."""
import math

import pytest
import torch

from paper_2205_11048_gb300 import binding as B
from tests.test_gpu_worker import IDS, TYPES, gen, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


def columns(n, d, many, gap, dtype):
    """A matrix with `many` columns of d side by side, `gap` elements between them, and those."""
    whole = torch.full((n, many * (d + gap)), math.nan, dtype=dtype, device="cuda")
    return whole, [whole[:, i * (d + gap):i * (d + gap) + d] for i in range(many)]


@pytest.mark.parametrize("dtype", TYPES, ids=IDS.get)
@pytest.mark.parametrize("n,d,gap", [(600, 64, 0), (37, 7, 0), (300, 501, 1), (5, 9000, 0), (260, 136, 8), (3, 1, 0)])
def test_outputs_beside_one_another(dtype, n, d, gap):
    """dx, df and dgate as columns of one matrix, the inputs as those of another: the bits of tensors of
    their own, and nothing between the columns is written."""
    w = B.Worker()
    g = gen(n + d)
    whole, (x, f, gate) = columns(n, d, 3, gap, dtype)
    into, (dx, df, dgate) = columns(n, d, 3, gap, dtype)
    for t in (x, f, gate):
        t.copy_(rand(g, n, d))
    seq, weight = B.sequences(1), torch.ones(d, device="cuda")
    block = B.residual_norm(post_norm="rms", gate="silu", post_weight=weight)
    y, _ = w.gated_scan(x, f, seq)
    z, stats = w.residual_norm(block, y, gate=gate)[1:]
    dz = rand(g, n, d, dtype=dtype)
    back = w.residual_norm_grad(block, None, dz, y, None, stats, gate, residual=False)
    want = w.gated_scan_grad(back["dx"], x, f, y, seq)
    m = B._matrix
    dh, sums = torch.empty_like(back["dx"]), torch.empty(d, device="cuda")
    grads = B.gba_block_grads(sums.data_ptr(), None, None, None)
    w._call("gba_residual_norm_grad", block.block, None, m(dz), m(y), None, m(gate), stats.data_ptr(), m(dh), None,
            m(dgate), grads)
    w._call("gba_gated_scan_grad", B.gba_scan(0, 1, 1, None, None), m(dh), None, m(x), m(f), None, m(y), m(dx), m(df), None)
    assert torch.equal(dh, back["dx"]) and torch.equal(dgate, back["dgate"]) and torch.equal(sums, back["dpost_weight"])
    assert torch.equal(dx, want[0]) and torch.equal(df, want[1])
    between = torch.ones_like(into, dtype=torch.bool)
    for i in range(3):
        between[:, i * (d + gap):i * (d + gap) + d] = False
    assert bool(into[between].isnan().all())
    # a scan's output beside its own inputs
    both, (a, b, out) = columns(n, d, 3, gap, dtype)
    a.copy_(x), b.copy_(f)
    w._call("gba_gated_scan", B.gba_scan(0, 1, 1, None, None), m(a), m(b), None, m(out), None)
    assert torch.equal(out, y) and torch.equal(a, x) and torch.equal(b, f) and bool(both[between].isnan().all())
    w.sync()
    w.close()
