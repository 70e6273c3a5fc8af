"""AdamW of gradients whose squares leave the normal numbers, beside an eps that is smaller still
(needs a GPU)."""
import pytest
import torch

from paper_2205_11048_gb300 import binding as B
from tests.test_gpu_block import BETAS, LR, by_blocks, read8, to_m8, to_v8
from tests.test_gpu_worker import TINY, U, UNIT, gen, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("eps", [1e-30, 2.0**-126])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [0, 1])
def test_small_gradients_and_a_small_eps(bits, offset, eps):
    """Second moments from normal numbers down to none.  The moments are those of the formulas, rounded
    one operation after another, and the weight is within 16 U of its movement (see test_gpu_block.py).
    What a block does not resolve is a code of at least 1."""
    w = B.Worker()
    g = gen(7)
    n = 2048 + 77
    size = 10.0 ** -torch.linspace(15.0, 22.4, n, device="cuda").double()
    if bits == 8:
        size = size.view(-1)  # blocks of neighbours: of about one size
    flat = torch.zeros(n + offset, device="cuda")
    weights = [flat[offset:]]
    st = B.adamw_states(weights, bits=bits, betas=BETAS, eps=eps)
    for step in (1, 2, 3):
        grad = (size * torch.sign(torch.randn(n, generator=g, device="cuda"))).float()
        w0 = weights[0].double()
        m, v = [t.clone() for t in read8(st, 0)] if bits == 8 else (st.m[0].clone(), st.v[0].clone())
        w.adamw(st.parts([grad]), LR)
        m = m * BETAS[0] + grad * (1.0 - BETAS[0])
        v = v * BETAS[1] + grad * grad * (1.0 - BETAS[1])
        if bits == 8:
            for fn, x, codes, scales in ((to_m8, m, st.m[0], st.m_scale[0]), (to_v8, v, st.v[0], st.v_scale[0])):
                c, s = by_blocks(fn, x)
                assert torch.equal(codes, c) and torch.equal(scales, s)
        else:
            assert torch.equal(st.m[0], m) and torch.equal(st.v[0], v)
        assert bool(((v > 0) & (v < 2.0**-126)).any()) and bool((v > 2.0**-126).any())
        move = LR * (m.double() / (1 - BETAS[0]**step)) / ((v.double() / (1 - BETAS[1]**step)).sqrt() + eps)
        bound = 16 * U * move.abs() + 2 * U * w0.abs()
        want = w0 - move
        within(weights[0], want, UNIT[torch.float32] * want.abs() + 2 * bound + TINY[torch.float32], "weight")
    w.sync()
    w.close()
