"""The gates of a block's norms over their whole range, in the forms for narrow rows and for rows of any
width (needs a GPU)."""
import pytest
import torch

from paper_2205_11048_gb300 import binding as B
from tests.test_gpu_worker import U, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("cols", [8, 7, 300_007])
@pytest.mark.parametrize("gate", ["sigmoid", "silu"])
def test_gates_and_their_slopes(gate, cols):
    """exp(-g) by the hardware's power of two is off by 4 U of itself, and its argument by its rounding
    (|g| U) and that of log2(e) (0.23 |g| U); the sigmoid by one minus itself times that, and 4 U for the
    sum, the reciprocal and the product.  A slope sig (1 - sig), where these partly cancel, by all of it and
    10 U, and silu's, sig (1 + g (1 - sig)), by as much of the sum of its terms."""
    w = B.Worker()
    g = torch.linspace(-86.0, 86.0, 300_007 // cols * cols, device="cuda").view(-1, cols)
    one = torch.ones_like(g)
    block = B.residual_norm(gate=gate)
    z, stats = w.residual_norm(block, one, gate=g)[1:]
    got = w.residual_norm_grad(block, None, one, one, None, stats, gate=g, residual=False)["dgate"]
    x = g.double()
    sig, rest, own = torch.sigmoid(x), torch.sigmoid(-x), 1.23 * x.abs() + 4.0
    act, slope = (sig, sig * rest) if gate == "sigmoid" else (x * sig, sig * (1 + x * rest))
    size = slope if gate == "sigmoid" else sig * (1 + x.abs() * rest)
    within(z, act, U * act.abs() * (own * rest + 5.0), "act")
    within(got, slope, U * size * (own + 10.0), "slope")
    w.sync()
    w.close()
