"""The decays of the gated scan, one by one and through long memories (needs a GPU).

A sequence of one row tells a gate's decay and one minus it: with a state of 1, an input of 0 and
no tie y is the decay itself, and tied, with an input of 1 and no state, y is one minus it."""
import math

import pytest
import torch

from paper_2205_11048_gb300 import binding as B
from tests.test_gpu_block import plain_scan
from tests.test_gpu_worker import U, gen, rand, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.fixture
def w():
    worker = B.Worker()
    yield worker
    worker.sync()
    worker.close()


def gates_of(w, f, decay):
    one, zero, seq = torch.ones_like(f), torch.zeros_like(f), B.sequences(f.shape[0])
    a = w.gated_scan(zero, f, seq, decay=decay, tied=False, state=one)[0]
    rest = w.gated_scan(one, f, seq, decay=decay, tied=True)[0]
    tied = w.gated_scan(zero, f, seq, decay=decay, tied=True, state=one)[0]
    return a, rest, tied


def test_log_decays(w):
    """Down to -0.69 one minus the decay is a quotient within 5.3 U of itself (its denominator 2.2 with
    what its series leaves out, a reciprocal 2, a product 1), and the decay, at least a half, one minus that,
    rounded once (half of U at the most).  Untied, down to -1/16 the decay is a series within 3 U of one
    minus it, rounded once.  Below, the hardware's power of two is off by 4 U of itself, and its
    argument by its own rounding (|f| U) and that of log2(e) to 24 bits, which is off by 0.23 U of itself;
    its difference from one is exact but for U."""
    f = -torch.cat([torch.logspace(-12, 1.9, 100_000, device="cuda"), torch.linspace(0.0, 1.5, 100_001, device="cuda")])
    f = torch.cat([f, -f[:10]]).view(1, -1)
    want = f.double().clamp(max=0.0).exp()
    least = -torch.expm1(f.double().clamp(max=0.0))
    near = f > -0.69
    off = (1.23 * f.abs().double() + 5.0) * U * want
    a, rest, tied = gates_of(w, f, "log")
    within(rest, least, torch.where(near, 5.3 * U * least, off + U), "1 - a")
    for k, at in ((a, f > -0.0625), (tied, near)):
        within(k, want, torch.where(at, 0.5 * U + 5.3 * U * least, off), "a")
    # so a constant input is kept: the two add up to one but for the decay's rounding
    within((tied.double() + rest.double())[near], torch.ones_like(want)[near], 0.5 * U, "a + (1 - a)")


def test_sigmoid_decays(w):
    """The hardware's power of two is off by 4 U of itself, and its argument by its own rounding (|f| U) and
    that of log2(e) (0.23 |f| U): a by one minus a times that, and one minus a by a times it, with 4 U for the
    sum, the quotient and the product."""
    f = torch.linspace(-86.0, 86.0, 300_001, device="cuda").view(1, -1)
    want, least = torch.sigmoid(f.double()), torch.sigmoid(-f.double())
    own = 1.23 * f.abs().double() + 4.0
    a, rest, tied = gates_of(w, f, "sigmoid")
    within(rest, least, U * least * (own * want + 4.0), "1 - a")
    for k in (a, tied):
        within(k, want, U * want * (own * least + 4.0), "a")


@pytest.mark.parametrize("tied", [True, False])
@pytest.mark.parametrize("f", [-1e-4, -1e-3])
def test_a_long_memory_of_log_decays(w, f, tied):
    """A constant decay near one over many times its memory.  A step adds half of U for the decay, 5.3 U
    of one minus it, and four roundings (of the input, of its own sum, and of the pairs that it is joined
    through)."""
    rows, d = 100_000, 8
    g = gen(5)
    x, fs = rand(g, rows, d, mean=1.0), torch.full((rows, d), f, device="cuda")
    y, last = w.gated_scan(x, fs, B.sequences(1), decay="log", tied=tied)
    want, h, _, _ = plain_scan(x, fs, [0], [rows], "log", tied, None)
    a = math.exp(float(fs[0, 0]))
    rest = -math.expm1(float(fs[0, 0]))
    size = x.double().abs() * (rest if tied else 1.0)
    m = torch.zeros_like(size)
    units = torch.zeros_like(size)
    total, bound = torch.zeros(d, dtype=torch.float64, device="cuda"), torch.zeros(d, dtype=torch.float64, device="cuda")
    # both by chunks: the sums of a^(n-i) over a chunk, and what the chunk before leaves
    step = 2000
    powers = a ** torch.arange(step, -1, -1, dtype=torch.float64, device="cuda")[:, None]
    down = torch.tril(a ** (torch.arange(step, device="cuda")[:, None] - torch.arange(step, device="cuda")).clamp(min=0).double())
    for i in range(0, rows, step):
        m[i:i + step] = down @ size[i:i + step] + powers[:-1].flip(0) * total
        total = m[i + step - 1]
        units[i:i + step] = down @ ((0.5 + 5.3 * rest + 4.0) * m[i:i + step] + 5.3 * size[i:i + step]) + powers[:-1].flip(0) * bound
        bound = units[i + step - 1]
    within(y, want, U * want.abs() + U * units, "y")
    within(last, h, U * h.abs() + U * units[-1:], "last")
