"""AdamW with states in 8 bits that are rounded by chance: to one of the two codes next to a value, and
right on average over thousands of steps (needs a GPU)."""
import math

import pytest
import torch

from paper_2205_11048_gb300 import binding as B
from tests.test_gpu_block import BETAS, LR, read8
from tests.test_gpu_worker import gen

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


def chance_states(weights, **how):
    return B.adamw_states(weights, bits=8, rounding="chance", **how)


def between(m, v, i):
    """The codes below and above a block's m and v, and their scales."""
    def scale(x, share):
        return x.abs().amax().clamp(min=2.0**-100) * share

    ms, vs = scale(m, 1.0 / 448.0), scale(v, 1.0 / 1.875)
    q, r = m * (1.0 / ms), v * (1.0 / vs)
    a = q.abs()
    fine = (a * 512.0).floor() / 512.0
    bits = a.view(torch.int32)
    low = torch.where(a < 2.0**-6, fine, (bits & ~0xFFFFF).view(torch.float32))
    high = torch.where(a < 2.0**-6, fine + (a != fine) / 512.0, ((bits + 0xFFFFF) & ~0xFFFFF).view(torch.float32))
    low, high = low.clamp(max=448.0) * torch.sign(q), high.clamp(max=448.0) * torch.sign(q)
    c = r.view(torch.int32)
    below, above = ((c >> 20) - 768).clamp(1, 255), (((c + 0xFFFFF) >> 20) - 768).clamp(1, 255)
    none = r <= 0
    return low, high, ms, torch.where(none, 0, below), torch.where(none, 0, above), vs


def test_a_step_rounds_to_a_neighbour_and_is_right_on_average(w):
    """Blocks of one large element and others of a few sizes, from a step down to what a block hardly
    resolves.  The mean of n values that are each up or down, a step s apart, is off by more than
    6 s / (2 sqrt(n)) once in 10^9 times; 2^-19 s beside it is for the chances' 20 bits."""
    blocks, sizes = 400, torch.tensor([0.3, -0.07, 4.1e-3, 2.3e-4, -1.3e-5, 3e-6, 0.0], device="cuda")
    grad = sizes.repeat(37)[:256].repeat(blocks, 1)
    grad[:, 0] = 1.0
    flat = grad.reshape(-1)
    st = chance_states([torch.zeros_like(flat)], betas=BETAS)
    w.adamw(st.parts([flat]), LR)
    m = flat * (1.0 - BETAS[0])
    v = flat * flat * (1.0 - BETAS[1])
    low, high, ms, below, above, vs = between(m[:256], v[:256], 0)
    codes = st.m[0].view(torch.float8_e4m3fn).float().view(blocks, 256)
    cv = st.v[0].int().view(blocks, 256)
    assert bool((st.m_scale[0] == ms).all()) and bool((st.v_scale[0] == vs).all())
    assert bool(((codes == low) | (codes == high)).all())
    assert bool(((cv == below) | (cv == above)).all())
    got_m, got_v = [t.double() for t in read8(st, 0)]
    for x in sizes[:-1]:
        at = (flat == x).nonzero().view(-1)
        at, one = at[at % 256 != 0], int(at[at % 256 != 0][0])
        n = len(at)
        for got, want, up, down in ((got_m, m, high * ms, low * ms), (got_v, v, ((above + 768) << 20).view(torch.float32) * vs,
                                                                      ((below + 768) << 20).view(torch.float32) * vs)):
            s = abs(float(up[one]) - float(down[one]))
            if got is got_v and float(v[one]) < float(vs) * 1.125 * 2.0**-31:
                continue  # below the smallest code, which it is given
            assert abs(float(got[at].mean()) - float(want[one])) <= 6 * s / (2 * math.sqrt(n)) + 2.0**-19 * s + 1e-6 * abs(float(want[one])), float(x)
            if s > 1e-3 * abs(float(want[one])) and abs(float(want[one]) - float(down[one])) > 0.1 * s < abs(float(want[one]) - float(up[one])):
                assert len(got[at].unique()) == 2
    zero = flat == 0.0
    assert not got_m[zero].any() and not got_v[zero].any()


def test_equal_calls_and_unequal_places_in_memory(w):
    """The chances are those of the step, the tensor's place in the list and the element: not of the
    addresses, of how many tensors follow, or of whether a tensor lies on a vector's boundary."""
    n = 70_001
    grads = [[torch.randn(n, generator=gen(s), device="cuda") for s in (1, 2)] for _ in range(4)]
    made = []
    for i, off in enumerate((0, 1, 0, 0)):
        ws = [torch.zeros(n + off, device="cuda")[off:] for _ in range(2)]
        gs = [torch.cat([torch.zeros(off, device="cuda"), g])[off:] for g in grads[i]]
        if i == 2:  # more tensors, in a list of another kind
            ws += [torch.zeros(5, device="cuda") for _ in range(200)]
            gs += [torch.ones(5, device="cuda") for _ in range(200)]
        st = chance_states(ws, step=torch.tensor(7 if i == 3 else 0, device="cuda"))
        for _ in range(3):
            w.adamw(st.parts(gs), LR)
        made.append([*st.m[:2], *st.v[:2], *st.m_scale[:2], *st.v_scale[:2], *ws[:2]])
    for a, b, c in zip(made[0], made[1], made[2]):
        assert torch.equal(a, b) and torch.equal(a, c)
    assert not torch.equal(made[0][0], made[3][0]) and not torch.equal(made[0][2], made[3][2])
    same = chance_states([torch.zeros(n, device="cuda") for _ in range(2)])
    w.adamw(same.parts([grads[0][0], grads[0][0]]), LR)
    assert not torch.equal(same.m[0], same.m[1]) and not torch.equal(same.v[0], same.v[1])


def test_a_captured_step_goes_on(w):
    with torch.cuda.stream(torch.cuda.Stream()):
        w = B.Worker()
        n = 5_000
        grad = torch.randn(n, generator=gen(3), device="cuda")
        a, b = [chance_states([torch.zeros(n, device="cuda")]) for _ in range(2)]
        pa, pb = a.parts([grad]), b.parts([grad])
        w.adamw(pa, LR)
        w.adamw(pb, LR)
        w.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=w.stream):
            w.adamw(pa, LR)
        for _ in range(4):
            graph.replay()
            w.adamw(pb, LR)
        assert int(a.step) == 5
        assert torch.equal(a.m[0], b.m[0]) and torch.equal(a.v[0], b.v[0]) and torch.equal(a.weights[0], b.weights[0])
        w.sync()
        del graph
        w.close()


@pytest.mark.parametrize("beta2,steps", [(0.99, 4_000), (0.999, 12_000)])
def test_states_follow_gradients_that_fall(w, beta2, steps):
    """Blocks whose largest element keeps its gradient; the others' fall to a tenth after 1,000 steps, a
    quarter of them to nothing.  Against states in 32 bits.

    A rounding by chance adds nothing on average, so a state's mean is that of 32 bits.  Its variance: a step
    moves u by d <= (1 - b) |g^2 - u| and the rounding adds at most d s, with steps of s <= u / 8; while u is
    about v = g^2, V = b^2 V + (1 - b) (v^2 + v u + ...) / 8 with E u^2 = v^2 + V stays below
    3 v^2 / 16 / (1 - 1/8) < 0.22 v^2, whatever b, and m's likewise.  So the mean of n of them is within
    6 sqrt(0.22 / n) of v, with 10^-3 for the float32 roundings of some thousand steps; and weights move, by
    1 / sqrt(u) on average, at least as fast and (u is hardly below 0.4 v) less than 1.9 times."""
    blocks = 64
    first = torch.full((blocks, 256), 0.5, device="cuda")
    first[:, 0] = 1.0
    then = torch.full_like(first, 0.05)
    then[:, 192:] = 0.0
    then[:, 0] = 1.0
    sts = [B.adamw_states([torch.zeros(blocks * 256, device="cuda")], betas=(0.9, beta2), eps=1e-12),
           chance_states([torch.zeros(blocks * 256, device="cuda")], betas=(0.9, beta2), eps=1e-12)]
    parts = [[st.parts([g.reshape(-1)]) for st in sts] for g in (first, then)]
    for t in range(steps):
        if t == steps - 1000:
            before = [st.weights[0].clone() for st in sts]
        for p in parts[t >= 1000]:
            w.adamw(p, 1e-4)
    assert [int(st.step) for st in sts] == [steps, steps]
    m, v = [t.view(blocks, 256).double() for t in read8(sts[1], 0)]
    m32, v32 = [t.view(blocks, 256).double() for t in (sts[0].m[0], sts[0].v[0])]
    some, none = slice(1, 192), slice(192, 256)
    bound = 6 * math.sqrt(0.22 / (blocks * 191)) + 1e-3
    for got, want in ((m, m32), (v, v32)):
        ratio = (got / want)[:, some]
        assert abs(float(ratio.mean()) - 1.0) <= bound
        assert float(ratio.std()) <= 1.1 * math.sqrt(0.22)
    moved = [(st.weights[0] - b).view(blocks, 256).double() for st, b in zip(sts, before)]
    assert 0.95 <= float((moved[1] / moved[0])[:, some].mean()) <= 1.9
    assert not m[:, none].any()
