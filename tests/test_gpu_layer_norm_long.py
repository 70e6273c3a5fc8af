"""Layer norm's gradient of very many rows (needs a GPU): what the sums over rows lose does not
grow with the rows.

The weight's gradients are sums in float32 in which a term passes through at most DEPTH additions:
512 rows of a thread, 5 between lanes, 16 between the groups of a block, the partial rows of a
launch by 32 warps (at most 2,048 blocks: 64), one for each launch (at most 40 here) and 31
between the warps; 8 more for the terms' own roundings."""
import pytest
import torch

from paper_2205_11048_gb300 import binding as B
from tests.test_gpu_worker import TINY, U, UNIT, within

pytestmark = pytest.mark.gpu

DEPTH = 512 + 5 + 16 + 64 + 40 + 31 + 8


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)
    yield
    torch.cuda.empty_cache()  # tens of GB


@pytest.mark.parametrize("n,d", [(5_000_000, 1003), (4_000_000, 1040)])
def test_equal_values_are_added_up(n, d):
    """The same value in every row: each addition to a long sum rounds the same way."""
    w = B.Worker()
    x = torch.full((n, d), 2.0, device="cuda")
    mean, rstd = torch.ones(n, device="cuda"), torch.full((n,), 0.5, device="cuda")
    value = float(torch.tensor(0.7))
    dx, dgamma, dbeta = w.layer_norm_grad(torch.full((n, d), value, device="cuda"), x, None, mean, rstd)
    w.sync()
    want = torch.full((d,), value * n, dtype=torch.float64)
    within(dbeta.cpu(), want, DEPTH * U * want, "dbeta")
    within(dgamma.cpu(), want / 2, DEPTH * U * want / 2, "dgamma")
    # every column has the same g and h = 0.5: dx = rstd (g - g - 0.5 (0.5 g)), up to its means' rounding
    within(dx[::4999].cpu(), torch.full((1 + (n - 1) // 4999, d), -0.125 * value, dtype=torch.float64), 1e-4 * value, "dx")
    w.close()


# rows held by lanes, by warps, through shared memory, of more columns than are read ahead, of any width
@pytest.mark.parametrize("n,d,dtype", [
    (100_000_007, 8, torch.float32), (100_000_003, 16, torch.bfloat16), (9_000_001, 66, torch.float16),
    (2_000_003, 520, torch.bfloat16), (600_001, 1040, torch.float32), (100_003, 8200, torch.bfloat16),
    (100_003, 5001, torch.float32), (70_001, 8201, torch.float16)])
def test_every_row_of_a_long_call_is_taken_once(n, d, dtype):
    w = B.Worker()
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(n, d, generator=g, device="cuda", dtype=dtype)
    dy = torch.randn(n, d, generator=g, device="cuda", dtype=dtype)
    gamma = torch.rand(d, generator=g, device="cuda") + 0.5
    _, mean, rstd = w.layer_norm(x, gamma)
    dx, dgamma, dbeta = w.layer_norm_grad(dy, x, gamma, mean, rstd)
    w.sync()
    sums = torch.zeros(5, d, dtype=torch.float64, device="cuda")
    step = 1 + (1 << 27) // d
    k = 16 + d // 1024 + 5 + 32 + 4  # additions of a row's sums, as in test_gpu_worker.py
    for i in range(0, n, step):
        e, r, m = dy[i:i + step].double(), rstd[i:i + step, None].double(), mean[i:i + step, None].double()
        xs = x[i:i + step].double()
        h = (xs - m) * r
        dh = 3 * U * r * (xs.abs() + m.abs())
        sums += torch.stack([e.sum(0), e.abs().sum(0), (e * h).sum(0), (e * h).abs().sum(0),
                             (e.abs() * dh).sum(0)])
        gg = e * gamma.double()
        mg, mgh = gg.mean(1, keepdim=True), (gg * h).mean(1, keepdim=True)
        want = r * (gg - mg - h * mgh)
        e_mg = (k + 2) * U * gg.abs().mean(1, keepdim=True)
        e_mgh = (k + 3) * U * (gg * h).abs().mean(1, keepdim=True) + (gg.abs() * dh).mean(1, keepdim=True)
        tol = r * (e_mg + h.abs() * e_mgh + dh * mgh.abs() + 5 * U * (gg.abs() + mg.abs() + (h * mgh).abs()))
        within(dx[i:i + step], want, tol * 1.01 + UNIT[dtype] * want.abs() + TINY[dtype], "dx")
    within(dbeta, sums[0], DEPTH * U * sums[1], "dbeta")
    within(dgamma, sums[2], DEPTH * U * sums[3] + sums[4], "dgamma")
    w.close()
