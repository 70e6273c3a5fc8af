"""Infinities and NaN in the gradients of rows that occur often: their sums are merged from
several parts, and must be what a plain sum gives (needs a GPU)."""
import math

import pytest
import torch

from paper_2205_11048_gb300 import binding as B
from tests.test_gpu_worker import GRAD_ADDS, U, gen, plain_grad, rand, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


def same(got, want):
    """Equal, NaN and infinities included; of the finite ones only which they are."""
    return bool((got.isnan() == want.isnan()).all()) and bool((got.isposinf() == want.isposinf()).all()) and bool(
        (got.isneginf() == want.isneginf()).all())


# tokens in all, width, tokens of the hot row: runs of one item or of two by where they start, of
# several, of many, of very many; small calls, larger ones, and ones of longer items
@pytest.mark.parametrize("n,d,hot", [(50, 8, k) for k in range(14, 42)] + [
    (1000, 24, 300), (8000, 17, 5000), (9000, 8, 37), (20_000, 36, 400), (30_000, 20, 9000),
    (70_000, 1024, 130), (70_000, 1024, 1500), (70_000, 1024, 20_000)])
def test_a_hot_row_keeps_its_infinities(n, d, hot):
    w = B.Worker()
    g = gen(n + hot)
    V, row = 40, 17
    ids = torch.randint(0, V - 1, (n,), generator=g, device="cuda")
    ids[ids >= row] += 1
    where = torch.randperm(n, generator=g, device="cuda")[:hot]
    ids[where] = row
    where = where.sort().values
    grad = rand(g, n, d)
    a, b = where[hot // 3], where[hot - 1]
    inf = math.inf
    grad[a, 0] = inf
    grad[b, 1] = -inf
    grad[a, 2], grad[b, 2] = inf, -inf
    grad[b, 3] = math.nan
    grad[a, 4] = grad[b, 4] = 3e38  # finite ones whose sum is not
    grad[where[0], 5] = grad[a, 5] = inf
    grad[a, 6], grad[where[1], 6] = inf, math.nan
    want = torch.tensor([-inf, inf, math.nan, math.nan, -inf, -inf, math.nan], device="cuda")
    uniq, sums, mags = plain_grad(ids, grad, -2.0, None, V)
    at = int((uniq == row).nonzero())
    bound = GRAD_ADDS * U * mags
    out_rows, rows, count = w.embed_grad(ids, grad, V, scale=-2.0)
    assert int(count) == uniq.numel()
    dense = w.embed_grad_dense(ids, grad, torch.empty(V, d, device="cuda"), scale=-2.0)[uniq]
    more = w.embed_grad_dense(ids, grad, torch.zeros(V, d, device="cuda"), scale=-2.0, accumulate=True)[uniq]
    w.sync()
    for got in (rows[:uniq.numel()], dense, more):
        assert same(got[at, :7], want), got[at, :7].tolist()
        within(got[at, 7:], sums[at, 7:], bound[at, 7:], "finite columns")
        rest = torch.arange(uniq.numel(), device="cuda") != at
        within(got[rest], sums[rest], bound[rest], "other rows")
    w.close()


def test_an_infinity_in_a_hot_row_is_clipped_to_nothing():
    """The norm of such a message is infinite and not NaN, so its other gradients become zero."""
    w = B.Worker()
    ids = torch.full((600,), 3, device="cuda")
    ids[::2] = torch.arange(300, device="cuda") + 10
    grad = rand(gen(1), 600, 16)
    grad[101, 5] = math.inf
    _, rows, count = w.embed_grad(ids, grad, 400)
    norm = float(w.clip_grads([rows], 1.0))
    w.sync()
    assert norm == math.inf and int(count) == 301
    assert bool(rows[0, 5].isnan())
    rows[0, 5] = 0.0
    assert not bool(rows.any())
    w.close()
