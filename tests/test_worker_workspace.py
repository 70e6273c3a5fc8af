"""What becomes of a worker's workspace when a call needs a larger one: captured graphs
hold its address, so it is there until the handle is destroyed.  Without a GPU (see
test_worker_host.py)."""
from paper_2205_11048_gb300 import binding as B
from tests.test_worker_host import AT, F, FAR, MALLOC, grad, ln_grad, mat, norm, w  # noqa: F401

BIG = dict(n=4000, g=mat(4000, data=FAR), ids=AT + (1 << 18), ids_out=FAR + (1 << 18), rows_out=FAR + (1 << 19))


def test_growth_frees_no_workspace(F, w):  # noqa: F811
    assert grad(F, w) == B.GBA_OK
    n = F.fake_allocations()
    assert grad(F, w, **BIG) == B.GBA_OK
    assert F.fake_allocations() == n + 1
    assert grad(F, w) == norm(F, w, (AT, None, 4, 0, 0)) == ln_grad(F, w) == grad(F, w, **BIG) == B.GBA_OK
    assert F.fake_allocations() == n + 1  # and calls of a size that was there allocate nothing


def test_a_workspace_that_could_not_grow_is_kept(F, w):  # noqa: F811
    assert grad(F, w) == B.GBA_OK
    n = F.fake_allocations()
    F.fake_fail(MALLOC, 1)
    assert grad(F, w, **BIG) == B.GBA_E_OOM
    assert F.gba_worker_last_error(w)
    assert F.fake_allocations() == n
    F.fake_fail(MALLOC, 1)
    assert grad(F, w) == B.GBA_OK  # without an allocation
    F.fake_fail(MALLOC, 0)


def test_a_worker_of_ever_larger_calls(F, w):  # noqa: F811
    """Every size of the norm's workspace up to its largest: growth is by a quarter, so there are
    few of them (the fixture checks that all are freed in the end)."""
    n = F.fake_allocations()
    parts = (B.gba_grad_part * (1 << 20))()
    for k in range(40):
        size = int(1.4**k)
        assert F.gba_grad_norm(w, parts, min(size, 1 << 20), AT) == B.GBA_OK
    assert F.fake_allocations() <= n + 62  # log of 2^20 to the base 1.25
