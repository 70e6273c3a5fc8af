"""Gated scans of no rows whose offsets or lengths are bad (needs a GPU)."""
import pytest
import torch

from paper_2205_11048_gb300 import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.mark.parametrize("how,good", [(dict(offsets=[0, 0, 0]), True), (dict(offsets=[0, 1, 1]), False),
                                      (dict(offsets=[-1, 0, 0]), False), (dict(lengths=[0, 0]), True),
                                      (dict(lengths=[0, 1]), False)])
def test_sequences_of_no_rows(how, good):
    w = B.Worker()
    e = torch.empty(0, 8, device="cuda")
    seq = B.sequences(2, **{k: torch.tensor(v, device="cuda") for k, v in how.items()})
    w.gated_scan_grad(e, e, e, e, seq)  # without states there is nothing to write either
    if good:
        w.sync()
    else:
        with pytest.raises(B.GBAError) as err:
            w.sync()
        assert err.value.status == B.GBA_E_ARG and "offsets" in str(err.value)
    w.sync()
    w.close()
