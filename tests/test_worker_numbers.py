"""Numbers that do not fit the library's types are refused, and not cut to their low bits.  Without
a GPU: stand-ins for tensors (see test_worker_devices.py), which hold no memory."""
import pytest
import torch

from paper_2205_11048_gb300 import binding as B
from tests.test_worker_devices import Stand, on, w  # noqa: F401

WIDE = 2**32 + 8  # columns: 8, in 32 bits


def wide(rows=1, cols=WIDE):
    return Stand(torch.empty(rows, cols, dtype=torch.bfloat16, device="meta"), 1)


def empty(*shape):
    return on(1, *shape)


REFUSED = {
    "columns of the weights": lambda w, ids: w.embed(wide(5), ids, out=wide(3)),
    "columns of the output": lambda w, ids: w.embed(empty(5, 8), ids, out=wide(3)),
    "columns of a gradient": lambda w, ids: w.embed_grad_dense(ids, wide(3), empty(5, 8)),
    "columns of a dense gradient": lambda w, ids: w.embed_grad_dense(ids, empty(3, 8), wide(5)),
    "the lookup's mode": lambda w, ids: w.embed(empty(5, 8), ids, id_mode=2**32, out=empty(3, 8)),
    "the gradient's mode": lambda w, ids: w.embed_grad(ids, empty(3, 8), 5, id_mode=2**32 + B.MODULO),
    "the dense gradient's mode": lambda w, ids: w.embed_grad_dense(ids, empty(3, 8), empty(5, 8), id_mode=-2**32),
    "a negative mode": lambda w, ids: w.embed(empty(5, 8), ids, id_mode=-1, out=empty(3, 8)),
    "the mode of a server's table": lambda w, ids: w.embed(empty(5, 8), ids, id_mode=B.HASH, out=empty(3, 8)),
    "the lookup's padding": lambda w, ids: w.embed(empty(5, 8), ids, pad_id=2**64 - 1, out=empty(3, 8)),
    "the gradient's padding": lambda w, ids: w.embed_grad(ids, empty(3, 8), 5, pad_id=2**64),
    "the dense gradient's padding": lambda w, ids: w.embed_grad_dense(ids, empty(3, 8), empty(5, 8), pad_id=-2**64),
    "the rows of a table": lambda w, ids: w.embed_grad(ids, empty(3, 8), 2**64 + 5),
}


@pytest.mark.parametrize("which", REFUSED)
def test_numbers_that_do_not_fit_are_refused(w, which):  # noqa: F811
    with pytest.raises(B.GBAError) as e:
        REFUSED[which](w, on(1, 3, dtype=torch.int64))
    assert e.value.status == B.GBA_E_ARG
    assert w.L.calls == []


def test_the_layer_norms_columns_are_refused(w, monkeypatch):  # noqa: F811
    monkeypatch.setattr(w, "_new", lambda *shape, dtype=None: Stand(torch.empty(shape, dtype=dtype, device="meta"), 1))
    for call in (lambda: w.layer_norm(wide(2)), lambda: w.layer_norm_grad(wide(2), wide(2), None, empty(2), empty(2))):
        with pytest.raises(B.GBAError) as e:
            call()
        assert e.value.status == B.GBA_E_ARG
    assert w.L.calls == []


def test_the_least_and_largest_numbers_are_taken(w):  # noqa: F811
    ids = on(1, 3, dtype=torch.int64)
    for pad in (-2**63, 2**63 - 1, -1, None):
        for mode in (B.DIRECT, B.MODULO):
            w.embed(empty(5, 8), ids, pad_id=pad, id_mode=mode, out=empty(3, 8))
    w.embed_grad(ids, empty(3, 8), 2**63 - 1)  # (the library refuses more than 2^32 - 3)
    assert len(w.L.calls) == 9
