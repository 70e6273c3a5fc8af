"""Outputs that overlap an input, or another output, are refused.  Without a GPU (see
test_worker_host.py)."""
import pytest

from paper_2205_11048_gb300 import binding as B
from tests.test_worker_host import AT, F, FAR, clip, dense, embed, grad, mat, w  # noqa: F401

IDS = AT + (1 << 18)  # of a lookup: 3, 24 bytes; its output is 96 bytes
OVERLAPS = {
    "lookup: out at the ids": lambda F, w: embed(F, w, out=mat(3, data=IDS)),
    "lookup: out's end at the ids": lambda F, w: embed(F, w, out=mat(3, data=IDS - 92)),
    "lookup: the ids' end at out": lambda F, w: embed(F, w, out=mat(3, data=IDS + 20)),
    "lookup: the ids in out's last row": lambda F, w: embed(F, w, out=mat(3, stride=100, data=IDS - 800)),
    # a gradient of 4 tokens: ids 32 bytes at AT, gradient 128 at FAR
    "gradient: rows at the ids": lambda F, w: grad(F, w, rows_out=AT),
    "gradient: rows' end at the ids": lambda F, w: grad(F, w, ids=AT + 8192 + 120),
    "gradient: ids out at the gradient": lambda F, w: grad(F, w, ids_out=FAR + 120),
    "gradient: ids out's end at the gradient": lambda F, w: grad(F, w, ids_out=FAR - 24),
    "gradient: count at the ids": lambda F, w: grad(F, w, n_out=AT + 24),
    "gradient: count at the gradient": lambda F, w: grad(F, w, n_out=FAR + 64),
    "gradient: count at the ids out": lambda F, w: grad(F, w, n_out=AT + 4096 + 8),
    "gradient: count at the rows": lambda F, w: grad(F, w, n_out=AT + 8192 + 120),
    "gradient: ids out at the rows": lambda F, w: grad(F, w, ids_out=AT + 8192),
    "gradient: ids out's end at the rows": lambda F, w: grad(F, w, ids_out=AT + 8192 - 24),
    "dense gradient: out's end at the ids": lambda F, w: dense(F, w, out=mat(10, data=AT + 28)),
    "clipping: norm at a gradient": lambda F, w: clip(F, w, (FAR, AT + 64, 4, 0, 0), out=FAR + 12),
    "clipping: norm at an output": lambda F, w: clip(F, w, (FAR, AT, 4, 0, 0), out=AT),
    "clipping: norm at a 16-bit output": lambda F, w: clip(F, w, (FAR, AT, 5, 0, 1), out=AT + 8),
    "clipping: norm at a later part": lambda F, w: clip(F, w, (FAR, AT, 4, 0, 0), (AT + 64, AT + 64, 3, 1, 1), out=AT + 64),
}
APART = [
    lambda F, w: embed(F, w, out=mat(3, data=IDS + 24)),
    lambda F, w: embed(F, w, out=mat(3, data=IDS - 96)),
    lambda F, w: grad(F, w, rows_out=AT + 32),
    lambda F, w: grad(F, w, ids_out=FAR - 32),
    lambda F, w: grad(F, w, n_out=AT + 32),
    lambda F, w: grad(F, w, n_out=AT + 4096 + 32),
    lambda F, w: grad(F, w, ids_out=AT + 8192 - 32, n_out=AT + 8192 + 128),
    lambda F, w: clip(F, w, (FAR, AT, 4, 0, 0), out=AT + 16),
    lambda F, w: clip(F, w, (FAR, AT, 5, 0, 1), out=AT + 12),
    lambda F, w: clip(F, w, (FAR, AT, 4, 0, 0), (AT + 64, AT + 64, 0, 1, 1), out=AT + 64),
]


@pytest.mark.parametrize("which", OVERLAPS)
def test_overlaps_are_refused(F, w, which):  # noqa: F811
    n = F.fake_launches()
    assert OVERLAPS[which](F, w) == B.GBA_E_ARG
    assert b"overlaps" in F.gba_worker_last_error(w)
    assert F.fake_launches() == n


@pytest.mark.parametrize("i", range(len(APART)))
def test_neighbours_are_taken(F, w, i):  # noqa: F811
    assert APART[i](F, w) == B.GBA_OK
