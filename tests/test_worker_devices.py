"""Tensors of another GPU than the worker's are refused before the library sees their
addresses.  Without a GPU: the tensors are stand-ins that say where they are."""
import pytest
import torch

from paper_2205_11048_gb300 import binding as B


class Stand:
    """A tensor in host memory that says it is on GPU `device` (-1: on the host)."""

    def __init__(self, tensor, device):
        self._tensor, self._device = tensor, device

    is_cuda = property(lambda self: self._device >= 0)
    device = property(lambda self: torch.device("cuda", self._device) if self._device >= 0 else torch.device("cpu"))

    def get_device(self):
        return self._device

    def contiguous(self):
        return self

    def __getattr__(self, name):
        return getattr(self._tensor, name)


class Library:
    def __getattr__(self, name):
        def call(*args):
            self.__dict__.setdefault("calls", []).append(name)
            return B.GBA_OK
        return call


@pytest.fixture
def w(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 7, raising=False)
    w = object.__new__(B.Worker)
    w.torch, w.L, w.h = torch, Library(), None
    w._raw_stream, w._index, w._device = 7, 1, torch.device("cpu")
    w.L.calls = []
    return w


def on(device, *shape, dtype=torch.float32):
    return Stand(torch.zeros(shape, dtype=dtype), device)


def calls(w, at):
    """Each operator with the tensors named in `at` on another device, the others on the worker's."""
    def t(name, *shape, dtype=torch.float32):
        return on(at.get(name, 1), *shape, dtype=dtype)

    ids = t("ids", 3, dtype=torch.int64)

    class Server:
        dims, h = [8], None

    return {
        "embed": lambda: w.embed(t("weights", 5, 8), ids, out=t("out", 3, 8)),
        "embed_table": lambda: w.embed_table(Server, 0, ids, out=t("out", 3, 8)),
        "embed_grad": lambda: w.embed_grad(ids, t("grad", 3, 8), 5),
        "embed_grad_dense": lambda: w.embed_grad_dense(ids, t("grad", 3, 8), t("out", 5, 8)),
        "grad_norm": lambda: w.grad_norm([t("grad", 8), t("other", 3)]),
        "clip_grads": lambda: w.clip_grads(B.grad_parts([t("grad", 8), t("other", 3)], [t("out", 8), t("other", 3)]), 1.0),
        "layer_norm": lambda: w.layer_norm(t("x", 3, 8), t("gamma", 8), t("beta", 8)),
        "layer_norm_grad": lambda: w.layer_norm_grad(t("dy", 3, 8), t("x", 3, 8), t("gamma", 8), t("mean", 3), t("rstd", 3)),
    }


TENSORS = {"embed": ["weights", "ids", "out"], "embed_table": ["ids", "out"], "embed_grad": ["ids", "grad"],
           "embed_grad_dense": ["ids", "grad", "out"], "grad_norm": ["grad", "other"], "clip_grads": ["grad", "other", "out"],
           "layer_norm": ["x", "gamma", "beta"], "layer_norm_grad": ["dy", "x", "gamma", "mean", "rstd"]}


@pytest.mark.parametrize("device", [0, 2, -1])
@pytest.mark.parametrize("op,name", [(op, name) for op, names in TENSORS.items() for name in names])
def test_a_tensor_of_another_device_is_refused(w, op, name, device):
    with pytest.raises(B.GBAError) as e:
        calls(w, {name: device})[op]()
    assert e.value.status == B.GBA_E_ARG
    assert w.L.calls == []


@pytest.mark.parametrize("op", TENSORS)
def test_tensors_of_the_workers_device_are_taken(w, op):
    calls(w, {})[op]()
    assert w.L.calls == ["gba_" + op]


@pytest.mark.parametrize("device", [0, 2])
def test_parts_made_for_another_device_are_refused(w, device):
    parts = B.grad_parts([on(device, 8)])
    for call in (lambda: w.grad_norm(parts), lambda: w.clip_grads(parts, 1.0)):
        with pytest.raises(B.GBAError) as e:
            call()
        assert e.value.status == B.GBA_E_ARG
    assert w.L.calls == []
    w.grad_norm(B.grad_parts([]))
    assert w.L.calls == ["gba_grad_norm"]


def test_a_worker_is_made_on_its_streams_device(monkeypatch):
    made = []

    class Current:  # stands for torch.cuda.device
        now = 0

        def __init__(self, device):
            self.device = torch.device(device).index

        def __enter__(self):
            self.before, Current.now = Current.now, self.device

        def __exit__(self, *_):
            Current.now = self.before

    class Stream:
        cuda_stream, device = 5, torch.device("cuda", 1)

    class Maker:
        def gba_worker_create(self, stream, out):
            made.append((stream, Current.now))
            return B.GBA_OK

        def gba_worker_destroy(self, h):
            pass

    monkeypatch.setattr(B, "load", Maker)
    monkeypatch.setattr(torch.cuda, "device", Current)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: Current.now)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream)
    for stream in (Stream, None):
        w = B.Worker(stream)
        assert made.pop() == (5, 1) and Current.now == 0
        with pytest.raises(B.GBAError):
            w._mine(on(0, 3))
        w._mine(on(1, 3))
