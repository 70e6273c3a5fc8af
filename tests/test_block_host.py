"""A block's operators without a GPU: what their entry points refuse, and what they do when an
allocation fails.  The host code is linked with a fake runtime and launchers that run nothing
(see test_worker_host.py), so "device" memory is host memory here."""
import ctypes
import math
import os
import re
import subprocess

import numpy as np
import pytest
import torch

from paper_2205_11048_gb300 import binding as B
from paper_2205_11048_gb300 import build as BLD
from tests.test_chained_loads import code_of, kernels
from tests.test_worker_devices import Library, on

HERE = os.path.dirname(os.path.abspath(__file__))
MALLOC = 0


@pytest.fixture(scope="module")
def F(tmp_path_factory):
    BLD.build()
    out = tmp_path_factory.mktemp("fake_block")
    objs = [os.path.join(BLD.OUT_DIR, o) for o in ("gba_worker.o", "gba_block.o")]
    lib = str(out / "libgba_fake_block.so")
    cc = [BLD.nvcc(), *BLD.ARCH]
    for src in ("fake_runtime.cpp", "fake_worker_launchers.cu", "fake_block_launchers.cu"):
        objs.append(str(out / (src + ".o")))
        subprocess.run([*cc, *BLD.FLAGS, "-I" + BLD.CSRC, "-c", os.path.join(HERE, src), "-o", objs[-1]],
                       check=True)
    subprocess.run([*cc, "-shared", "-cudart", "none", "-Xlinker", "-Bsymbolic", "-o", lib, *objs], check=True)
    L = ctypes.CDLL(lib)
    for name, (res, args) in B._SIGNATURES.items():
        if hasattr(L, name):
            getattr(L, name).restype, getattr(L, name).argtypes = res, args
    L.fake_allocations.restype = ctypes.c_long
    return L


@pytest.fixture
def w(F):
    F.fake_fail(MALLOC, 0)
    n, bad = F.fake_allocations(), F.fake_bad()
    h = ctypes.c_void_p()
    assert F.gba_worker_create(None, ctypes.byref(h)) == B.GBA_OK
    yield h
    F.gba_worker_destroy(h)
    assert F.fake_bad() == bad, "a launcher was given memory that is not there"
    assert F.fake_allocations() == n, "allocations outlive their handle"


MEM = np.zeros(1 << 16, np.float64)  # stands for device memory, 64 places of 4 KB and more
AT = (MEM.ctypes.data + 15) // 16 * 16


def place(i):
    return AT + 4096 * i


def mat(i, rows=4, cols=8, stride=None, type=B.F32, **k):
    return B.gba_matrix(k.get("data", place(i)), rows, cols if stride is None else stride, cols, type)


def block(post=1, pre=1, gate=3, ptype=B.F32, qw=place(20), qb=None, pw=place(21), pb=None, eps=1e-6, rs=1.0, bs=1.0):
    return B.gba_block(post, pre, gate, ptype, qw, qb, pw, pb, eps, rs, bs)


def norm(F, w, b=None, x=None, r=mat(1), g=mat(2), z=mat(3), y=mat(4), stats=place(5)):
    return F.gba_residual_norm(w, b or block(), x or mat(0), r, g, z, y, stats)


def norm_grad(F, w, b=None, dy=mat(6), dz=mat(7), x=None, z=mat(3), g=mat(2), stats=place(5), dx=mat(8), dr=mat(9),
              dg=mat(10), sums=(place(11), None, place(12), None)):
    return F.gba_residual_norm_grad(w, b or block(), dy, dz, x or mat(0), z, g, stats, dx, dr, dg,
                                    sums and B.gba_block_grads(*sums))


def scan_of(decay=0, tied=1, n_seq=2, lengths=None, offsets=None):
    return B.gba_scan(decay, tied, n_seq, lengths, offsets)


def scan(F, w, s=None, x=None, f=mat(1), state=mat(2, rows=2), y=mat(3), out=mat(4, rows=2)):
    return F.gba_gated_scan(w, s or scan_of(), x or mat(0), f, state, y, out)


def scan_grad(F, w, s=None, dy=mat(5), ds=mat(6, rows=2), x=None, f=mat(1), state=mat(2, rows=2), y=mat(3),
              dx=mat(7), df=mat(8), out=mat(9, rows=2)):
    return F.gba_gated_scan_grad(w, s or scan_of(), dy, ds, x or mat(0), f, state, y, dx, df, out)


def part(w=place(0), g=place(1), m=place(2), v=place(3), ms=None, vs=None, copy=None, n=100, type=B.F32, gt=B.F32,
         ct=B.F32, bits=32, decay=0.0):
    return B.gba_adamw_part(w, g, m, v, ms, vs, copy, n, type, gt, ct, bits, decay)


def narrow(**k):
    return part(**{"bits": 8, "ms": place(4), "vs": place(5), **k})


def adamw(F, w, *p, n=None, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, now=None, norm=None, most=0.0, step=place(30),
          desc=True):
    p = p or (part(),)
    d = B.gba_adamw_desc(lr, b1, b2, eps, now, norm, most) if desc else None
    return F.gba_adamw(w, (B.gba_adamw_part * len(p))(*p), len(p) if n is None else n, d, step)


def values(F, w, p=None, m=place(6), v=place(7)):
    p = p or narrow()
    arrays = [None if o is None else (ctypes.c_void_p * 1)(o) for o in (m, v)]
    return F.gba_adamw_values(w, (B.gba_adamw_part * 1)(p), 1, *arrays)


BF = B.BF16
BAD_MATRICES = [dict(cols=0), dict(cols=(1 << 20) + 1), dict(rows=-1), dict(stride=7), dict(type=3), dict(data=None),
                dict(data=place(40) + 2), dict(rows=5), dict(cols=9, stride=16), dict(type=B.F16)]

REFUSED = (
    [lambda F, w, b=b, k=k: norm(F, w, **{k: mat(40, **b)}) for b in BAD_MATRICES for k in ("r", "g", "z", "y")]
    + [lambda F, w, b=b: norm(F, w, x=mat(40, **b)) for b in BAD_MATRICES]
    + [lambda F, w, k=k: norm(F, w, block(**k)) for k in (
        dict(post=3), dict(post=-1), dict(pre=5), dict(gate=4), dict(gate=0), dict(ptype=3), dict(qw=place(20) + 2),
        dict(pb=place(20) + 1), dict(eps=-1.0), dict(eps=math.nan), dict(rs=math.inf), dict(bs=math.nan), dict(pre=0),
        dict(qw=place(3)), dict(pw=place(5)), dict(qb=place(4) + 16))]
    + [lambda F, w, k=k: norm(F, w, **k) for k in (
        dict(g=None), dict(y=None), dict(stats=place(5) + 4), dict(z=mat(0)), dict(z=mat(2)), dict(y=mat(0)),
        dict(y=mat(1)), dict(z=mat(4)), dict(stats=place(0)), dict(stats=place(3)), dict(stats=place(4)),
        dict(z=mat(1, stride=9)), dict(z=mat(0, data=place(1) + 4)), dict(z=mat(3, type=BF)),
        dict(b=block(pre=0, pw=None), z=None, y=None), dict(b=block(pre=0, pw=None)),
        dict(x=mat(0, type=BF), g=mat(2, type=BF), y=mat(4, type=BF), r=mat(1, type=B.F16), z=mat(3, type=B.F16)))]
    + [lambda F, w, b=b, k=k: norm_grad(F, w, **{k: mat(40, **b)})
       for b in BAD_MATRICES for k in ("dy", "dz", "z", "g", "dx", "dr", "dg", "x")]
    + [lambda F, w, k=k: norm_grad(F, w, **k) for k in (
        dict(g=None), dict(dg=None), dict(dy=None), dict(z=None), dict(stats=None), dict(stats=place(5) + 8),
        dict(sums=(place(11) + 2, None, None, None)), dict(dx=mat(0)), dict(dx=mat(6)), dict(dx=mat(9)),
        dict(dr=mat(3)), dict(dg=mat(2)), dict(dg=mat(8)), dict(sums=(place(8), None, None, None)),
        dict(sums=(place(11), place(11), None, None)), dict(sums=(place(20), None, None, None)),
        dict(sums=(place(5), None, None, None)), dict(dr=mat(0, data=place(7) + 4)),
        dict(b=block(pre=0, pw=None), dy=None, z=None), dict(b=block(pre=0, pw=None), dy=None, z=None, dz=None,
                                                             sums=None))]
    + [lambda F, w, b=b, k=k: scan(F, w, **{k: mat(40, **b)}) for b in BAD_MATRICES for k in ("x", "f", "y")]
    + [lambda F, w, b=b, k=k: scan(F, w, **{k: mat(40, **{"rows": 2, **b})}) for b in BAD_MATRICES
       for k in ("state", "out")]
    + [lambda F, w, k=k: scan(F, w, scan_of(**k)) for k in (
        dict(decay=2), dict(decay=-1), dict(tied=2), dict(n_seq=-1), dict(n_seq=1 << 29), dict(n_seq=0),
        dict(n_seq=3), dict(lengths=place(50), offsets=place(51)), dict(lengths=place(50) + 4),
        dict(offsets=place(50) + 1), dict(lengths=place(3)), dict(offsets=place(4)))]
    + [lambda F, w, k=k: scan(F, w, **k) for k in (
        dict(y=mat(0)), dict(y=mat(1)), dict(y=mat(2)), dict(y=mat(4)), dict(out=mat(0, rows=2)),
        dict(out=mat(2, rows=2, stride=9)), dict(out=mat(0, rows=2, data=place(2) + 4)),
        dict(x=mat(0, type=BF), f=mat(1, type=BF), y=mat(3, type=B.F16)))]
    + [lambda F, w, b=b, k=k: scan_grad(F, w, **{k: mat(40, **b)}) for b in BAD_MATRICES
       for k in ("x", "f", "y", "dy", "dx", "df")]
    + [lambda F, w, b=b, k=k: scan_grad(F, w, **{k: mat(40, **{"rows": 2, **b})}) for b in BAD_MATRICES
       for k in ("state", "ds", "out")]
    + [lambda F, w, k=k: scan_grad(F, w, **k) for k in (
        dict(dx=mat(0)), dict(dx=mat(5)), dict(df=mat(1)), dict(df=mat(7)), dict(out=mat(2, rows=2)),
        dict(out=mat(7, rows=2)), dict(dx=mat(3)), dict(dx=mat(6)), dict(s=scan_of(n_seq=3)),
        dict(s=scan_of(offsets=place(7))))]
    + [lambda F, w, p=p: adamw(F, w, p) for p in (
        part(n=-1), part(n=(1 << 40) + 1), part(w=None), part(g=None), part(m=None), part(v=None), part(type=3),
        part(gt=-1), part(copy=place(6), ct=3), part(bits=16), part(w=place(0) + 2), part(g=place(1) + 1, gt=BF),
        part(m=place(2) + 2), part(copy=place(6) + 2), part(decay=-1.0), part(decay=math.nan), part(ms=place(4)),
        part(g=place(0)), part(m=place(0) + 16), part(v=place(2)), part(copy=place(0), ct=BF), part(w=place(30)),
        narrow(ms=None), narrow(vs=None), narrow(ms=place(4) + 2), narrow(ms=place(2)), narrow(vs=place(4)))]
    + [lambda F, w, k=k: adamw(F, w, **k) for k in (
        dict(n=-1), dict(n=(1 << 20) + 1), dict(lr=-1.0), dict(lr=math.nan), dict(lr=1e300), dict(b1=1.0),
        dict(b1=-0.1), dict(b2=1.0), dict(b2=math.nan), dict(eps=0.0), dict(eps=1e-60), dict(eps=math.inf),
        dict(norm=place(31), most=-1.0), dict(norm=place(31), most=math.nan), dict(norm=place(31) + 2),
        dict(now=place(31) + 1), dict(step=None), dict(step=place(30) + 4), dict(desc=False), dict(norm=place(2)),
        dict(now=place(0) + 8), dict(step=place(3)))]
    + [lambda F, w: F.gba_adamw(w, None, 1, B.gba_adamw_desc(1e-3, 0.9, 0.999, 1e-8, None, None, 0.0), place(30))]
    + [lambda F, w, k=k: values(F, w, **k) for k in (
        dict(m=None), dict(v=None), dict(p=narrow(m=None)), dict(p=narrow(ms=None)), dict(m=place(6) + 2),
        dict(m=place(2)), dict(v=place(5)), dict(m=place(7)), dict(p=narrow(n=-1)))]
)


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_bad_arguments_are_refused_and_nothing_is_launched(F, w, i):
    n = F.fake_block_launches()
    assert REFUSED[i](F, w) == B.GBA_E_ARG
    assert F.gba_worker_last_error(w)
    assert F.fake_block_launches() == n


def test_good_arguments_are_taken(F, w):
    n = F.fake_block_launches()
    half = {k: mat(i, type=BF) for i, k in enumerate(("x", "r", "g", "z", "y"))}
    calls = [
        lambda: norm(F, w), lambda: norm(F, w, z=mat(1)), lambda: norm(F, w, z=None, stats=None),
        lambda: norm(F, w, r=None), lambda: norm(F, w, block(gate=0), g=None),
        lambda: norm(F, w, block(pre=0, pw=None), y=None), lambda: norm(F, w, **half),
        lambda: norm(F, w, **{**half, "r": mat(1), "z": mat(1)}), lambda: norm(F, w, **{**half, "r": None, "z": mat(3)}),
        lambda: norm_grad(F, w), lambda: norm_grad(F, w, dr=mat(7)), lambda: norm_grad(F, w, dr=None, sums=None),
        lambda: norm_grad(F, w, dz=None), lambda: norm_grad(F, w, block(gate=0), g=None, dg=None),
        lambda: norm_grad(F, w, block(pre=0, pw=None), dy=None, z=None, sums=(place(11), place(12), None, None)),
        lambda: scan(F, w), lambda: scan(F, w, out=mat(2, rows=2)), lambda: scan(F, w, state=None, out=None),
        lambda: scan(F, w, scan_of(n_seq=3, offsets=place(50)), state=None, out=None),
        lambda: scan(F, w, scan_of(lengths=place(50), decay=1, tied=0)),
        lambda: scan(F, w, x=mat(0, type=BF), f=mat(1, type=BF)),
        lambda: scan_grad(F, w), lambda: scan_grad(F, w, out=mat(6, rows=2)),
        lambda: scan_grad(F, w, ds=None, state=None, out=None),
        lambda: adamw(F, w), lambda: adamw(F, w, part(), narrow(w=place(8), g=place(9), m=place(10), v=place(11))),
        lambda: adamw(F, w, part(n=0, w=None, g=None, m=None, v=None)), lambda: adamw(F, w, n=0),
        lambda: adamw(F, w, part(copy=place(6), ct=BF, decay=0.1), now=place(31), norm=place(32), most=1.0),
        lambda: values(F, w), lambda: values(F, w, part())]
    for i, call in enumerate(calls):
        assert call() == B.GBA_OK, i
    assert F.fake_block_launches() == n + len(calls)
    assert F.gba_worker_last_error(w) == b""


def test_empty_calls(F, w):
    n = F.fake_block_launches()
    e = dict(rows=0, data=None)
    assert norm(F, w, x=mat(0, **e), r=mat(0, **e), g=mat(0, **e), z=mat(0, **e), y=mat(0, **e), stats=None) == B.GBA_OK
    MEM[:] = 7.0
    assert norm_grad(F, w, **{k: mat(0, **e) for k in ("dy", "dz", "x", "z", "g", "dx", "dr", "dg")}, stats=None) == B.GBA_OK
    sums = [ctypes.cast(place(i), ctypes.POINTER(ctypes.c_float)) for i in (11, 12)]
    assert all(s[i] == 0.0 for s in sums for i in range(8)) and all(s[9] != 0.0 for s in sums)  # the high word of a 7.0
    s = scan_of(n_seq=0)
    rows = {k: mat(0, **e) for k in ("x", "f", "y", "state", "out")}
    assert scan(F, w, s, **rows) == B.GBA_OK
    assert F.fake_block_launches() == n
    # sequences of no rows pass their states on
    assert scan(F, w, scan_of(n_seq=2), **{**rows, "state": mat(2, rows=2), "out": mat(4, rows=2)}) == B.GBA_OK
    assert F.fake_block_launches() == n + 1


def test_null_handles_are_refused(F):
    for call in (norm, norm_grad, scan, scan_grad, adamw, values):
        assert call(F, None) == B.GBA_E_ARG


def test_a_workspace_that_could_not_grow(F, w):
    assert scan(F, w) == B.GBA_OK
    n = F.fake_block_launches()
    rows = 4096
    big = {k: mat(0, rows=rows, cols=1, data=AT + (1 << 20) * (i + 1)) for i, k in enumerate(("x", "f", "y"))}
    states = {k: mat(0, rows=2, cols=1, data=AT + (1 << 23) + 64 * i) for i, k in enumerate(("state", "out"))}
    F.fake_fail(MALLOC, 1)
    assert scan(F, w, **big, **states) == B.GBA_E_OOM
    assert F.gba_worker_last_error(w) and F.fake_block_launches() == n
    assert scan(F, w, **big, **states) == scan(F, w) == norm_grad(F, w) == B.GBA_OK


def test_following_kernels_read_by_ordinary_loads():
    """As test_worker_host.py has it for the other operators."""
    found = 0
    for name in ("gba_resnorm.cu", "gba_scan.cuh", "gba_scan.cu", "gba_scan_grad.cu", "gba_adamw.cu"):
        code = code_of(os.path.join(BLD.CSRC, name))
        assert "__ldg" not in code and "ld.global.nc" not in code
        for kernel, params, body in kernels(code):
            found += 1
            assert re.search(r"\bfollow\(\)", body), kernel
            assert not [p for p in params.split(",") if "const" in p and "__restrict__" in p], kernel
    assert found >= 10


# ---- the Python side ----------------------------------------------------------------------

@pytest.fixture
def worker(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 7, raising=False)
    w = object.__new__(B.Worker)
    w.torch, w.L, w.h = torch, Library(), None
    w._raw_stream, w._index, w._device = 7, 1, torch.device("cpu")
    w.L.calls = []
    return w


def calls(w, at):
    """Each operator with the tensors named in `at` on another device, the others on the worker's."""
    def t(name, *shape, dtype=torch.float32):
        return on(at.get(name, 1), *shape, dtype=dtype)

    def made():
        return B.residual_norm(post_norm="rms", pre_norm="rms", gate="silu", post_weight=t("weight", 8),
                               pre_weight=t("weight", 8))

    def seq():
        return B.sequences(2, lengths=t("lengths", 2, dtype=torch.int64))

    def parts():
        states = B.adamw_states([t("w", 8)], m=[t("m", 8)], v=[t("v", 8)], step=t("step", 1, dtype=torch.int64),
                                copies=[t("copy", 8)])
        return states.parts([t("grad", 8)])

    return {
        "residual_norm": lambda: w.residual_norm(made(), t("x", 4, 8), t("residual", 4, 8), t("gate", 4, 8),
                                                 sum_out=t("out", 4, 8)),
        "residual_norm_grad": lambda: w.residual_norm_grad(made(), t("dy", 4, 8), t("dz", 4, 8), t("x", 4, 8),
                                                           t("z", 4, 8), t("stats", 4, 4), t("gate", 4, 8)),
        "gated_scan": lambda: w.gated_scan(t("x", 4, 8), t("f", 4, 8), seq(), state=t("state", 2, 8),
                                           state_out=t("out", 2, 8)),
        "gated_scan_grad": lambda: w.gated_scan_grad(t("dy", 4, 8), t("x", 4, 8), t("f", 4, 8), t("y", 4, 8), seq(),
                                                     state=t("state", 2, 8), dstate=t("dstate", 2, 8)),
        "adamw": lambda: w.adamw(parts(), t("lr", 1), norm=t("norm", 1), max_norm=1.0),
        "adamw_values": lambda: w.adamw_values(parts(), [t("m_out", 8)], [t("v_out", 8)]),
    }


TENSORS = {"residual_norm": ["weight", "x", "residual", "gate", "out"],
           "residual_norm_grad": ["weight", "dy", "dz", "x", "z", "stats", "gate"],
           "gated_scan": ["lengths", "x", "f", "state", "out"],
           "gated_scan_grad": ["lengths", "dy", "x", "f", "y", "state", "dstate"],
           "adamw": ["w", "m", "v", "step", "copy", "grad", "lr", "norm"], "adamw_values": ["m_out", "v_out"]}


@pytest.mark.parametrize("device", [0, 2, -1])
@pytest.mark.parametrize("op,name", [(op, name) for op, names in TENSORS.items() for name in names])
def test_a_tensor_of_another_device_is_refused(worker, op, name, device):
    with pytest.raises(B.GBAError) as e:
        calls(worker, {name: device})[op]()
    assert e.value.status == B.GBA_E_ARG
    assert worker.L.calls == []


@pytest.mark.parametrize("op", list(TENSORS))
def test_tensors_of_the_workers_device_are_taken(worker, op):
    calls(worker, {})[op]()
    assert worker.L.calls == ["gba_" + op]


T = lambda *s, dtype=torch.float32: on(1, *s, dtype=dtype)  # noqa: E731
STEP = lambda: T(1, dtype=torch.int64)  # noqa: E731
BAD = {
    "norm kind": lambda w: B.residual_norm(post_norm="batch"),
    "gate kind": lambda w: B.residual_norm(gate="tanh"),
    "weights of two widths": lambda w: B.residual_norm(post_weight=T(8), post_bias=T(7)),
    "weights of two types": lambda w: B.residual_norm(post_weight=T(8), post_bias=T(8, dtype=torch.float16)),
    "weights of no norm": lambda w: B.residual_norm(pre_weight=T(8)),
    "width": lambda w: w.residual_norm(B.residual_norm(post_weight=T(7)), T(4, 8)),
    "no block": lambda w: w.residual_norm(None, T(4, 8)),
    "shapes": lambda w: w.residual_norm(B.residual_norm(), T(4, 8), T(8, 4)),
    "sum not kept": lambda w: w.residual_norm(B.residual_norm(), T(4, 8), sum_out=T(4, 8), keep_sum=False),
    "doubles": lambda w: w.residual_norm(B.residual_norm(), T(4, 8, dtype=torch.float64)),
    "stats": lambda w: w.residual_norm_grad(B.residual_norm(), None, T(4, 8), T(4, 8), None, T(4, 3)),
    "no gradient": lambda w: w.residual_norm_grad(B.residual_norm(), None, None, T(4, 8), None, T(4, 4)),
    "lengths and offsets": lambda w: B.sequences(2, T(2, dtype=torch.int64), T(3, dtype=torch.int64)),
    "lengths' type": lambda w: B.sequences(2, T(2, dtype=torch.int32)),
    "offsets' size": lambda w: B.sequences(2, offsets=T(2, dtype=torch.int64)),
    "many sequences": lambda w: B.sequences(2**29),
    "decay": lambda w: w.gated_scan(T(4, 8), T(4, 8), B.sequences(2), decay="linear"),
    "no sequences": lambda w: w.gated_scan(T(4, 8), T(4, 8), 2),
    "scan shapes": lambda w: w.gated_scan(T(4, 8), T(4, 1), B.sequences(2)),
    "states": lambda w: w.gated_scan(T(4, 8), T(4, 8), B.sequences(2), state=T(4, 8)),
    "16-bit states": lambda w: w.gated_scan(T(4, 8), T(4, 8), B.sequences(2), state=T(2, 8, dtype=torch.float16)),
    "bits": lambda w: B.adamw_states([T(8)], bits=4),
    "states' size": lambda w: B.adamw_states([T(8)], m=[T(7)], v=[T(8)]),
    "states' type": lambda w: B.adamw_states([T(8)], bits=8, m=[T(8)], m_scale=[T(1)]),
    "no scales": lambda w: B.adamw_states([T(8)], bits=8, m=[T(8, dtype=torch.uint8)]),
    "decays": lambda w: B.adamw_states([T(8)], m=[T(8)], v=[T(8)], weight_decay=[0.0, 0.1]),
    "copies' size": lambda w: B.adamw_states([T(8)], m=[T(8)], v=[T(8)], copies=[T(9)]),
    "step's type": lambda w: B.adamw_states([T(8)], m=[T(8)], v=[T(8)], step=T(1)),
    "a weight twice": lambda w: (lambda t: B.adamw_states([t, t], m=[T(8), T(8)], v=[T(8), T(8)], step=STEP()))(T(8)),
    "a weight that is a state": lambda w: (lambda t: B.adamw_states([T(8)], m=[t], v=[t], step=STEP()))(T(8)),
    "norm without bound": lambda w: w.adamw(states().parts([T(8)]), 1e-3, norm=T(1)),
    "bound without norm": lambda w: w.adamw(states().parts([T(8)]), 1e-3, max_norm=1.0),
    "lr's type": lambda w: w.adamw(states().parts([T(8)]), T(1, dtype=torch.float64)),
    "no parts": lambda w: w.adamw([T(8)], 1e-3),
    "gradients' number": lambda w: states().parts([]),
    "gradients' size": lambda w: states().parts([T(9)]),
    "values' size": lambda w: w.adamw_values(states().parts([T(8)]), [T(9)], [T(8)]),
}


def states():
    return B.adamw_states([T(8)], m=[T(8)], v=[T(8)], step=T(1, dtype=torch.int64))


@pytest.mark.parametrize("what", list(BAD))
def test_bad_tensors_are_refused(worker, what):
    with pytest.raises(B.GBAError) as e:
        BAD[what](worker)
    assert e.value.status == B.GBA_E_ARG
    assert worker.L.calls == []
