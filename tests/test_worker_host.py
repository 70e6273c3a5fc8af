"""The worker handle without a GPU: what its entry points refuse, and what they
do when an allocation fails.  The host code is linked with a fake runtime and
launchers that run nothing, so "device" memory is host memory here."""
import ctypes
import math
import os
import re
import subprocess

import numpy as np
import pytest

from paper_2205_11048_gb300 import binding as B
from paper_2205_11048_gb300 import build as BLD
from tests.test_chained_loads import code_of, kernels

HERE = os.path.dirname(os.path.abspath(__file__))
MALLOC = 0


@pytest.fixture(scope="module")
def F(tmp_path_factory):
    BLD.build()
    out = tmp_path_factory.mktemp("fake_worker")
    objs, lib = [os.path.join(BLD.OUT_DIR, "gba_worker.o")], str(out / "libgba_fake_worker.so")
    cc = [BLD.nvcc(), *BLD.ARCH]
    for src in ("fake_runtime.cpp", "fake_worker_launchers.cu"):
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


MEM = np.zeros(1 << 16, np.float64)  # stands for device memory
AT = MEM.ctypes.data


def mat(rows=4, cols=8, stride=None, type=B.F32, data=AT):
    return B.gba_matrix(data, rows, cols if stride is None else stride, cols, type)


FAR = AT + (1 << 17)


def embed(F, w, weights=None, mode=B.DIRECT, ids=AT + (1 << 18), n=3, out=None):
    return F.gba_embed(w, weights or mat(), mode, ids, n, 1.0, B.NO_PAD, out or mat(n, data=FAR))


def grad(F, w, ids=AT, n=4, g=None, rows=100, mode=B.DIRECT, ids_out=AT + 4096, rows_out=AT + 8192,
         n_out=AT + 2048):
    return F.gba_embed_grad(w, ids, n, g or mat(n, data=FAR), rows, mode, 1.0, B.NO_PAD, ids_out,
                            rows_out, n_out)


def dense(F, w, ids=AT, n=4, g=None, mode=B.DIRECT, out=None, accumulate=0):
    return F.gba_embed_grad_dense(w, ids, n, g or mat(n, data=FAR), mode, 1.0, B.NO_PAD,
                                  out or mat(10, data=AT + 4096), accumulate)


def parts(*p):
    return (B.gba_grad_part * max(1, len(p)))(*[B.gba_grad_part(*x) for x in p])


def norm(F, w, *p, n=None, out=AT):
    return F.gba_grad_norm(w, parts(*p), len(p) if n is None else n, out)


def clip(F, w, *p, n=None, out=AT, most=1.0):
    return F.gba_clip_grads(w, parts(*p), len(p) if n is None else n, most, out)


def ln(F, w, x=None, y=None, gamma=AT, beta=AT, ptype=B.F32, eps=1e-5, mean=AT, rstd=AT):
    return F.gba_layer_norm(w, x or mat(), gamma, beta, ptype, eps, y or mat(data=FAR), mean, rstd)


def ln_grad(F, w, dy=None, x=None, dx=None, gamma=AT, ptype=B.F32, mean=AT, rstd=AT, dg=AT, db=AT):
    return F.gba_layer_norm_grad(w, dy or mat(), x or mat(data=FAR), gamma, ptype, mean, rstd,
                                 dx or mat(data=FAR + 4096), dg, db)


BAD_MATRICES = [dict(cols=0), dict(cols=(1 << 20) + 1), dict(rows=-1), dict(stride=7), dict(type=3), dict(type=-1),
                dict(data=None), dict(data=AT + 2), dict(rows=1 << 62, stride=1 << 30)]

REFUSED = (
    [lambda F, w, b=b: embed(F, w, weights=mat(**b)) for b in BAD_MATRICES]
    + [lambda F, w, b=b: embed(F, w, out=mat(**{"rows": 3, "data": FAR, **b})) for b in BAD_MATRICES]
    + [lambda F, w, b=b: ln(F, w, x=mat(**b)) for b in BAD_MATRICES]
    + [lambda F, w, b=b: ln_grad(F, w, dx=mat(**{"data": FAR + 4096, **b})) for b in BAD_MATRICES]
    + [lambda F, w, k=k: embed(F, w, **k) for k in (
        dict(mode=B.HASH), dict(mode=-1), dict(weights=mat(rows=0)), dict(weights=mat(rows=2**32 - 2, cols=1)),
        dict(ids=None), dict(ids=AT + 4), dict(n=-1), dict(n=1 << 30), dict(out=mat(3, cols=9, data=FAR)),
        dict(out=mat(2, data=FAR)), dict(out=mat(3)), dict(out=mat(3, data=AT + 4 * 31)),
        dict(weights=mat(type=B.BF16), out=mat(3, type=B.F16, data=FAR)))]
    + [lambda F, w, k=k: grad(F, w, **k) for k in (
        dict(ids=None), dict(ids=AT + 1), dict(n=-1), dict(n=1 << 30), dict(g=mat(3, data=FAR)), dict(rows=0),
        dict(rows=2**32 - 2), dict(mode=B.HASH), dict(ids_out=None), dict(rows_out=None), dict(n_out=None),
        dict(n_out=AT + 4), dict(ids_out=AT + 4100), dict(rows_out=AT + 8200), dict(rows_out=FAR),
        dict(ids_out=AT + 8))]
    + [lambda F, w, k=k: dense(F, w, **k) for k in (
        dict(ids=None), dict(n=-1), dict(g=mat(5, data=FAR)), dict(mode=B.HASH), dict(accumulate=2),
        dict(out=mat(10, type=B.BF16, data=AT + 4096)), dict(out=mat(10, cols=4, data=AT + 4096)),
        dict(out=mat(10, data=FAR)), dict(out=mat(0, data=AT + 4096)), dict(out=mat(10)))]
    + [lambda F, w: norm(F, w, n=-1), lambda F, w: norm(F, w, n=(1 << 20) + 1), lambda F, w: norm(F, w, out=None),
       lambda F, w: norm(F, w, out=AT + 2), lambda F, w: F.gba_grad_norm(w, None, 1, AT)]
    + [lambda F, w, p=p: norm(F, w, p) for p in (
        (None, None, 4, 0, 0), (AT, None, -1, 0, 0), (AT, None, (1 << 40) + 1, 0, 0), (AT, None, 4, 3, 0),
        (AT + 2, None, 4, 0, 0), (AT + 1, None, 4, 1, 0))]
    + [lambda F, w, p=p: clip(F, w, p) for p in (
        (AT, None, 4, 0, 0), (AT, FAR, 4, 0, 3), (AT, AT, 4, 0, 1), (AT, AT + 8, 4, 0, 0), (AT + 8, AT, 4, 0, 0),
        (AT, FAR + 2, 4, 0, 0), (AT, AT + 12, 4, 0, 1))]
    + [lambda F, w: clip(F, w, most=-1.0), lambda F, w: clip(F, w, most=math.nan)]
    + [lambda F, w, k=k: ln(F, w, **k) for k in (
        dict(y=mat(5, data=FAR)), dict(y=mat(cols=9, data=FAR)), dict(y=mat(type=B.BF16, data=FAR)),
        dict(y=mat(data=AT + 4)), dict(y=mat(stride=9)), dict(ptype=3), dict(gamma=AT + 2), dict(beta=AT + 1),
        dict(mean=AT + 2), dict(rstd=AT + 1), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf))]
    + [lambda F, w, k=k: ln_grad(F, w, **k) for k in (
        dict(dy=mat(5)), dict(dx=mat(5, data=FAR + 4096)), dict(dx=mat(data=FAR)), dict(dx=mat(data=FAR + 4)),
        dict(dx=mat(data=AT + 4)), dict(dx=mat(stride=9)), dict(ptype=-1), dict(gamma=AT + 2), dict(mean=None), dict(rstd=None),
        dict(mean=AT + 2), dict(dg=AT + 2), dict(db=AT + 1))]
)


@pytest.mark.parametrize("i", range(len(REFUSED)))
def test_bad_arguments_are_refused_and_nothing_is_launched(F, w, i):
    n = F.fake_launches()
    assert REFUSED[i](F, w) == B.GBA_E_ARG
    assert F.gba_worker_last_error(w)
    assert F.fake_launches() == n


def test_good_arguments_are_taken(F, w):
    n = F.fake_launches()
    for call in (embed, grad, dense, norm, clip, ln, ln_grad):
        assert call(F, w) == B.GBA_OK
    assert embed(F, w, out=mat(3, type=B.F16, data=FAR), mode=B.MODULO) == B.GBA_OK
    assert clip(F, w, (AT, AT, 4, 1, 1), (FAR, FAR, 5, 0, 0), (None, None, 0, 0, 1), out=None) == B.GBA_OK
    assert ln(F, w, y=mat(), gamma=None, beta=None, mean=None, rstd=None) == B.GBA_OK
    assert ln_grad(F, w, dx=mat(), gamma=None, dg=None, db=None) == B.GBA_OK
    assert F.fake_launches() == n + 11
    assert F.gba_worker_last_error(w) == b""


def test_empty_calls_launch_nothing_and_clear_their_sums(F, w):
    n = F.fake_launches()
    MEM[:64] = 7.0
    assert embed(F, w, n=0, ids=None, out=mat(0, data=None)) == B.GBA_OK
    assert grad(F, w, n=0, ids=None, g=mat(0, data=None), ids_out=None, rows_out=None, n_out=AT) == B.GBA_OK
    assert MEM[0] == 0.0
    assert ln(F, w, x=mat(0, data=None), y=mat(0, data=None)) == B.GBA_OK
    e = mat(0, data=None)
    assert ln_grad(F, w, dy=e, x=e, dx=e, mean=None, rstd=None, dg=AT + 64, db=AT + 128) == B.GBA_OK
    assert not MEM[8:12].any() and not MEM[16:20].any() and MEM[12] == 7.0
    assert F.fake_launches() == n


def test_null_handles_are_refused(F):
    for call in (embed, grad, dense, norm, clip, ln, ln_grad):
        assert call(F, None) == B.GBA_E_ARG
    assert F.gba_worker_create(None, None) == B.GBA_E_ARG
    assert F.gba_worker_sync(None) == B.GBA_E_ARG
    assert F.gba_worker_last_error(None) == b""
    F.gba_worker_destroy(None)
    assert F.gba_embed_table(None, None, 0, None, 0, 1.0, 0, None) == B.GBA_E_ARG


def test_a_lookup_in_no_table_is_refused(F, w):
    n = F.fake_launches()
    assert F.gba_embed_table(w, None, 0, AT, 3, 1.0, 0, mat(3, data=FAR)) == B.GBA_E_ARG
    assert F.gba_worker_last_error(w)
    assert F.fake_launches() == n


def test_a_workspace_that_could_not_grow_serves_the_next_call(F, w):
    """A call that finds no memory launches nothing; the calls that follow do not run on the
    workspace that is gone."""
    assert grad(F, w) == B.GBA_OK
    n = F.fake_launches()
    big = dict(n=4000, g=mat(4000, data=FAR), ids=AT + (1 << 18), ids_out=FAR + (1 << 18), rows_out=FAR + (1 << 19))
    for _ in range(2):
        F.fake_fail(MALLOC, 1)
        assert grad(F, w, **big) == B.GBA_E_OOM
        assert F.gba_worker_last_error(w)
    assert F.fake_launches() == n
    assert norm(F, w, (AT, None, 4, 0, 0)) == B.GBA_OK
    assert grad(F, w, **big) == B.GBA_OK
    assert grad(F, w) == B.GBA_OK
    assert F.gba_worker_sync(w) == B.GBA_OK


def test_a_worker_that_finds_no_memory_is_not_made(F):
    n = F.fake_allocations()
    F.fake_fail(MALLOC, 1)
    h = ctypes.c_void_p(1)
    assert F.gba_worker_create(None, ctypes.byref(h)) == B.GBA_E_OOM
    assert not h.value
    assert F.fake_allocations() == n


def test_a_worker_without_a_gpu_fails_cleanly():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    BLD.build()
    h = ctypes.c_void_p()
    assert B.load().gba_worker_create(None, ctypes.byref(h)) == B.GBA_E_CUDA
    assert not h.value


def test_following_kernels_read_by_ordinary_loads():
    """A kernel that may be set up while its predecessor writes (its first act is follow(), but
    for clearing its own shared memory) reads nothing through the read-only path."""
    found = 0
    for name in ("gba_embed.cu", "gba_norm.cu", "gba_layernorm.cu"):
        code = code_of(os.path.join(BLD.CSRC, name))
        assert "__ldg" not in code and "ld.global.nc" not in code
        for kernel, params, body in kernels(code):
            found += 1
            assert re.search(r"\bfollow\(\)", body), kernel
            assert not [p for p in params.split(",") if "const" in p and "__restrict__" in p], kernel
    assert found >= 12
