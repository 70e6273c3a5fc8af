"""A worker's calls work on its device and leave the caller's current one as it was.  Without a
GPU (see test_worker_host.py)."""
import ctypes
import os
import subprocess

import pytest

from paper_2205_11048_gb300 import binding as B
from paper_2205_11048_gb300 import build as BLD
from tests.test_worker_host import AT, FAR, clip, dense, embed, grad, ln, ln_grad, mat, norm

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def F(tmp_path_factory):
    BLD.build()
    out = tmp_path_factory.mktemp("fake_current")
    objs, lib = [os.path.join(BLD.OUT_DIR, "gba_worker.o")], str(out / "libgba_fake_current.so")
    cc = [BLD.nvcc(), *BLD.ARCH]
    for src in ("fake_runtime.cpp", "fake_worker_launchers.cu", "fake_current_device.cpp"):
        objs.append(str(out / (src + ".o")))
        subprocess.run([*cc, *BLD.FLAGS, "-I" + BLD.CSRC, "-c", os.path.join(HERE, src), "-o", objs[-1]], check=True)
    wrap = [x for f in ("SetDevice", "GetDevice", "StreamSynchronize", "MemsetAsync", "Malloc")
            for x in ("-Xlinker", "--wrap=cuda" + f)]
    subprocess.run([*cc, "-shared", "-cudart", "none", "-Xlinker", "-Bsymbolic", *wrap, "-o", lib, *objs], check=True)
    L = ctypes.CDLL(lib)
    for name, (res, args) in B._SIGNATURES.items():
        if hasattr(L, name):
            getattr(L, name).restype, getattr(L, name).argtypes = res, args
    return L


E0 = dict(rows=0, data=None)
CALLS = [embed, grad, dense, norm, clip, ln, ln_grad,
         lambda F, w: grad(F, w, n=4000, g=mat(4000, data=FAR), ids=AT + (1 << 18), ids_out=FAR + (1 << 18),
                           rows_out=FAR + (1 << 19)),
         lambda F, w: grad(F, w, n=0, ids=None, g=mat(**E0), ids_out=None, rows_out=None, n_out=AT),
         lambda F, w: ln_grad(F, w, dy=mat(**E0), x=mat(**E0), dx=mat(**E0), dg=AT + 64, db=AT + 128),
         lambda F, w: F.gba_worker_sync(w)]


@pytest.mark.parametrize("of,current", [(0, 0), (0, 1), (1, 0), (2, 1)])
def test_calls_leave_the_current_device(F, of, current):
    F.fake_make_current(of)
    w = ctypes.c_void_p()
    assert F.gba_worker_create(None, ctypes.byref(w)) == B.GBA_OK
    for call in CALLS:
        F.fake_make_current(current)
        assert call(F, w) == B.GBA_OK
        assert F.fake_current() == current
    assert F.fake_worked_on() == of
    assert F.gba_embed_table(w, None, 0, AT, 3, 1.0, 0, mat(3, data=FAR)) == B.GBA_E_ARG
    assert F.gba_embed(w, mat(cols=0), B.DIRECT, AT, 3, 1.0, 0, mat(3, data=FAR)) == B.GBA_E_ARG
    assert F.fake_current() == current
    F.gba_worker_destroy(w)
    assert F.fake_current() == current and F.fake_worked_on() == of
