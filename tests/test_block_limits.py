"""How much shared memory the kernels of a block's norms and scans may ask for, without a GPU: the
limit belongs to a kernel on a device, not to a call, and workers of several threads share it.  The
launchers are linked with a runtime that keeps such limits (fake_limits.cpp)."""
import ctypes
import itertools
import os
import subprocess

import pytest

from paper_2205_11048_gb300 import binding as B
from paper_2205_11048_gb300 import build as BLD

HERE = os.path.dirname(os.path.abspath(__file__))
CALL = ctypes.CFUNCTYPE(None)


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    BLD.build()
    out = tmp_path_factory.mktemp("fake_limits")
    objs = [os.path.join(BLD.OUT_DIR, o) for o in ("gba_resnorm.o", "gba_scan.o", "gba_scan_grad.o")]
    lib = str(out / "libfake_limits.so")
    cc = [BLD.nvcc(), *BLD.ARCH]
    for src in ("fake_limits.cpp", "fake_limits_calls.cu"):
        objs.append(str(out / (src + ".o")))
        subprocess.run([*cc, *BLD.FLAGS, "-I" + BLD.CSRC, "-c", os.path.join(HERE, src), "-o", objs[-1]], check=True)
    subprocess.run([*cc, "-shared", "-cudart", "none", "-Xlinker", "-Bsymbolic", "-o", lib, *objs], check=True)
    return lib


@pytest.fixture
def F(tmp_path_factory, fake):
    """A fresh copy of the library each time: its limits are its own."""
    lib = str(tmp_path_factory.mktemp("limits") / "libfake.so")
    subprocess.run(["cp", fake, lib], check=True)
    L = ctypes.CDLL(lib)
    i64, i32 = ctypes.c_int64, ctypes.c_int32
    L.fake_norm.argtypes = [i64, i32, i64, i32, i32, ctypes.c_int, ctypes.c_int]
    L.fake_scan.argtypes = [i64, i64, i32, i64, i32, i32, ctypes.c_int, ctypes.c_int]
    L.fake_meanwhile.argtypes = [CALL]
    L.fake_most.restype = ctypes.c_size_t
    return L


WIDTHS = [1, 8, 40, 64, 256, 257, 300, 1001, 1024, 2048, 4096, 5120, 8000, 8192, 8200, 12_000, 14_336, 16_384, 20_000]
PAIRS = [(B.F32, B.F32), (B.BF16, B.BF16), (B.BF16, B.F32), (B.F16, B.F16), (B.F16, B.F32)]


@pytest.mark.parametrize("grad", [0, 1])
@pytest.mark.parametrize("type,wide", PAIRS)
def test_a_kernel_of_the_norms_has_one_limit(F, type, wide, grad):
    for n, d, off, biases in itertools.product((1, 30, 100_000), WIDTHS, (0, 8, 1), (0, 1)):
        assert F.fake_norm(n, d, d + off, type, wide, grad, biases) == 0, (n, d, off, biases)
    assert F.fake_refused() == F.fake_changed() == 0
    assert F.fake_most() > 48 * 1024


@pytest.mark.parametrize("grad", [0, 1])
@pytest.mark.parametrize("type,out", PAIRS)
def test_a_kernel_of_the_scan_has_one_limit(F, type, out, grad):
    for n_seq, each, d, off, ragged in itertools.product((1, 2, 30, 152, 300, 3000), (1, 70, 3000), (1, 64, 132, 512, 2048),
                                                         (0, 8, 1), (0, 1)):
        assert F.fake_scan(n_seq, n_seq * each, d, d + off, type, out, ragged, grad) == 0, (n_seq, each, d, off, ragged)
    assert F.fake_refused() == F.fake_changed() == 0
    assert F.fake_most() > (48 if grad or type == B.F32 else 32) * 1024


@pytest.mark.parametrize("mine,theirs", [
    (lambda F: F.fake_norm(1000, 8192, 8192, B.F32, B.F32, 0, 0), lambda F: F.fake_norm(1000, 4000, 4000, B.F32, B.F32, 0, 0)),
    (lambda F: F.fake_norm(1000, 8192, 8192, B.BF16, B.BF16, 1, 0), lambda F: F.fake_norm(1000, 4104, 4104, B.BF16, B.BF16, 1, 0)),
    (lambda F: F.fake_norm(1000, 4001, 4001, B.BF16, B.BF16, 1, 0), lambda F: F.fake_norm(1000, 3001, 3001, B.BF16, B.BF16, 1, 0)),
    (lambda F: F.fake_scan(304, 304 * 300, 128, 128, B.BF16, B.BF16, 0, 1),
     lambda F: F.fake_scan(3000, 3000 * 70, 2048, 2048, B.BF16, B.BF16, 0, 1)),
], ids=["norm", "norm gradient", "norm gradient, odd", "scan gradient"])
def test_another_threads_call_between_a_limit_and_its_launch(F, mine, theirs):
    """A call that needs much shared memory, and another thread's of the same kernel, which needs
    less, after the first has asked for its limit and before it launches."""
    others = []
    call = CALL(lambda: others.append(theirs(F)))
    F.fake_meanwhile(call)
    assert mine(F) == 0
    assert others and not any(others) and F.fake_refused() == 0
