"""Layer norm's launches on a second device of a process, and how many blocks they take, without a
GPU: the launchers are linked with a runtime of two devices (fake_devices.cpp)."""
import ctypes
import os
import subprocess

import pytest

from paper_2205_11048_gb300 import binding as B
from paper_2205_11048_gb300 import build as BLD

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture
def F(tmp_path_factory, fake):
    """A fresh copy of the library each time: what it keeps of the runtime's answers is its own."""
    lib = str(tmp_path_factory.mktemp("devices") / "libfake.so")
    subprocess.run(["cp", fake, lib], check=True)
    L = ctypes.CDLL(lib)
    L.fake_layer_norm.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int64, ctypes.c_int32, ctypes.c_int]
    return L


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    BLD.build()
    out = tmp_path_factory.mktemp("fake_devices")
    objs, lib = [os.path.join(BLD.OUT_DIR, "gba_layernorm.o")], str(out / "libfake_devices.so")
    cc = [BLD.nvcc(), *BLD.ARCH]
    for src in ("fake_devices.cpp", "fake_devices_calls.cu"):
        objs.append(str(out / (src + ".o")))
        subprocess.run([*cc, *BLD.FLAGS, "-I" + BLD.CSRC, "-c", os.path.join(HERE, src), "-o", objs[-1]], check=True)
    subprocess.run([*cc, "-shared", "-cudart", "none", "-Xlinker", "-Bsymbolic", "-o", lib, *objs], check=True)
    return lib


@pytest.mark.parametrize("type", [B.F32, B.BF16, B.F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("grad", [0, 1])
def test_every_width_is_launched_on_every_device(F, type, grad):
    for device in (0, 1, 0):
        F.fake_device(device)
        for d in (8, 500, 1000, 2048, 4096, 5120, 5632, 6144, 6148, 8192, 8200, 12_000, 16_384, 20_000):
            for n in (1, 30, 100_000):
                for stride in (d, d + 4, d + 1):
                    assert F.fake_layer_norm(n, d, stride, type, grad) == 0, (device, d, n, stride)
    assert F.fake_refused() == 0


@pytest.mark.parametrize("type,d,stride", [
    (B.BF16, 5120, 5124), (B.BF16, 5124, 5128), (B.F16, 6144, 6148), (B.BF16, 6148, 6156), (B.F32, 5632, 5634),
    (B.F32, 5634, 5636), (B.F32, 6144, 6146), (B.F32, 6146, 6150), (B.F32, 6143, 6143)])
def test_the_grid_fills_the_sms_whatever_the_parameters_shared_memory(F, type, d, stride):
    """Parameters of 48 KB to the byte, a little less and a little more."""
    assert F.fake_layer_norm(1_000_000, d, stride, type, 0) == 0
    assert F.fake_held() >= 3
    assert F.fake_grid() == 152 * F.fake_held()
