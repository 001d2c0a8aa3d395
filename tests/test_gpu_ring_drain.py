"""A warp that leaves its ring of bulk copies after an abandoned wait stays until the copies still under way have landed, although the
flag that ends the other waits is set, and no longer than a limit where one never lands.  A small kernel built only by this test
plays the late copy; nothing is made to fail."""
import ctypes
import subprocess
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parents[1]


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    out = tmp_path_factory.mktemp("ring_probe") / "libring_probe.so"
    subprocess.run(["/usr/local/cuda/bin/nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-O2", "-std=c++17", "-Xcompiler", "-fPIC", "-shared",
                    "-cudart", "shared", "-I", str(ROOT / "include"), "-I", str(ROOT / "paper_2501_09849_b200" / "csrc"), "-o", str(out),
                    str(ROOT / "tests" / "cuda" / "ring_probe.cu")], check=True)
    lib = ctypes.CDLL(str(out))
    lib.ring_probe.argtypes = [ctypes.c_ulonglong, ctypes.c_void_p, ctypes.c_void_p]
    lib.ring_probe.restype = ctypes.c_int
    return lib


@pytest.mark.parametrize("late_ms", [0, 1, 5])
def test_drain_waits_for_a_late_copy(probe, late_ms):
    import torch
    out = torch.zeros(2, dtype=torch.int64, device="cuda")
    assert probe.ring_probe(late_ms * 1_000_000, out.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    landed, took = out.tolist()
    if late_ms:
        assert landed == 1 and late_ms * 900_000 <= took < 9_000_000
    else:                                   # never: given up after 10 ms
        assert landed == 0 and 9_000_000 <= took < 100_000_000
