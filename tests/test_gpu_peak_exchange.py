"""Two epilogue warps that share a checkpoint's groups exchange their rows' peaks.  Where one of them gives up before it gets there, the other returns as
well, whether it is already waiting or comes later.  A small kernel built only by this test calls the exchange itself."""
import ctypes
import subprocess
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parents[1]
MS = 1_000_000


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    out = tmp_path_factory.mktemp("peak_probe") / "libpeak_probe.so"
    subprocess.run(["/usr/local/cuda/bin/nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-O2", "-std=c++17", "-Xcompiler", "-fPIC", "-shared", "-cudart", "shared",
                    "-I", str(ROOT / "include"), "-I", str(ROOT / "paper_2501_09849_b200" / "csrc"), "-o", str(out), str(ROOT / "tests" / "cuda" / "peak_probe.cu")], check=True)
    lib = ctypes.CDLL(str(out))
    lib.peak_probe.argtypes = [ctypes.c_int] * 4 + [ctypes.c_ulonglong] * 2 + [ctypes.c_void_p] * 3
    lib.peak_probe.restype = ctypes.c_int

    def call(rounds, quitter=-1, quit=0, flag=0, late=0, limit=MS):
        import torch
        out = torch.zeros(4, dtype=torch.int32, device="cuda")
        assert lib.peak_probe(rounds, quitter, quit, flag, late, limit, out.data_ptr(), out.data_ptr() + 8, torch.cuda.current_stream().cuda_stream) == 0
        met = out.tolist()
        assert met[2:] == [0, 0]
        return met[:2]
    return call


def test_both_get_the_larger_number(probe):
    assert probe(1000, limit=50 * MS) == [1000, 1000]


@pytest.mark.parametrize("quitter", [0, 1])
@pytest.mark.parametrize("quit", [0, 1, 2, 5])
@pytest.mark.parametrize("flag", [0, 1])
@pytest.mark.parametrize("late", [0, 3 * MS])
def test_a_warp_that_gives_up_does_not_keep_the_other(probe, quitter, quit, flag, late):
    """The partner's exchanges before that one count, that one and those behind it do not; the limit of 50 ms is not needed where the flag is set."""
    met = probe(8, quitter, quit, flag, late, limit=50 * MS if flag else MS if late == 0 else 5 * MS)
    assert met[quitter] == quit and met[1 - quitter] == quit
