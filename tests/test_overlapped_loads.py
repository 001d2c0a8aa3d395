"""Kernels that are set up while the stream's previous kernel drains must not load their inputs as read-only data: the previous kernel
may still be writing them, and a load through the read-only path (``__ldg``, or a ``const __restrict__`` pointer of the kernel) may be
moved ahead of the wait for it.  Checked on the sources of every kernel that waits with follow_previous()."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parents[1] / "paper_2501_09849_b200" / "csrc"


def code(path):
    text = re.sub(r"/\*.*?\*/", "", path.read_text(), flags=re.S)
    return re.sub(r"//[^\n]*", "", text)


def with_headers(path, seen):
    if path in seen:
        return
    seen.add(path)
    for name in re.findall(r'#include "([^"]+)"', path.read_text()):
        if (CSRC / name).exists():
            with_headers(CSRC / name, seen)


FILES = sorted(p.name for p in CSRC.glob("*.cu") if "follow_previous();" in code(p))


def test_there_are_such_kernels():
    assert {"cdl_dropout.cu", "cdl_fp8_gemm.cu", "cdl_fp8_quantize.cu", "cdl_fp8_rows.cu", "cdl_vocab_loss.cu", "cdl_vocab_rows.cu"} <= set(FILES)


@pytest.mark.parametrize("name", FILES)
def test_inputs_are_not_read_only_loads(name):
    seen = set()
    with_headers(CSRC / name, seen)
    for path in seen:
        assert not re.search(r"__ldg\b|__restrict__|global\.nc", code(path)), path.name


@pytest.mark.parametrize("name", FILES)
def test_every_kernel_waits_for_the_previous_one(name):
    text = code(CSRC / name)
    # fill_bias_kernel is launched in the ordinary way
    kernels = [k for k in re.split(r"__global__", text)[1:] if "fill_bias_kernel" not in k[:200]]
    assert kernels and all("follow_previous();" in k for k in kernels)
