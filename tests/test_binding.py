"""The compiled argument marshalling of the language-model calls: what it takes for a pointer and a stream, and what it refuses
before the library is entered."""
import pytest

import paper_2501_09849_b200 as cdl
from paper_2501_09849_b200 import api, build as cdl_build


class Holder:
    def __init__(self, at):
        self.at = at

    def data_ptr(self):
        return self.at


class Stream:
    cuda_stream = 0


@pytest.fixture(scope="module", autouse=True)
def lib():
    cdl_build.build()
    return cdl.load_library()


def dropout(x=0x1000, ldx=8, y=0x1000, rows=0, p=0.5, seed=1, stream=0, check=False, type=cdl.CDL_F32):
    return cdl.cdl_dropout(x, ldx, None, 0, y, 8, type, rows, 8, p, seed, stream=stream, check=check)


def test_pointers_and_streams():
    for x in (None, 0x1000, Holder(0x1000)):
        assert dropout(x=x) == 0
    assert dropout(x=Holder(0x1002), rows=2) == -2           # the address arrived: it is misaligned
    assert dropout(x=Holder(2 ** 63 + 1), rows=2) == -2      # all 64 bits of it
    for stream in (None, 0, Stream()):
        assert dropout(stream=stream) == 0
    assert dropout(seed=2 ** 64 - 1) == 0


def test_wrong_arguments_raise():
    with pytest.raises(AttributeError):
        dropout(x="tensor")
    with pytest.raises(AttributeError):
        dropout(stream=1.5)
    with pytest.raises(TypeError):
        dropout(ldx="8")
    with pytest.raises(TypeError):
        dropout(p="half")
    with pytest.raises(OverflowError):
        dropout(type=2 ** 40)
    with pytest.raises(TypeError):
        api._calls().dropout(1, 2, 3)
    with pytest.raises(cdl.CdlError, match="out of range"):
        dropout(p=2.0, check=True)
