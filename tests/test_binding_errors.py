"""A bad argument of a compiled call raises its own exception whatever stands behind it: the conversions that follow run no Python code
while an exception is pending."""
import pytest

import paper_2501_09849_b200 as cdl
from paper_2501_09849_b200 import api, build as cdl_build


class Holder:
    def __init__(self, at=0x10000):
        self.at, self.asked = at, 0

    def data_ptr(self):
        self.asked += 1
        return self.at


class Number:
    """an integer by __index__ and a float by __float__"""

    def __init__(self, v):
        self.v, self.asked = v, 0

    def __index__(self):
        self.asked += 1
        return self.v

    def __float__(self):
        self.asked += 1
        return float(self.v)


class Stream:
    @property
    def cuda_stream(self):
        return 0


class Broken:
    def data_ptr(self):
        raise ZeroDivisionError("of the caller")


# arguments of each call that are valid and enqueue nothing (a dimension of 0), with their kinds: pointer, 64-bit, 32-bit, float, stream
CALLS = {
    "dropout": "p q p q p q i q q f u u s",
    "fp8_quantize": "p q i i i i p q p p q p s",
    "fp8_matmul": "p q p p q p i i i i p q i p p q s",
    "vocab_loss_fwd": "p q p q i p i i i p p p q s",
    "vocab_loss_bwd": "p q p q i p p p i i i p q p q p q s",
}
BAD = {"p": ("text", AttributeError), "q": ("8", TypeError), "i": (2 ** 40, OverflowError), "f": ("half", TypeError), "u": ("seed", TypeError),
       "s": (1.5, AttributeError)}


@pytest.fixture(scope="module", autouse=True)
def lib():
    cdl_build.build()
    return cdl.load_library()


def good(kind):
    return {"p": Holder, "s": Stream, "f": lambda: Number(0)}.get(kind, lambda: Number(0))()


@pytest.mark.parametrize("name", list(CALLS))
def test_first_failure_is_the_one_raised(name):
    kinds = CALLS[name].split()
    call = getattr(api._calls(), name)
    for at, kind in enumerate(kinds):
        bad, error = BAD[kind]
        args = [good(k) for k in kinds]
        args[at] = bad
        with pytest.raises(error):
            call(*args)
        if kind == "p":
            args[at] = Broken()
            with pytest.raises(ZeroDivisionError, match="of the caller"):
                call(*args)


def test_objects_that_convert_are_taken():
    args = [good(k) for k in CALLS["dropout"].split()]
    assert api._calls().dropout(*args) == 0                  # rows = cols = 0
    assert all(a.asked == 1 for a in args if isinstance(a, (Holder, Number)))


def test_two_bad_arguments_raise_once():
    with pytest.raises((AttributeError, TypeError)):
        api._calls().dropout("x", "8", Broken(), "8", Holder(), 8, cdl.CDL_F32, 0, 0, "half", 0, 0, Stream())
