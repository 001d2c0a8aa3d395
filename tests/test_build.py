"""What the build needs: nvcc alone for the library, a C compiler and Python's headers for the compiled part of the Python binding, which is
named for its interpreter."""
import sysconfig

import pytest

import paper_2501_09849_b200 as cdl
from paper_2501_09849_b200 import api, build as cdl_build


def test_extension_is_named_for_its_interpreter():
    cdl_build.build()
    assert cdl_build.CALLS.exists() and cdl_build.CALLS.name == "_cdl_calls" + sysconfig.get_config_var("EXT_SUFFIX")
    api._calls()
    from paper_2501_09849_b200 import _cdl_calls
    assert _cdl_calls.__file__ == str(cdl_build.CALLS)


@pytest.mark.parametrize("what", ["headers", "compiler"])
def test_library_is_built_without_them(monkeypatch, tmp_path, what):
    built = []
    monkeypatch.setattr(cdl_build, "LIB", tmp_path / "libcdl.so")
    monkeypatch.setattr(cdl_build, "CALLS", tmp_path / cdl_build.CALLS.name)
    # (nvcc itself is not run here)
    monkeypatch.setattr(cdl_build, "_build_library", lambda verbose: built.append(cdl_build.LIB.write_bytes(b"")))
    if what == "headers":
        monkeypatch.setattr(cdl_build.sysconfig, "get_paths", lambda: {"include": str(tmp_path)})
    else:
        monkeypatch.setenv("CC", str(tmp_path / "no-such-compiler"))
    with pytest.warns(UserWarning, match="libcdl.so is complete"):
        assert cdl_build.build() == tmp_path / "libcdl.so"
    assert built and not cdl_build.CALLS.exists()


def test_binding_of_another_interpreter_does_not_count(monkeypatch, tmp_path):
    made = []
    (tmp_path / "_cdl_calls.cpython-399-x86_64-linux-gnu.so").write_bytes(b"")
    monkeypatch.setattr(cdl_build, "CALLS", tmp_path / cdl_build.CALLS.name)
    monkeypatch.setattr(cdl_build, "_build_calls", lambda: made.append(1))
    cdl_build.build()
    assert made


def test_calls_without_the_extension_say_what_is_missing(monkeypatch):
    import sys
    cdl_build.build()
    monkeypatch.setattr(api, "_CALLS", None)
    monkeypatch.setitem(sys.modules, "paper_2501_09849_b200._cdl_calls", None)
    monkeypatch.delattr(sys.modules["paper_2501_09849_b200"], "_cdl_calls", raising=False)
    with pytest.raises(RuntimeError, match="headers of this Python"):
        cdl.cdl_dropout(0x1000, 8, None, 0, 0x1000, 8, cdl.CDL_F32, 0, 8, 0.5, 1)
    assert cdl.cdl_version() == 100 and cdl.cdl_fp8_matmul_workspace_bytes(1, 1, 1) >= 256
