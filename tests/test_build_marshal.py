"""How the binding's shortcuts (csrc/marshal.cpp) are built beside the library, and left out where they cannot be."""
import os

import pytest

from paper_2606_22968_amd import build


@pytest.fixture
def elsewhere(monkeypatch, tmp_path):
    """A library of one host source, and its shortcuts, in a folder of their own."""
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    monkeypatch.setattr(build, "SOURCES", ["plan.cpp"])
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build, "MARSHAL", str(tmp_path / "marshal.so"))
    return lambda: build.build(lib_path=build.LIB, build_dir=str(tmp_path / "objects"))


@pytest.mark.parametrize("compiler", ["/bin/false", "/nowhere/g++"])
def test_a_library_without_the_shortcuts(elsewhere, monkeypatch, capsys, compiler):
    """Where they cannot be compiled, the library is built all the same, with a warning, and old ones do not stay."""
    monkeypatch.setenv("CXX", compiler)
    with open(build.MARSHAL, "w") as f:
        f.write("old")
    with pytest.warns(UserWarning, match="shortcuts were not built"):
        assert elsewhere() == build.LIB
    assert os.path.exists(build.LIB) and not os.path.exists(build.MARSHAL)
