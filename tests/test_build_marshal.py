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


def test_what_is_built_again(monkeypatch, tmp_path):
    """The library after a change to any of its sources or to any header, the shortcuts after one to theirs."""
    folders = {}
    for name in ("csrc", "include"):
        folders[name] = tmp_path / name
        folders[name].mkdir()
    made = [tmp_path / "lib.so", tmp_path / "marshal.so"]
    parts = [folders["csrc"] / x for x in ("api.cpp", "cache.h", "marshal.cpp", "kv4_chunk.hip")]
    parts += [folders["include"] / x for x in ("mocap_attn.h", "mocap_cache.h", "mocap_serve.h")]
    for x in (*made, *parts):
        x.write_text("")
    for name, value in (("CSRC", folders["csrc"]), ("INCLUDE", folders["include"]), ("LIB", made[0]), ("MARSHAL", made[1])):
        monkeypatch.setattr(build, name, str(value))
    lib, marshal = (str(x) for x in made)

    def stale(changed):
        for x in (*made, *parts):
            os.utime(x, (2000, 2000) if x in made else (3000, 3000) if x.name == changed else (1000, 1000))
        return build.stale()

    assert stale(None) == []
    for changed, want in (("api.cpp", [lib]), ("cache.h", [lib]), ("kv4_chunk.hip", [lib]), ("marshal.cpp", [marshal]),
                          ("mocap_attn.h", [lib, marshal]), ("mocap_cache.h", [lib, marshal]), ("mocap_serve.h", [lib, marshal])):
        assert stale(changed) == want, changed
    os.remove(made[1])
    assert build.stale() == [lib, marshal]


def test_shortcuts_for_another_torch_or_python_are_not_used(mocap_lib, monkeypatch):
    """The extension's name has this Python's tag, and one that was built for another torch is refused with a warning."""
    import importlib.util
    import sys
    import sysconfig
    import types

    import torch

    import paper_2606_22968_amd as package
    assert os.path.basename(build.MARSHAL) == "_marshal" + sysconfig.get_config_var("EXT_SUFFIX")
    if mocap_lib._marshal is not None:
        assert os.path.realpath(mocap_lib._marshal.__file__) == os.path.realpath(build.MARSHAL)

    def load():
        spec = importlib.util.spec_from_file_location("paper_2606_22968_amd.binding_again", mocap_lib.__file__)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        return module

    def no_address(*args):
        return None

    for version, used in ((torch.__version__, True), ("1.0", False), (None, False)):
        fake = types.SimpleNamespace(address=no_address, rows=no_address, __file__="_marshal.so")
        if version is not None:
            fake.torch_version = version
        monkeypatch.setattr(package, "_marshal", fake, raising=False)
        monkeypatch.setitem(sys.modules, "paper_2606_22968_amd._marshal", fake)
        if used:
            assert load()._address is no_address
        else:
            with pytest.warns(UserWarning, match="another torch"):
                again = load()
            assert again._marshal is None and again._address is not no_address
