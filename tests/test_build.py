"""What building makes of a missing compiler, and what it takes for out of date (nothing is compiled here but by the build itself)."""
import os

import pytest
import torch

from paper_2601_15305_b200 import binding as gsa, build


@pytest.fixture
def away(tmp_path, monkeypatch):
    """The build's outputs in a folder of their own, the library there and up to date."""
    build.build()
    lib = tmp_path / "lib.so"
    lib.write_bytes(b"")
    monkeypatch.setattr(build, "LIB_PATH", str(lib))
    monkeypatch.setattr(build, "CALL_PATH", str(tmp_path / "call.so"))
    monkeypatch.setattr(build, "CALL_STAMP", str(tmp_path / "objects" / "stamp"))
    return tmp_path


def _extension_here(folder):
    (folder / "objects").mkdir(exist_ok=True)
    (folder / "call.so").write_bytes(b"old")
    (folder / "objects" / "stamp").write_text(build.built_for())


def test_the_library_stands_without_a_cpp_compiler(away, monkeypatch):
    made = []
    monkeypatch.setattr(build, "_build_library", lambda verbose: made.append("library"))
    for cxx in ("false", str(away / "no such compiler")):
        monkeypatch.setattr(build, "CXX", cxx)
        for force in (False, True):
            with pytest.warns(RuntimeWarning, match="extension"):
                assert build.build(force=force) == str(away / "lib.so")
    assert made == ["library", "library"]                       # (forced; otherwise it was up to date)
    assert not (away / "call.so").exists()


def test_a_failure_leaves_nothing_beside_the_outputs(away, monkeypatch):
    """Files of a compiler that fails after it has written stay among the objects, which no commit takes up."""
    fake = away / "compiler"
    fake.write_text('#!/bin/sh\nwhile [ "$1" != "-o" ]; do shift; done\ntouch "$2"\nexit 1\n')
    fake.chmod(0o755)
    monkeypatch.setattr(build, "CXX", str(fake))
    with pytest.warns(RuntimeWarning):
        build.build()
    assert {p.name for p in away.iterdir()} == {"compiler", "lib.so", "objects"} and list((away / "objects").iterdir())


def test_a_failing_library_is_an_error(away, monkeypatch):
    monkeypatch.setattr(build, "NVCC", "false")
    monkeypatch.setattr(build, "_PKG", str(away))
    with pytest.raises(RuntimeError, match="failed"):
        build.build(force=True)


@pytest.mark.parametrize("change", ["torch", "abi", "interpreter", "no stamp", "source"])
def test_an_extension_built_for_something_else_is_out_of_date(away, monkeypatch, change):
    _extension_here(away)
    assert not build._stale()
    if change == "torch":
        monkeypatch.setattr(torch, "__version__", "1.0.0")
    elif change == "abi":
        monkeypatch.setattr(torch, "compiled_with_cxx11_abi", lambda: not torch._C._GLIBCXX_USE_CXX11_ABI)
    elif change == "interpreter":
        monkeypatch.setattr(build.sysconfig, "get_config_var", lambda name: "other")
    elif change == "no stamp":
        (away / "objects" / "stamp").unlink()
    else:
        os.utime(away / "call.so", (1, 1))
    assert build._call_stale() and build._stale() and not build._library_stale()
    # what cannot be built again does not stay, to be loaded
    monkeypatch.setattr(build, "CXX", "false")
    with pytest.warns(RuntimeWarning):
        build.build()
    assert not (away / "call.so").exists() and not (away / "objects" / "stamp").exists()


def test_the_binding_refuses_an_extension_built_for_another_pytorch(monkeypatch):
    build.build()
    assert gsa._extension().built_for == build.built_for()
    monkeypatch.setattr(gsa, "_ext", None)
    monkeypatch.setattr(torch, "__version__", "1.0.0")
    with pytest.raises(gsa.GsaError, match="force"):
        gsa._extension()
