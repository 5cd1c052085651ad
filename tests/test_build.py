"""What is built from what: the C library stands without the binding's extension module."""
import os

import pytest

from paper_2411_00853_amd import build


@pytest.fixture
def elsewhere(tmp_path, monkeypatch):
    """Builds into a folder of its own, of the library's smallest source."""
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libspecverify.so"))
    monkeypatch.setattr(build, "NATIVE", str(tmp_path / "_native.so"))
    monkeypatch.setattr(build, "OBJ_DIR", str(tmp_path / "obj"))
    monkeypatch.setattr(build, "SOURCES", ["lookahead.hip"])
    return tmp_path


def no_compiler():
    raise RuntimeError("no host compiler")


def test_the_library_is_built_where_the_extension_module_cannot_be(elsewhere, monkeypatch):
    monkeypatch.setattr(build, "_native_command", no_compiler)
    assert build.build_library(force=True) == build.LIB and os.path.exists(build.LIB)
    built = os.path.getmtime(build.LIB)
    assert build.build_library() == build.LIB and os.path.getmtime(build.LIB) == built      # nothing is left to do
    with pytest.raises(RuntimeError, match="host compiler"):
        build.build_native()
    assert os.path.exists(build.LIB)


def test_an_extension_module_that_does_not_compile_is_an_error(elsewhere, monkeypatch):
    monkeypatch.setattr(build, "_native_command", lambda: ["false"])
    with pytest.raises(RuntimeError, match="_native.so"):
        build.build_native(force=True)
    assert not os.path.exists(build.NATIVE)


def test_each_is_rebuilt_for_its_own_age(elsewhere):
    for path in (build.LIB, build.NATIVE):
        assert build.sources_newer_than_lib(path)
        open(path, "w").close()
        assert not build.sources_newer_than_lib(path)
        os.utime(path, (1, 1))
        assert build.sources_newer_than_lib(path)
