"""The library is built and used without the Python module of the attention operators,
and that module only where it was built for the running Python and torch."""
import importlib.metadata
import os
import sysconfig

import pytest

from paper_2304_07613_amd import build, nmg


@pytest.fixture
def elsewhere(tmp_path, monkeypatch):
    """A library and module of a package of its own, no compilation of the kernels."""
    lib = tmp_path / "libnmg.so"

    def library(verbose=False, jobs=None):
        lib.write_bytes(b"built")
        return str(lib)

    monkeypatch.setattr(build, "HERE", str(tmp_path))
    monkeypatch.setattr(build, "LIB_PATH", str(lib))
    monkeypatch.setattr(build, "build_library", library)
    return tmp_path


def test_library_without_a_host_compiler(elsewhere, monkeypatch):
    monkeypatch.setenv("CXX", "/bin/false")
    before = build.calls_path()
    with open(before, "wb") as f:
        f.write(b"of other sources")
    with pytest.warns(RuntimeWarning, match="calls.cpp failed"):
        assert build.build() == str(elsewhere / "libnmg.so")
    assert os.path.exists(elsewhere / "libnmg.so") and not os.path.exists(before)
    monkeypatch.setattr(nmg, "_calls", None)
    with pytest.raises(RuntimeError, match="not built"):
        nmg.rotary(None, 1, None, None)
    assert nmg._calls is None


def test_module_is_of_this_python_and_torch(elsewhere, monkeypatch):
    build.build_library()
    path = build.calls_path()
    assert path.endswith(sysconfig.get_config_var("EXT_SUFFIX"))
    with open(path, "wb") as f:
        f.write(b"built")
    for p in (path, build.LIB_PATH):
        os.utime(p, (2 ** 33, 2 ** 33))       # newer than the sources
    assert not build.is_stale()
    version = importlib.metadata.version
    monkeypatch.setattr(importlib.metadata, "version",
                        lambda name: "99.0" if name == "torch" else version(name))
    assert build.calls_path() != path and build.is_stale()
