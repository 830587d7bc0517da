"""The library is built where the Python binding of the token operators cannot be,
and is there when the binding fails.  (On a source folder of one function.)"""

import ctypes
import os
import shutil

import pytest

from paper_2307_04963_amd import build

pytestmark = pytest.mark.skipif(not (shutil.which("hipcc") or os.path.exists("/opt/rocm/bin/hipcc")), reason="needs hipcc")


@pytest.fixture
def folder(tmp_path, monkeypatch):
    (tmp_path / "csrc" / "binding").mkdir(parents=True)
    (tmp_path / "csrc" / "one.cpp").write_text('extern "C" int dycl_seven() { return 7; }\n')
    (tmp_path / "csrc" / "binding" / "tokens.cpp").write_text("#error a binding that does not compile\n")
    for name, path in (("CSRC", "csrc"), ("BUILD", "_build"), ("OUT", "libdycl.so"), ("BINDING", "_tokens.so"), ("PKG", ".")):
        monkeypatch.setattr(build, name, str(tmp_path / path))
    return tmp_path


def seven(folder):
    return ctypes.CDLL(str(folder / "libdycl.so")).dycl_seven()


def test_library_without_a_host_compiler(folder, monkeypatch, capfd):
    monkeypatch.setenv("CXX", "no-such-compiler")
    (folder / "_tokens.so").write_text("the binding of an earlier library")
    assert build.build() == str(folder / "libdycl.so") and seven(folder) == 7
    assert not (folder / "_tokens.so").exists()
    assert "no-such-compiler" in capfd.readouterr().err


def test_library_beside_a_binding_that_fails(folder):
    with pytest.raises(RuntimeError, match="does not compile"):
        build.build()
    assert seven(folder) == 7
