"""The build: what the library needs and what the compiled side of the Python calls needs are kept apart."""
import os
import stat
import sys

import pytest

from paper_2511_23227_amd import build as b

pytestmark = pytest.mark.timeout(300)


@pytest.fixture
def small(tmp_path, monkeypatch):
    """The build of one source into a folder of its own."""
    monkeypatch.setattr(b, "SOURCES", {"scan.hip": []})
    for name, file in (("OBJ", "_build"), ("LIB", "libpcpp.so"), ("PROBE_LIB", "libpcpp_probe.so")):
        monkeypatch.setattr(b, name, str(tmp_path / file))
    monkeypatch.setattr(b, "CALLS_LIB", str(tmp_path / "_torch_calls.so"))
    return tmp_path


def test_library_is_built_without_torch(small, monkeypatch, capfd):
    monkeypatch.setitem(sys.modules, "torch", None)                                 # (an import of it fails)
    b.build()
    assert (small / "libpcpp.so").exists() and (small / "libpcpp_probe.so").exists()
    assert "torch" in capfd.readouterr().err                                        # ... and says what was left out
    with pytest.raises((ImportError, RuntimeError), match="torch"):
        b.build_calls()


def test_library_is_built_where_the_calls_do_not_compile(small, monkeypatch):
    broken = small / "bin" / "g++"
    broken.parent.mkdir()
    broken.write_text("#!/bin/sh\necho no compiler here >&2\nexit 1\n")
    broken.chmod(broken.stat().st_mode | stat.S_IXUSR)
    monkeypatch.setenv("PATH", str(broken.parent) + os.pathsep + os.environ["PATH"])
    with pytest.raises(RuntimeError, match="no compiler here"):
        b.build()
    assert (small / "libpcpp.so").exists() and (small / "libpcpp_probe.so").exists()
