"""The build: what the library needs and what the compiled side of the Python calls needs are kept apart."""
import os
import stat
import sys
import threading
import time

import pytest

import paper_2511_23227_amd
from paper_2511_23227_amd import binding
from paper_2511_23227_amd import build as b

pytestmark = pytest.mark.timeout(300)


@pytest.fixture
def small(tmp_path, monkeypatch):
    """The build of one source into a folder of its own."""
    monkeypatch.setattr(b, "SOURCES", {"scan.hip": []})
    for name, file in (("OBJ", "_build"), ("LIB", "libpcpp.so"), ("PROBE_LIB", "libpcpp_probe.so")):
        monkeypatch.setattr(b, name, str(tmp_path / file))
    monkeypatch.setattr(b, "CALLS_DIR", str(tmp_path))
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


def test_compiled_calls_belong_to_one_python_and_torch(monkeypatch):
    import torch
    here = b.calls_lib()
    assert sys.implementation.cache_tag in os.path.basename(here)
    monkeypatch.setattr(torch, "__version__", "99.0+other")
    other = b.calls_lib()
    assert other != here and not os.path.exists(other)
    # a module of another version is not loaded: the calls ask for their own
    asked = []
    monkeypatch.setattr(b, "build_calls", lambda: asked.append(b.calls_lib()))
    monkeypatch.setattr(binding, "_calls", None)
    with pytest.raises((ImportError, OSError)):
        binding._compiled()
    assert asked == [other]


def test_builds_at_the_same_time_take_turns(small, monkeypatch):
    inside, most = [0], [0]

    def run(cmd, **_):
        inside[0] += 1
        most[0] = max(most[0], inside[0])
        time.sleep(0.2)
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("built")
        inside[0] -= 1
        return type("Done", (), {"returncode": 0, "stderr": ""})

    monkeypatch.setattr(b.subprocess, "run", run)
    failed = []

    def build():
        try:
            b.build_calls()
        except Exception as e:                         # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=build) for _ in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed and most[0] == 1 and [p.name for p in small.glob("_torch_calls*")] and not list(small.glob("*.tmp"))


def test_the_package_has_its_compiled_calls():
    assert os.path.dirname(b.calls_lib()) == os.path.dirname(os.path.abspath(paper_2511_23227_amd.__file__))
    binding._compiled()
