"""The compiled marshalling module: the library loads without it, and one that does not fit is noticed (CPU only)."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_2607_16184_b200 import binding as B
from paper_2607_16184_b200 import build as pwbuild

PACKAGE = os.path.dirname(os.path.abspath(B.__file__))
USE = "from pkg import binding as B\nassert B.pw_page_bytes(128, 128, 4)[0] > 0\n"
CALL = USE + "try:\n    B._load_pwtorch()\nexcept RuntimeError as e:\n    print(e)\nelse:\n    print('loaded')\n"


@pytest.fixture
def package(tmp_path):
    """A copy of the package's Python files with its libraries."""
    pwbuild.build()
    to = tmp_path / "pkg"
    shutil.copytree(PACKAGE, to, ignore=shutil.ignore_patterns("csrc", "__pycache__", "*.o"))
    return to


def run(package, code):
    r = subprocess.run([sys.executable, "-c", code], cwd=package.parent, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return r.stdout.strip()


def other_torch(path):
    data, stamp = path.read_bytes(), pwbuild.module_stamp().encode()
    assert stamp in data
    path.write_bytes(data.replace(stamp, stamp.replace(b"torch ", b"torch_", 1)))


def test_module_loads_beside_the_library(package):
    assert run(package, CALL) == "loaded"


def test_library_loads_without_the_module(package):
    (package / "_pwtorch.so").unlink()
    run(package, USE)
    assert "python -m paper_2607_16184_b200.build" in run(package, CALL)


def test_module_that_does_not_load_is_named(package):
    (package / "_pwtorch.so").write_bytes(b"not a library")
    run(package, USE)
    assert "_pwtorch.so" in run(package, CALL) and "paper_2607_16184_b200.build" in run(package, CALL)


def test_module_of_another_torch_is_refused(package):
    other_torch(package / "_pwtorch.so")
    assert "was built for torch_" in run(package, CALL)


def test_module_of_another_torch_is_built_again(tmp_path, monkeypatch):
    pwbuild.build()
    assert pwbuild.module_is_current()
    copy = tmp_path / "_pwtorch.so"
    shutil.copy2(pwbuild.MODULE, copy)
    monkeypatch.setattr(pwbuild, "MODULE", str(copy))
    assert pwbuild.module_is_current()
    other_torch(copy)
    os.utime(copy)                                   # newer than the sources all the same
    commands = []
    monkeypatch.setattr(pwbuild.subprocess, "check_call", commands.append)
    pwbuild.build_module()
    assert len(commands) == 1 and str(copy) in commands[0] and "-w" not in commands[0]
