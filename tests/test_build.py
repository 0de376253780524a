"""What a build needs and when it is done again (no GPU needed; the compilers are stand-ins that write down how they were called, and so is torch, of
which a build asks little)."""
import os
import shutil
import subprocess
import sys
from pathlib import Path

import pytest
import torch

ROOT = Path(__file__).resolve().parents[1]
FAKE = """#!/bin/sh
echo "$(basename "$0") $@" >> {log}
while [ $# -gt 0 ]; do if [ "$1" = -o ]; then echo built > "$2"; fi; shift; done
"""


def torch_of(tree, version):
    """Another torch for the interpreters that run() starts."""
    (tree / "torch" / "utils").mkdir(parents=True, exist_ok=True)
    (tree / "torch" / "__init__.py").write_text(f"__version__ = '{version}'\nclass _C: _GLIBCXX_USE_CXX11_ABI = True\n")
    (tree / "torch" / "utils" / "__init__.py").write_text("")
    (tree / "torch" / "utils" / "cpp_extension.py").write_text("include_paths = library_paths = lambda: ['/nowhere']\n")


@pytest.fixture
def tree(tmp_path):
    """A copy of the package's sources and of the C header, and stand-ins for nvcc, g++ and torch."""
    torch_of(tmp_path, "1.0")
    shutil.copytree(ROOT / "paper_2412_05270_b200", tmp_path / "paper_2412_05270_b200", ignore=shutil.ignore_patterns("*.so", "_build", "__pycache__"))
    shutil.copytree(ROOT / "include", tmp_path / "include")
    for name in ("nvcc", "g++"):
        (tmp_path / name).write_text(FAKE.format(log=tmp_path / "log"))
        (tmp_path / name).chmod(0o755)
    return tmp_path


def run(tree, code):
    """What the stand-ins were called with while a new interpreter ran `code`."""
    (tree / "log").write_text("")
    env = os.environ | {"NVCC": str(tree / "nvcc"), "CXX": str(tree / "g++"), "PYTHONPATH": str(tree)}
    r = subprocess.run([sys.executable, "-c", code], cwd=tree, env=env, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    return (tree / "log").read_text().splitlines()


BUILD = "from paper_2412_05270_b200.build import *\n"


def test_the_library_is_built_without_torch(tree):
    log = run(tree, "import sys; sys.modules['torch'] = None\n" + BUILD + "build_library()")
    assert log and all(line.startswith("nvcc") for line in log)
    assert (tree / "paper_2412_05270_b200" / "libapollo.so").exists() and not list((tree / "paper_2412_05270_b200").glob("_marshal*.so"))


def test_the_extension_is_built_again_for_another_torch_and_when_forced(tree):
    package = tree / "paper_2412_05270_b200"
    log = run(tree, BUILD + "build_library()")
    assert sum(line.startswith("g++") for line in log) == 1 and len(list(package.glob("_marshal*.so"))) == 1
    assert run(tree, BUILD + "build_library()") == []
    log = run(tree, BUILD + "build_library(force=True)")
    assert sum(line.startswith("g++") for line in log) == 1 and sum(line.startswith("nvcc") for line in log) > 1
    # after an upgrade the old one is younger than every source
    torch_of(tree, "99.0")
    log = run(tree, BUILD + "build_library()")
    assert [line.split()[0] for line in log] == ["g++"]
    os.utime(package / "csrc" / "marshal.cpp", (2 ** 31 - 1, 2 ** 31 - 1))
    assert [line.split()[0] for line in run(tree, BUILD + "build_marshal()")] == ["g++"]


def test_an_extension_for_another_torch_is_not_loaded(monkeypatch):
    from paper_2412_05270_b200 import binding as B
    from paper_2412_05270_b200.build import build_library
    build_library()
    monkeypatch.setattr(B, "_marshal_module", None)
    monkeypatch.setattr(torch, "__version__", "99.0")
    with pytest.raises(ImportError, match="one torch"):
        B._marshal()
    monkeypatch.undo()
    assert B._marshal().describe(torch.zeros(3))[2] == 0
