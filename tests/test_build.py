"""What is built when: the library needs nvcc only, the operators' extension more than that."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_1806_04965_b200 import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def no(*a, **k):
    raise OSError("no compiler here")


def test_a_graph_needs_the_library_only(monkeypatch, tmp_path):
    path = str(tmp_path / "lib.so")

    def built(*a):
        shutil.copy(build.LIB, path)
        return path
    monkeypatch.setattr(binding, "_lib", None)
    monkeypatch.setattr(binding, "_LIB_PATH", path)
    monkeypatch.setattr(build, "build_library", built, raising=False)
    monkeypatch.setattr(build, "build", no)
    monkeypatch.setattr(build, "build_extension", no)
    assert binding.load_library().sr_status_str(0)


def test_without_the_extensions_tools_the_library_is_built_once(monkeypatch, tmp_path):
    monkeypatch.setattr(build, "EXTENSION", str(tmp_path / "missing.so"))
    monkeypatch.setattr(build, "build_extension", no)
    monkeypatch.setattr(subprocess, "Popen", no)                # nothing of the library is compiled again
    monkeypatch.setattr(subprocess, "check_call", no)
    os.utime(build.LIB)
    for _ in range(2):
        with pytest.warns(UserWarning, match="no compiler here"):
            assert build.build() == build.LIB


def test_an_extension_that_does_not_load_is_built_again_or_says_why(tmp_path):
    package = tmp_path / "paper_1806_04965_b200"
    shutil.copytree(build.HERE, package, ignore=shutil.ignore_patterns("_build", "__pycache__"))
    shutil.copytree(os.path.join(ROOT, "include"), tmp_path / "include")
    good, bad = tmp_path / "good.so", package / "_operators.so"
    shutil.copy(build.EXTENSION, good)
    compiler = tmp_path / "compiler"                            # stands for one that succeeds: puts the good file where it is told to
    compiler.write_text("#!/bin/sh\nwhile [ $# -gt 0 ]; do if [ $1 = -o ]; then cp %s $2; fi; shift; done\n" % good)
    compiler.chmod(0o755)
    for cxx, works in (("/bin/false", False), (str(compiler), True)):
        bad.write_bytes(b"not a library")
        out = subprocess.run([sys.executable, "-c", "import paper_1806_04965_b200 as sr; sr.quantize; print(sr.operators.__file__)"], cwd=tmp_path,
                             env=dict(os.environ, CXX=cxx, PYTHONPATH=str(tmp_path)), capture_output=True, text=True, timeout=300)
        if works:
            assert out.returncode == 0 and str(tmp_path) in out.stdout, out.stderr[-800:]
        else:
            assert out.returncode and "cannot be loaded" in out.stderr and "building it failed" in out.stderr, out.stderr[-800:]
