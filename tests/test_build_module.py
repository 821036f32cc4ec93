"""The compiled module of the binding: when it is built, loaded and left alone.  No GPU needed."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_2511_15898_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build_library()
    assert os.path.exists(build.TENSORS)


def python(code, cwd=ROOT):
    res = subprocess.run([sys.executable, "-c", code], cwd=cwd, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-3000:]
    return res.stdout.split()


def test_importing_the_package_does_not_load_it():
    out = python("import paper_2511_15898_b200 as G, paper_2511_15898_b200.binding as B\n"
                 "print('_tensors' in open('/proc/self/maps').read(), 'libgr_b200' in open('/proc/self/maps').read())\n"
                 "G.load_library(); print(B._tensors is not None, '_tensors' in open('/proc/self/maps').read())")
    assert out == ["False", "False", "True", "True"]


def test_a_module_that_is_built_after_the_import_is_used(tmp_path):
    package = tmp_path / "paper_2511_15898_b200"
    package.mkdir()
    for name in os.listdir(build.HERE):
        if name.endswith(".py"):
            shutil.copy(os.path.join(build.HERE, name), package)
    os.symlink(build.LIB, package / "libgr_b200.so")
    out = python("import os, shutil, paper_2511_15898_b200 as G, paper_2511_15898_b200.binding as B\n"
                 f"assert B.__file__.startswith({str(tmp_path)!r})\n"
                 "print(B._tensors is None)\n"
                 f"shutil.copy({build.TENSORS!r}, {str(package)!r})\n"
                 "G.load_library(); print(B._tensors is None)", cwd=tmp_path)
    assert out == ["True", "False"]


def test_a_module_for_another_torch_is_left_alone():
    assert python("import torch, paper_2511_15898_b200 as G, paper_2511_15898_b200.binding as B\n"
                  "torch.__version__ = '1.0'; G.load_library(); print(B._tensors is None)") == ["True"]


def test_it_is_built_again_when_what_it_is_made_of_changes(tmp_path, monkeypatch):
    assert build._tensors_fresh() and not build.needs_build()
    shutil.copytree(os.path.join(ROOT, "include"), tmp_path / "include")
    with monkeypatch.context() as m:
        m.setattr(build, "ROOT", str(tmp_path))
        assert build._tensors_fresh()
        with open(tmp_path / "include" / "gr.h", "a") as f:
            f.write("\n")
        assert not build._tensors_fresh() and build.needs_build()
    with monkeypatch.context() as m:
        m.setattr("torch.__version__", "1.0")
        assert not build._tensors_fresh()
    assert build._tensors_fresh()


@pytest.mark.parametrize("compiler", ["/nowhere/g++", "false"])
def test_the_library_is_built_without_it(tmp_path, monkeypatch, capsys, compiler):
    monkeypatch.setenv("CXX", compiler)
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libgr_b200.so"))
    monkeypatch.setattr(build, "TENSORS", str(tmp_path / "_tensors.so"))
    assert os.path.exists(build.build_library()) and not os.path.exists(build.TENSORS)
    assert "could not be compiled" in capsys.readouterr().err
    # (not tried again until something changes)
    assert not build.needs_build()
