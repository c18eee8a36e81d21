"""The build: nothing is left behind by a compile that fails."""
import os
import subprocess

import pytest

from paper_2604_20368_b200 import build


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A source tree of its own in place of the package's."""
    for name, value in (("CSRC", tmp_path / "csrc"), ("LIB_DIR", tmp_path / "lib"), ("OBJ_DIR", tmp_path / "lib" / "obj"),
                        ("LIB", tmp_path / "lib" / "lib.so")):
        monkeypatch.setattr(build, name, str(value))
    (tmp_path / "csrc").mkdir()
    (tmp_path / "csrc" / "a.cu").write_text('extern "C" int a() { return 1; }\n')
    return tmp_path


def _files(tree):
    return sorted(f for _, _, files in os.walk(tree / "lib") for f in files)


def test_a_source_that_does_not_compile_leaves_nothing_behind(tree):
    (tree / "csrc" / "b.cu").write_text("this is not a program\n")
    with pytest.raises(subprocess.CalledProcessError):
        build.build()
    assert _files(tree) == []
    (tree / "csrc" / "b.cu").write_text('extern "C" int b() { return 2; }\n')
    build.build()
    assert _files(tree) == ["a.o", "b.o", "lib.so"]


def test_a_library_that_does_not_link_leaves_only_objects(tree):
    (tree / "csrc" / "b.cu").write_text('extern "C" int a() { return 2; }\n')      # defined twice
    with pytest.raises(subprocess.CalledProcessError):
        build.build()
    assert _files(tree) == ["a.o", "b.o"]


def test_marshalling_that_does_not_compile_leaves_nothing_behind(tree, monkeypatch):
    def fails(cmd):
        open(cmd[cmd.index("-o") + 1], "w").close()
        raise subprocess.CalledProcessError(1, cmd)
    (tree / "csrc" / "ln_torch.cpp").write_text("")
    monkeypatch.setattr(subprocess, "check_call", fails)
    with pytest.raises(subprocess.CalledProcessError):
        build.build_marshal()
    assert _files(tree) == []


def test_marshalling_belongs_to_one_torch_and_one_python(tree, monkeypatch):
    """A module built against another torch or Python is not taken: classes may be laid out differently."""
    import sysconfig

    import torch
    made = []

    def makes(cmd):
        made.append(cmd[cmd.index("-o") + 1])
        open(made[-1], "w").close()
    src, header = tree / "csrc" / "ln_torch.cpp", os.path.join(build.ROOT, "include", "laplace_nystrom.h")
    src.write_text("")
    for f in (src, header):
        assert os.path.exists(f)
    monkeypatch.setattr(subprocess, "check_call", makes)
    first = build.build_marshal()
    assert build.build_marshal() == first and len(made) == 1           # up to date
    monkeypatch.setattr(torch, "__version__", "9.9.9")
    second = build.build_marshal()
    assert second != first and len(made) == 2 and build.build_marshal() == second and len(made) == 2
    soabi = sysconfig.get_config_var
    monkeypatch.setattr(sysconfig, "get_config_var", lambda name: "cpython-999" if name == "SOABI" else soabi(name))
    assert build.build_marshal() not in (first, second) and len(made) == 3
