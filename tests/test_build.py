"""What is built when torch, or the compiler of its binding, is missing or another one: on copies, with stand-ins for the compilers."""
import os
import stat

import pytest


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """build.py over an empty copy: nvcc and g++ write their output's name into it; `torch` is a folder with a version."""
    from paper_2509_22418_b200 import build
    here = tmp_path / "pkg"
    (here / "csrc").mkdir(parents=True)
    (tmp_path / "include").mkdir()
    (tmp_path / "include" / "ppu.h").write_text("")
    for src in build.SOURCES:
        (here / "csrc" / src).write_text("")
    (here / "csrc" / "bind.cpp").write_text("")
    tools = tmp_path / "bin"
    tools.mkdir()

    def tool(name, status=0):
        path = tools / name
        path.write_text(f'#!/bin/sh\necho {name} "$@" >> {tmp_path}/log\n'
                        f'[ {status} = 0 ] || exit {status}\nwhile [ $# -gt 1 ]; do [ "$1" = -o ] && echo built > "$2"; shift; done\n')
        path.chmod(path.stat().st_mode | stat.S_IXUSR)
        return str(path)

    torch = tmp_path / "site" / "torch"
    (torch / "lib").mkdir(parents=True)
    (torch / "lib" / "libtorch_cuda.so").write_text("")
    (torch / "__init__.py").write_text("")
    (torch / "version.py").write_text("__version__ = '2.0'\n")
    monkeypatch.setenv("NVCC", tool("nvcc"))
    tool("g++")
    monkeypatch.setenv("PATH", str(tools) + os.pathsep + os.environ["PATH"])
    for name, path in (("HERE", here), ("CSRC", here / "csrc"), ("LIB", here / "libppu.so"), ("OPS", here / "_ops.so"), ("OPS_OBJ", here / "_build" / "bind.o")):
        monkeypatch.setattr(build, name, str(path))

    class Spec:
        origin = str(torch / "__init__.py")
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: Spec)
    build.tool, build.torch_dir, build.runs = tool, torch, lambda: (tmp_path / "log").read_text().count("\n") if (tmp_path / "log").exists() else 0
    yield build
    del build.tool, build.torch_dir, build.runs


@pytest.mark.parametrize("which", ["none", "for CPUs"])
def test_library_without_torch(tree, monkeypatch, which):
    if which == "none":
        monkeypatch.setattr(tree.importlib.util, "find_spec", lambda name: None)
    else:
        (tree.torch_dir / "lib" / "libtorch_cuda.so").unlink()
    tree.build()
    assert os.path.exists(tree.LIB) and not os.path.exists(tree.OPS)
    n = tree.runs()
    tree.build()                           # nothing is stale
    assert tree.runs() == n


def test_library_where_the_binding_does_not_compile(tree):
    tree.tool("g++", status=1)
    with pytest.raises(RuntimeError, match="bind.cpp"):
        tree.build()
    assert os.path.exists(tree.LIB) and not os.path.exists(tree.OPS)


def test_library_that_does_not_compile(tree):
    tree.tool("nvcc", status=1)
    with pytest.raises(RuntimeError):
        tree.build()
    assert not os.path.exists(tree.LIB) and not os.path.exists(tree.OPS)


def test_built_once(tree):
    tree.build()
    assert os.path.exists(tree.LIB) and os.path.exists(tree.OPS)
    n = tree.runs()
    tree.build()
    assert tree.runs() == n


def test_built_again_for_another_torch(tree):
    tree.build()
    n = tree.runs()
    (tree.torch_dir / "version.py").write_text("__version__ = '2.1'\n")
    tree.build()
    assert tree.runs() > n
    n = tree.runs()
    tree.build()
    assert tree.runs() == n


def test_library_without_a_compiler_for_the_binding(tree, monkeypatch):
    tools = os.path.dirname(os.environ["NVCC"])
    os.remove(os.path.join(tools, "g++"))
    monkeypatch.setenv("PATH", tools)
    with pytest.raises(RuntimeError, match="bind.cpp"):
        tree.build()
    assert os.path.exists(tree.LIB) and not os.path.exists(tree.OPS)
