"""The library builds whatever becomes of the host side on torch tensors, which needs more (torch, its headers, g++).  No
compiler runs here: commands are recorded and their outputs made up."""
import os
import types

import pytest

from paper_1902_01064_b200 import build


@pytest.fixture
def tree(tmp_path, monkeypatch):
    state = types.SimpleNamespace(commands=[], fails=lambda cmd: False, lib=str(tmp_path / "libhop_b200.so"), nn=str(tmp_path / "_hop_nn.so"))

    def run(cmd, **kw):
        state.commands.append(cmd)
        if state.fails(cmd):
            return types.SimpleNamespace(returncode=1, stdout="", stderr="")
        with open(cmd[cmd.index("-o") + 1], "w"):
            pass
        return types.SimpleNamespace(returncode=0, stdout="", stderr="")
    monkeypatch.setattr(build, "LIB", state.lib)
    monkeypatch.setattr(build, "NN_LIB", state.nn)
    monkeypatch.setattr(build.subprocess, "run", run)
    return state


def of_nn(cmd):
    return any(str(c).endswith(build.NN_SOURCE) for c in cmd)


def test_both_are_built(tree):
    assert build.build(force=True) == tree.lib
    assert os.path.exists(tree.lib) and os.path.exists(tree.nn) and not build.needs_build(tree.lib)


def test_the_library_is_linked_although_the_torch_side_fails(tree):
    tree.fails = of_nn
    with pytest.raises(RuntimeError, match="_hop_nn"):
        build.build(force=True)
    assert os.path.exists(tree.lib)
    assert build.needs_build(tree.lib)                   # asked again, it tries again


def test_a_torch_side_older_than_the_sources_is_built_again(tree):
    build.build(force=True)
    os.utime(tree.nn, (1, 1))
    assert build.needs_build(tree.lib)


def test_without_torch_the_library_alone_is_built(tree, monkeypatch):
    import importlib.util
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    assert build.build(force=True) == tree.lib
    assert os.path.exists(tree.lib) and not os.path.exists(tree.nn) and not any(of_nn(c) for c in tree.commands)
    assert not build.needs_build(tree.lib)


def test_a_failing_kernel_is_an_error(tree):
    tree.fails = lambda cmd: "-c" in cmd and any(str(c).endswith("hop_linear.cu") for c in cmd)
    with pytest.raises(RuntimeError, match="libhop"):
        build.build(force=True)
    assert not os.path.exists(tree.lib)
