"""What a build needs: the C library nvcc alone, the binding for torch tensors the torch that it is built against."""
import importlib.util
import os
import types

import pytest

from paper_2505_03983_b200 import build as b


@pytest.fixture
def runs(monkeypatch, tmp_path):
    """The commands that building the binding runs, which make an empty file."""
    b.build()  # the tree's own, before anything is replaced
    monkeypatch.setattr(b, "TORCH_LIB", str(tmp_path / "_asd_torch.so"))
    commands = []

    def run(cmd, **_):
        commands.append(cmd)
        open(b.TORCH_LIB, "w").close()
        return types.SimpleNamespace(returncode=0, stdout="", stderr="")

    monkeypatch.setattr(b.subprocess, "run", run)
    return commands


def test_the_c_library_is_built_without_torch(monkeypatch, runs):
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name.split(".")[0] == "torch" else find(name, *a))
    for name in ("torch", "torch.utils", "torch.utils.cpp_extension"):
        monkeypatch.setitem(__import__("sys").modules, name, None)  # import raises
    assert b.build() == b.LIB and os.path.exists(b.LIB)
    assert not runs and not os.path.exists(b.TORCH_LIB)


def test_the_binding_is_built_again_for_another_torch(monkeypatch, runs):
    import torch
    b.build()
    assert len(runs) == 1
    b.build()
    assert len(runs) == 1
    monkeypatch.setattr(torch, "__version__", "0.0.0")
    b.build()
    assert len(runs) == 2
    b.build()
    assert len(runs) == 2
