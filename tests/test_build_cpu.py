"""What a build runs, with the compilers replaced: the library needs no PyTorch, the module goes by the one that is installed."""
import importlib.util
import os

import pytest
import torch

from paper_2604_17861_amd import build as B


@pytest.fixture
def ran(monkeypatch):
    """The commands of every call, in the order of their ends."""
    commands = []
    monkeypatch.setattr(B, "_all", lambda jobs: commands.extend(jobs) or "")
    return commands


@pytest.fixture
def no_torch(monkeypatch):
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *rest: None if name == "torch" else find(name, *rest))


def links(commands):
    return [c for c in commands if B.LIB in c]


def test_the_library_is_built_without_pytorch(ran, no_torch):
    assert B.build(force=True) == B.LIB
    assert len(links(ran)) == 1 and len(ran) == len(B.SOURCES) + 1 and all(os.path.basename(c[0]) == "hipcc" for c in ran)


def test_without_pytorch_a_module_that_is_not_there_is_not_missing(monkeypatch, no_torch, tmp_path):
    made = tmp_path / "made.so"
    made.write_bytes(b"")
    monkeypatch.setattr(B, "LIB", str(made))
    monkeypatch.setattr(B, "BINDING", str(tmp_path / "none.so"))
    assert not B.needs_build()


def test_with_pytorch_it_is(monkeypatch, tmp_path):
    made = tmp_path / "made.so"
    made.write_bytes(b"")
    monkeypatch.setattr(B, "LIB", str(made))
    monkeypatch.setattr(B, "BINDING", str(tmp_path / "none.so"))
    assert B.needs_build()


def test_the_library_is_linked_where_the_module_fails(monkeypatch):
    commands = []

    def run(jobs):
        if any(B.BINDING in j for j in jobs):
            raise RuntimeError("g++ failed")
        commands.extend(jobs)
        return ""
    monkeypatch.setattr(B, "_all", run)
    with pytest.raises(RuntimeError, match="g.. failed"):
        B.build(force=True)
    assert len(links(commands)) == 1


@pytest.mark.parametrize("abi", (False, True))
def test_the_module_has_the_abi_of_pytorch(monkeypatch, abi):
    monkeypatch.setattr(torch, "compiled_with_cxx11_abi", lambda: abi)
    assert "-D_GLIBCXX_USE_CXX11_ABI=%d" % abi in B.binding_command()
