"""What build() leaves behind where the module of torch calls cannot be built."""
import importlib.util

import pytest

from paper_2608_14586_amd import build


@pytest.fixture
def dry(monkeypatch):
    """build() with the compilers of the library and the linker left out; returns what was linked."""
    linked = []
    monkeypatch.setattr(build, "_compile", lambda src: src + ".o")
    monkeypatch.setattr(build, "_link", lambda cmd, out: linked.append(out))
    return linked


def test_without_torch(dry, monkeypatch):
    """The library is there, and the error names what is missing."""
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    with pytest.raises(RuntimeError, match="torch is not installed"):
        build.build()
    assert dry == [build.LIB]


def test_without_a_host_compiler(dry, monkeypatch):
    monkeypatch.setenv("PATH", "/nonexistent")
    with pytest.raises(RuntimeError, match=r"g\+\+"):
        build.build()
    assert dry == [build.LIB]
