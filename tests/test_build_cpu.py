"""The build command where there is no torch: the C library and its example do not need it."""
import sys

import pytest

from paper_2510_08525_amd import build


@pytest.fixture
def built(monkeypatch):
    done = []
    for name in ("build_library", "build_example", "build_tensor_calls"):
        monkeypatch.setattr(build, name, lambda name=name: done.append(name))
    return done


def test_without_torch_the_c_library_and_its_example_are_built(built, monkeypatch, capsys):
    monkeypatch.setitem(sys.modules, "torch", None)
    build.main()
    assert built == ["build_library", "build_example"]
    assert "_tensor_calls.so" in capsys.readouterr().out


def test_with_torch_everything_is(built):
    build.main()
    assert built == ["build_library", "build_example", "build_tensor_calls"]


def test_what_fails_to_build_is_not_hidden(built, monkeypatch):
    def fails():
        raise RuntimeError("compiler")

    monkeypatch.setattr(build, "build_tensor_calls", fails)
    with pytest.raises(RuntimeError, match="compiler"):
        build.main()
    assert built == ["build_library", "build_example"]
