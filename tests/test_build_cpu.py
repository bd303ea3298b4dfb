"""What is built when, and what is loaded: the extension that marshals the attention calls is bound to one torch."""
import pytest

from paper_2506_04985_b200 import binding as B, build


@pytest.fixture(autouse=True, scope="module")
def built():
    build.build()


def test_the_extension_of_another_torch_is_built_again(monkeypatch):
    assert build._calls_fit()
    here = build.calls_abi()
    monkeypatch.setattr(build, "calls_abi", lambda: here + "1")
    assert not build._calls_fit()


def test_the_extension_of_another_torch_is_not_loaded(monkeypatch):
    monkeypatch.setattr(B, "_calls", None)
    monkeypatch.setattr(build, "calls_abi", lambda: "python 2.7 torch 0.4")
    with pytest.raises(RuntimeError, match="build it with"):
        B._native()
    assert B._calls is None
    monkeypatch.undo()
    assert B._native().abi == build.calls_abi()


def test_the_library_is_built_without_torch(monkeypatch, tmp_path):
    """A caller of the C functions alone."""
    import sys
    calls = tmp_path / "_calls.so"
    monkeypatch.setattr(build, "CALLS", str(calls))
    monkeypatch.setitem(sys.modules, "torch", None)
    assert build.build() == build.LIB
    assert not calls.exists()
