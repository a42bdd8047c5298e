"""The build of the module that hands on tensors: after the library and apart from it, and again when what it was compiled against
changes.  No GPU."""
import os

import pytest

FAILS = "/bin/false"                               # a compiler that cannot


@pytest.fixture
def build(monkeypatch, tmp_path):
    from paper_2604_18655_b200 import build as b
    b.build()                                      # objects are up to date: below, the library is only linked
    monkeypatch.setattr(b, "LIB", str(tmp_path / "libmlora.so"))
    monkeypatch.setattr(b, "MARSHAL", str(tmp_path / "_marshal.so"))
    return b


@pytest.mark.parametrize("compiler", [FAILS, "/nowhere/no-such-compiler"])
def test_library_is_built_where_the_module_fails(build, monkeypatch, compiler):
    monkeypatch.setenv("CXX", compiler)
    with pytest.raises(RuntimeError) as e:
        build.build()
    assert "_marshal.so" in str(e.value) and compiler in str(e.value) and "nvcc failed" not in str(e.value)
    assert os.path.exists(build.LIB) and not os.path.exists(build.MARSHAL)


def test_library_is_built_without_torch(build, monkeypatch):
    find = build.importlib.util.find_spec
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    monkeypatch.setenv("CXX", FAILS)
    assert build.build() == build.LIB and os.path.exists(build.LIB)


def test_module_is_made_again_for_another_torch_or_python(build, monkeypatch):
    build.build()
    monkeypatch.setenv("CXX", FAILS)
    assert build.build() == build.LIB              # up to date: nothing is compiled
    monkeypatch.setattr(build.importlib.metadata, "version", lambda name: "0.0")
    with pytest.raises(RuntimeError):
        build.build()
    monkeypatch.undo()
    monkeypatch.setenv("CXX", FAILS)
    monkeypatch.setattr(build.sys.implementation, "cache_tag", "cpython-999")
    monkeypatch.setattr(build, "_newer", lambda target, deps: True)
    with pytest.raises(RuntimeError):
        build.build_marshal()


def test_torch_without_a_distribution_is_known_by_its_files(build, monkeypatch):
    def missing(name):
        raise build.importlib.metadata.PackageNotFoundError(name)
    known = build._marshal_made_for()
    monkeypatch.setattr(build.importlib.metadata, "version", missing)
    other = build._marshal_made_for()
    assert other and other != known and other == build._marshal_made_for()
