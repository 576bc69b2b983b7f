"""What a build writes and what it leaves alone, in directories of its own; and the lists of tensors where they are not built."""
import os

import pytest
import torch

from paper_2504_04673_amd import binding, build


@pytest.fixture
def elsewhere(monkeypatch, tmp_path):
    """Everything that a build writes, in a directory of the test, and nothing of the library to compile."""
    for name in ("LIB", "MARSHAL", "GRADLIST"):
        monkeypatch.setattr(build, name, str(tmp_path / os.path.basename(getattr(build, name))))
    monkeypatch.setattr(build, "SOURCES", [])
    monkeypatch.setenv("HIPCC", "true")
    return tmp_path


def test_building_the_library_leaves_the_lists_alone(elsewhere, monkeypatch):
    """Whether there is a compiler for them or not."""
    for compiler in ("g++", str(elsewhere / "none")):
        monkeypatch.setenv("CXX", compiler)
        with open(build.GRADLIST, "w") as f:
            f.write("what was there")
        build.build_hip()
        assert open(build.GRADLIST).read() == "what was there" and os.path.exists(build.MARSHAL)


def test_lists_are_built_whole_or_not_at_all(elsewhere, monkeypatch):
    build.build_all()
    assert sorted(os.listdir(elsewhere)) == sorted(os.path.basename(p) for p in (build.MARSHAL, build.GRADLIST))
    monkeypatch.setenv("CXX", str(elsewhere / "none"))
    with pytest.warns(UserWarning, match="lists of tensors"):
        build.build_all()
    assert os.listdir(elsewhere) == [os.path.basename(build.MARSHAL)]


def test_lists_are_read_in_python_where_they_are_not_built(monkeypatch, tmp_path):
    monkeypatch.setattr(binding, "_rows", None)
    monkeypatch.setattr(build, "GRADLIST", str(tmp_path / "none"))
    assert binding._grad_list([]) == (b"", 0) and binding._rows is binding._rows_in_python


def test_lists_built_for_another_torch_are_out_of_date_and_not_loaded(elsewhere, monkeypatch):
    assert not build.gradlist_fits()
    build.build_gradlist()
    assert build.gradlist_fits() and not build.gradlist_stale()
    monkeypatch.setattr(torch, "__version__", "2.1")               # (a prefix of 2.10 among others)
    assert not build.gradlist_fits() and build.gradlist_stale()
    monkeypatch.setattr(binding, "_rows", None)
    monkeypatch.setattr(binding, "_extension", lambda *a: pytest.fail("loaded"))
    assert binding._grad_list([]) == (b"", 0) and binding._rows is binding._rows_in_python
