"""What csrc/marshal.c binds: integers and pointers in their places, one double among them at most."""
import ctypes
import importlib.util
import math
import os

import pytest

from paper_2504_04673_amd import binding, build


@pytest.fixture(scope="module")
def ext(tmp_path_factory):
    """Built beside the package's own, which stays as it is."""
    with pytest.MonkeyPatch.context() as patch:
        patch.setattr(build, "MARSHAL", str(tmp_path_factory.mktemp("ext") / os.path.basename(build.MARSHAL)))
        spec = importlib.util.spec_from_file_location("_marshal", build.build_marshal())
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_a_second_double_has_no_place(ext):
    address = ctypes.cast(binding.lib().sagnn_version, ctypes.c_void_p).value
    for kinds in ("dd", "pdid", "d" * 24):
        with pytest.raises(ValueError, match="doubles"):
            ext.bind(address, kinds, TypeError)
    for kinds in ("x", "pi ", "f", "P"):
        with pytest.raises(ValueError, match="expected"):
            ext.bind(address, kinds, TypeError)
    with pytest.raises(ValueError):
        ext.bind(0, "p", TypeError)
    with pytest.raises(ValueError):
        ext.bind(address, "i" * 25, TypeError)


def test_a_double_arrives_wherever_it_stands(ext):
    """A C function of this process that is given nine integers and a double, the double in every place."""
    got = []
    for at in range(10):
        kinds = "i" * at + "d" + "i" * (9 - at)
        types = [ctypes.c_double if k == "d" else ctypes.c_int64 for k in kinds]

        @ctypes.CFUNCTYPE(ctypes.c_int, *types)
        def seen(*args):
            got.append(args)
            return len(got)

        call = ext.bind(ctypes.cast(seen, ctypes.c_void_p).value, kinds, TypeError)
        args = [math.pi if k == "d" else 100 * at + i for i, k in enumerate(kinds)]
        assert call(*args) == len(got) and list(got[-1]) == args
        for wrong in ("1.0", None, [1.0]):
            with pytest.raises(TypeError, match="a number expected"):
                call(*[wrong if k == "d" else a for k, a in zip(kinds, args)])
    assert len(got) == 10


def test_no_exported_call_has_two(ext):
    for name in binding.EXPORTS[3:]:
        assert sum(t is ctypes.c_double for t in getattr(binding.lib(), name).argtypes or ()) <= 1, name
