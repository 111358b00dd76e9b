"""The Python module of the library's entries is compiled with torch's and Python's memory layouts: another torch or Python does not
take it, and one that does not load is built anew by the command that its error names."""
import os
import sysconfig

import pytest
import torch

import paper_1905_04035_b200 as dst
from paper_1905_04035_b200 import binding, build


@pytest.fixture
def fresh(monkeypatch):
    """A binding that has not loaded the module yet."""
    build.build_library()
    monkeypatch.setattr(binding, "_calls", None)


def test_the_module_s_file_is_that_of_this_torch_and_this_python(fresh, monkeypatch):
    here = binding.calls_path()
    assert os.path.exists(here) and torch.__version__ in here and here.endswith(sysconfig.get_config_var("EXT_SUFFIX"))
    assert binding.load_calls().__file__ == here and not build.is_stale()
    binding._calls = None
    monkeypatch.setattr(torch, "__version__", "1.2.3+other")
    assert binding.calls_path() != here and build.is_stale()
    with pytest.raises(ImportError, match="paper_1905_04035_b200.build"):
        binding.load_calls()
    monkeypatch.undo()
    monkeypatch.setattr(binding, "_calls", None)
    monkeypatch.setattr(torch, "compiled_with_cxx11_abi", lambda: False)
    assert binding.calls_path() != here and build.is_stale()


def test_a_module_that_does_not_load_is_built_anew_and_the_library_is_not(fresh, monkeypatch, tmp_path):
    path = tmp_path / ("_calls" + sysconfig.get_config_var("EXT_SUFFIX"))
    path.write_bytes(b"this is no module")
    os.symlink(build.LIB_PATH, tmp_path / os.path.basename(build.LIB_PATH))   # (the module looks for the library beside itself)
    monkeypatch.setattr(binding, "calls_path", lambda: str(path))
    with pytest.raises(ImportError, match="paper_1905_04035_b200.build"):
        binding.load_calls()
    before = os.stat(build.LIB_PATH)
    assert build.is_stale()
    build.build_library()
    assert os.stat(build.LIB_PATH).st_mtime_ns == before.st_mtime_ns and not build.is_stale()
    calls = binding.load_calls()
    assert calls.__file__ == str(path) and calls.dst_clip(None, None, 0, 256, None) == 0
    assert calls.matrix(torch.zeros(3, 8)[:, :5], 3, 5, -1, "x")[1:] == (8, 0)


def test_a_library_that_does_not_load_is_stale(fresh, monkeypatch, tmp_path):
    path = tmp_path / "libdst_b200.so"
    path.write_bytes(b"this is no library")
    for module, name in ((binding, "_LIB_PATH"), (build, "LIB_PATH")):
        monkeypatch.setattr(module, name, str(path))
    monkeypatch.setattr(binding, "_lib", None)
    assert build.is_stale() and build.stale_parts() == (True, True)
    with pytest.raises(OSError):
        dst.load_library()


def test_the_module_is_compiled_without_a_toolkit_s_headers():
    """It includes none of CUDA's, and the compiler that the library is built with may lie anywhere."""
    compile_calls, link_calls = build._calls_commands("a.o", "a.so")
    assert not any("cuda" in os.path.relpath(a, os.path.dirname(torch.__file__)) for a in compile_calls + link_calls if a.startswith("/"))
