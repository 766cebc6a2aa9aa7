"""The compiled Python calls' place in the build: theirs alone needs Python's headers, and one interpreter's are not another's."""
import os
import sys
import sysconfig

import pytest

from paper_2511_04063_b200 import binding, build


@pytest.fixture(autouse=True)
def built():
    build.build()


def test_the_module_carries_the_interpreters_tag():
    suffix = sysconfig.get_config_var("EXT_SUFFIX")
    assert suffix != ".so" and os.path.basename(build.CALLS) == "_calls" + suffix and os.path.exists(build.CALLS)
    assert not os.path.exists(os.path.join(build.HERE, "_calls.so"))     # (any interpreter would load that one)
    from paper_2511_04063_b200 import _calls
    assert _calls.__file__ == build.CALLS


def test_an_untagged_module_does_not_stay():
    open(build.UNTAGGED, "w").close()
    build.build()
    assert not os.path.exists(build.UNTAGGED)


def test_without_pythons_headers_the_library_is_still_built(monkeypatch, tmp_path):
    missing = str(tmp_path / "_calls.so")
    monkeypatch.setattr(build, "CALLS", missing)
    monkeypatch.setattr(sysconfig, "get_paths", lambda *a, **k: {"include": str(tmp_path), "platinclude": str(tmp_path)})
    before = os.path.getmtime(build.LIB)
    with pytest.warns(UserWarning, match="Python.h"):
        assert build.build() == build.LIB
    assert not os.path.exists(missing) and os.path.getmtime(build.LIB) == before     # nor is the library built over and over
    assert binding.load_library().dq_version() is not None


def test_without_the_module_the_operators_say_what_is_missing(monkeypatch):
    monkeypatch.setattr(binding, "_calls", None)
    monkeypatch.delattr(sys.modules["paper_2511_04063_b200"], "_calls", raising=False)
    monkeypatch.setitem(sys.modules, "paper_2511_04063_b200._calls", None)
    with pytest.raises(ImportError, match="Python.h"):
        binding.dq_mx_quantize(None, 0, None, None)


def test_a_fault_in_its_source_is_an_error(monkeypatch, tmp_path):
    monkeypatch.setattr(build, "CALLS", str(tmp_path / "_calls.so"))
    monkeypatch.setenv("CXX", "false")
    with pytest.raises(RuntimeError, match="py_calls"):
        build.build()
