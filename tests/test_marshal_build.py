"""The binding's Python module on the CPU: which file is loaded, and how it is replaced."""
from __future__ import annotations

import os
import shutil
import sysconfig

import pytest

from tests.test_library_cpu import psc  # noqa: F401

torch = pytest.importorskip("torch")
SUFFIX = sysconfig.get_config_var("EXT_SUFFIX")


@pytest.fixture
def module(psc):  # noqa: F811
    """The path of the built module; the binding's own is put back afterwards."""
    from paper_2608_03065_gb300 import build
    if not os.path.exists(build.MARSHAL):
        pytest.skip("the module is not built here")
    yield build.MARSHAL
    psc._load_marshal(psc.load())


@pytest.mark.parametrize("name,loaded", [("_marshal" + SUFFIX, True), ("_marshal.so", False),
                                         ("_marshal.cpython-39-other.so", False)])
def test_only_this_interpreters_module_is_loaded(psc, monkeypatch, tmp_path, module, name, loaded):  # noqa: F811
    shutil.copy(module, tmp_path / name)
    with monkeypatch.context() as m:
        m.setattr(psc, "_HERE", str(tmp_path))
        m.setattr(psc, "_marshal", None)
        psc._load_marshal(psc.load())
        assert (psc._marshal is not None) == loaded
