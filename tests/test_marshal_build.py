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


def test_a_rebuild_replaces_the_module_whole(monkeypatch, tmp_path, psc):  # noqa: F811
    """While it compiles, and where that fails, the file in place is the old one."""
    from paper_2608_03065_gb300 import build
    if not os.path.exists(build.MARSHAL):
        pytest.skip("the module is not built here")
    path, seen = tmp_path / "_marshal.so", []
    path.write_bytes(b"old")
    os.utime(path, (0, 0))                      # older than its source
    run = build.subprocess.run

    class Failed:
        returncode, stdout, stderr = 1, "", "no space left"

    def compiler(works):
        def f(cmd, **kw):
            out = cmd[cmd.index("-o") + 1]
            assert "marshal.cpp" in " ".join(cmd), "nothing else is stale"
            seen.append((out, path.read_bytes()))
            r = run(cmd, **kw)
            assert path.read_bytes() == b"old"
            return r if works else Failed
        return f

    monkeypatch.setattr(build, "MARSHAL", str(path))
    # the library is not linked again for a module that it does not hold
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    (tmp_path / "lib.so").write_bytes(b"")
    monkeypatch.setattr(build.subprocess, "run", compiler(False))
    with pytest.raises(RuntimeError, match="no space left"):
        build.build()
    assert path.read_bytes() == b"old"
    monkeypatch.setattr(build.subprocess, "run", compiler(True))
    build.build()
    assert path.read_bytes()[:4] == b"\x7fELF" and all(out != str(path) for out, _ in seen)
    assert sorted(os.listdir(tmp_path)) == ["_marshal.so", "lib.so"]
