"""CPU-only: when the compiled part of the binding is built again.  It holds torch's C++ interface, so another torch or another
Python makes it stale as a newer source does.  Compilers are replaced by a recorder."""

import importlib.metadata
import importlib.util
import os
import types

import pytest

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def builder(tmp_path, monkeypatch):
    spec = importlib.util.spec_from_file_location("_build_under_test", os.path.join(ROOT, "paper_1811_10751_b200", "build.py"))
    b = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(b)
    made = []

    def run(cmd, **kw):
        out = cmd[cmd.index("-o") + 1]
        open(out, "w").close()
        made.append(os.path.basename(out).split(".so")[0].split(".tmp")[0])
        return types.SimpleNamespace(returncode=0, stdout="", stderr="")
    monkeypatch.setattr(b.subprocess, "run", run)
    monkeypatch.setattr(b, "BUILD_DIR", str(tmp_path / "_build"))
    monkeypatch.setattr(b, "LIB_PATH", str(tmp_path / "libgpd.so"))
    monkeypatch.setattr(b, "BINDING_PATH", str(tmp_path / "_lm.so"))
    monkeypatch.setattr(b, "sources", lambda: [])
    monkeypatch.setattr(b, "_nvcc", lambda: "nvcc")
    return b, made


def test_binding_is_built_once_and_again_for_another_torch(builder, monkeypatch):
    b, made = builder
    b.build()
    assert made == ["libgpd", "_lm"]
    b.build()
    assert made == ["libgpd", "_lm"]                         # up to date
    real = importlib.metadata.version
    monkeypatch.setattr(torch, "__version__", "99.0.0+cu999")
    monkeypatch.setattr(importlib.metadata, "version", lambda name: "99.0.0+cu999" if name == "torch" else real(name))
    b.build()
    assert made == ["libgpd", "_lm", "_lm"]
    b.build()
    assert made == ["libgpd", "_lm", "_lm"]
    monkeypatch.undo()


def test_binding_of_unknown_origin_is_built_again(builder):
    """A binary without a record of what it was built for, such as an older checkout's."""
    b, made = builder
    open(b.LIB_PATH, "w").close()
    open(b.BINDING_PATH, "w").close()
    b.build()
    assert made == ["_lm"]
    b.build()
    assert made == ["_lm"]


def test_failed_build_is_not_recorded(builder, monkeypatch):
    b, made = builder
    run = b.subprocess.run
    monkeypatch.setattr(b.subprocess, "run", lambda cmd, **kw: types.SimpleNamespace(returncode=1, stdout="", stderr="no"))
    open(b.LIB_PATH, "w").close()
    open(b.BINDING_PATH, "w").close()
    with pytest.raises(RuntimeError):
        b.build()
    monkeypatch.setattr(b.subprocess, "run", run)
    b.build()
    assert made == ["_lm"]
