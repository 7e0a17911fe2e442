"""The library builds and loads where the binding's module does not: without torch, where torch's
headers do not compile, or with a module that does not load."""
import os
import subprocess
import sys
import sysconfig
import time

import pytest
import torch

from paper_2608_24658_gb300 import _lib, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def aside(monkeypatch, tmp_path, tensors):
    """A build of a small library in a folder of its own, with `tensors` as the module's source."""
    out = tmp_path / "out"
    out.mkdir()
    src, module = tmp_path / "small.cpp", tmp_path / "tensors.cpp"
    src.write_text('extern "C" int small() { return 7; }\n')
    module.write_text(tensors)
    monkeypatch.setattr(build, "BUILD", str(out))
    monkeypatch.setattr(build, "LIB", str(out / "libsmall.so"))
    monkeypatch.setattr(build, "TENSORS_SRC", str(module))
    monkeypatch.setattr(build, "_sources", lambda: ([str(src)], []))
    if hasattr(build, "TENSORS"):
        monkeypatch.setattr(build, "TENSORS", str(out / os.path.basename(build.TENSORS)))
    for f in (src, module):                                # (older than this build's own code, as files of a checkout are)
        os.utime(f, (1, 1))
    return out, module


def test_a_module_that_does_not_compile(monkeypatch, tmp_path, capsys):
    out, module = aside(monkeypatch, tmp_path, "#error no headers\n")
    assert build.build() == str(out / "libsmall.so") and os.path.exists(build.build())
    made = {f: os.path.getmtime(out / f) for f in os.listdir(out)}
    assert not any(f.startswith("_tensors") and f.endswith(".so") for f in made)
    if os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        assert "did not compile" in capsys.readouterr().err
        assert any("no headers" in (out / f).read_text() for f in made if f.endswith(".failed"))
    # neither is tried again until something changes
    build.build()
    assert made == {f: os.path.getmtime(out / f) for f in os.listdir(out)}


def test_a_source_that_is_mended(monkeypatch, tmp_path):
    out, module = aside(monkeypatch, tmp_path, "#error no headers\n")
    build.build()
    if not any(f.endswith(".failed") for f in os.listdir(out)):
        pytest.skip("nothing here to build the module with")
    lib = os.path.getmtime(out / "libsmall.so")
    module.write_text("extern \"C\" int nothing() { return 0; }\n")
    os.utime(module, (time.time() + 5, time.time() + 5))
    build.build()
    assert any(f.startswith("_tensors") and f.endswith(".so") for f in os.listdir(out))
    assert os.path.getmtime(out / "libsmall.so") == lib


def test_a_module_that_does_not_load(monkeypatch, tmp_path):
    name = f"_tensors-{torch.__version__}{sysconfig.get_config_var('EXT_SUFFIX')}"
    (tmp_path / name).write_bytes(b"no library")
    monkeypatch.setattr(_lib, "LIB_PATH", str(tmp_path / "libparason.so"))
    for f in ("flat", "rows", "alike"):
        monkeypatch.setattr(_lib, f, _lib._unknown)
    with pytest.warns(UserWarning):
        _lib._load_tensors()
    assert _lib.flat is _lib.rows is _lib.alike is _lib._unknown


@pytest.mark.parametrize("what", ["from paper_2608_24658_gb300 import build; build.build()",
                                  "from paper_2608_24658_gb300 import _lib; assert _lib.load().parason_version()"])
def test_without_torch(what):
    """Building (nothing is left to do here) and loading the library ask for no torch."""
    build.build()
    run = subprocess.run([sys.executable, "-c", f"import sys; sys.modules['torch'] = None; {what}"], cwd=ROOT,
                         capture_output=True, text=True)
    assert run.returncode == 0, run.stderr
