"""The C library builds without torch; the Python binding of the calls on rows is built, and loaded, for the torch that is there."""
import os
import shutil
import subprocess
import sys

import pytest
import torch

from paper_2110_14871_b200 import build as gbuild
from paper_2110_14871_b200 import gdws

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def built():
    gbuild.build_library()


def test_the_library_needs_no_torch(tmp_path):
    """The build script in a Python without site-packages, beside an up-to-date library and no binding."""
    shutil.copytree(os.path.join(ROOT, "include"), tmp_path / "include")
    shutil.copytree(os.path.join(ROOT, "paper_2110_14871_b200"), tmp_path / "package", ignore=shutil.ignore_patterns("_rows.so", "_build", "__pycache__"))
    r = subprocess.run([sys.executable, "-S", str(tmp_path / "package" / "build.py")], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == str(tmp_path / "package" / "libgdws.so"), r.stderr[-2000:]
    assert not (tmp_path / "package" / "_rows.so").exists()


def test_the_binding_is_rebuilt_for_another_torch(tmp_path, monkeypatch):
    assert not gbuild.binding_is_stale()
    monkeypatch.setattr(gbuild, "_torch_version", lambda: "1.0")
    assert gbuild.binding_is_stale()
    monkeypatch.undo()
    monkeypatch.setattr(gbuild, "BINDING_FOR", str(tmp_path / "none.txt"))
    assert gbuild.binding_is_stale()


def test_a_binding_for_another_torch_is_not_loaded(monkeypatch):
    monkeypatch.setattr(torch, "__version__", "1.0.0+cu1")
    monkeypatch.setattr(gdws, "_rows", None)
    q = torch.zeros((4, 8), dtype=torch.int8)
    with pytest.raises(ImportError, match="1.0.0"):
        gdws.quantize_rows(torch.zeros((4, 8)), q, torch.zeros(4))


def test_a_pre_release_of_the_same_torch_is(monkeypatch):
    """Its version has a suffix that its headers leave out."""
    monkeypatch.setattr(torch, "__version__", torch.__version__.split("+")[0] + "a0+git1234567")
    monkeypatch.setattr(gdws, "_rows", None)
    assert gdws._rows_setup() is not None
