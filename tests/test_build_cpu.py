"""The optional module ``_rows`` never stands in the way of the library."""
import os
from types import SimpleNamespace

import pytest
import torch

from paper_2608_06146_amd import _lib, build

HEADER = "include/torch/csrc/autograd/python_variable.h"
ROCM = ["include/c10/hip/HIPStream.h", "lib/libc10_hip.so"]


def pytorch_of(monkeypatch, root, files):
    """A PyTorch at ``root`` that has these files, and an empty build folder."""
    for f in ["version.py"] + files:
        path = root / "torch" / f
        path.parent.mkdir(parents=True, exist_ok=True)
        path.write_text("__version__ = '0.0'\n" if f == "version.py" else "")
    monkeypatch.setattr(build.importlib.util, "find_spec",
                        lambda name: SimpleNamespace(submodule_search_locations=[str(root / "torch")]))
    monkeypatch.setattr(build, "BUILD", str(root))


@pytest.mark.parametrize("files", [[], [HEADER], [HEADER, ROCM[0]]])
def test_a_pytorch_without_rocm(monkeypatch, tmp_path, files):
    pytorch_of(monkeypatch, tmp_path, files)
    out = tmp_path / "_rows.so.tmp"
    assert build._compile_rows("/bin/false", str(out), force=True) is False and not out.exists()


def test_a_pytorch_whose_headers_do_not_compile(monkeypatch, tmp_path):
    pytorch_of(monkeypatch, tmp_path, [HEADER] + ROCM)
    out = tmp_path / "_rows.so.tmp"
    with pytest.warns(UserWarning, match="_rows is left out"):
        assert build._compile_rows(build.hipcc(), str(out), force=True) is False
    assert not out.exists() and not [f for f in os.listdir(tmp_path) if f.startswith("rows.")]


def test_a_module_of_another_pytorch_is_not_used(monkeypatch):
    rows = _lib.native_rows()
    assert rows is not None and rows.torch_version == torch.__version__
    monkeypatch.setattr(torch, "__version__", "2.0.0+other")
    assert _lib.native_rows() is None
