"""The bindings' native module refuses to load under another torch than it was built for (CPU only)."""
import importlib.util
import os
import shutil

import pytest
import torch

from paper_2607_28848_amd import _marshal


def load(path):
    spec = importlib.util.spec_from_file_location("_marshal", path)
    return importlib.util.module_from_spec(spec)


def test_another_torch(tmp_path, monkeypatch):
    copies = [shutil.copy(_marshal.__file__, os.path.join(tmp_path, "%d_marshal.so" % i)) for i in range(2)]
    assert load(copies[0]).where(torch.zeros(1)) == -1
    monkeypatch.setattr(torch, "__version__", "2.0.0")
    with pytest.raises(ImportError, match="build it again"):
        load(copies[1])
