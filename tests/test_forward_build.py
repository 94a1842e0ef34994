"""The marshalling module is built for one torch and one Python, and no other takes it; no device."""
import importlib.metadata
import os
import sys

import pytest
import torch

from paper_2601_12917_b200 import build as zbuild
from paper_2601_12917_b200 import zgr


def test_the_module_is_named_by_what_it_was_built_for():
    zbuild.build()
    path = zbuild.bind_path()
    assert os.path.exists(path) and torch.__version__ in os.path.basename(path) and sys.implementation.cache_tag in path
    zgr._load_bind()


def test_another_torch_does_not_take_it(monkeypatch):
    zbuild.build()
    here, real = zbuild.bind_path(), importlib.metadata.version
    monkeypatch.setattr(importlib.metadata, "version", lambda name: "1.0+other" if name == "torch" else real(name))
    assert zbuild.bind_path() != here and not os.path.exists(zbuild.bind_path())
    monkeypatch.setattr(zgr, "_bind", None)
    with pytest.raises(ImportError, match="is missing"):
        zgr._load_bind()
    built = []
    monkeypatch.setattr(zbuild, "_build_bind", lambda: built.append(zbuild.bind_path()))      # up to date by its times, but another module's
    zbuild.build()
    assert built == [zbuild.bind_path()]
