"""When the module that marshals arguments is compiled again: it is tied to the C++ interface of the torch and the Python it was built for."""
import importlib.metadata
import os
import shutil
import subprocess
import sys

import pytest


@pytest.fixture
def builder(monkeypatch):
    from paper_2009_03106_b200 import build as b
    if not (os.path.exists("/usr/local/cuda/bin/nvcc") or shutil.which("nvcc")):
        pytest.skip("no nvcc")
    b.build()
    started = []
    monkeypatch.setattr(subprocess, "Popen", lambda cmd, *a, **k: started.append(cmd))
    return b, started


def test_up_to_date(builder):
    b, started = builder
    assert b._start_marshal(False) is None and not started


def test_another_torch(builder, monkeypatch):
    b, started = builder
    version = importlib.metadata.version
    monkeypatch.setattr(importlib.metadata, "version", lambda name: "0.0.0" if name == "torch" else version(name))
    assert b._start_marshal(False) is not None and len(started) == 1


def test_another_python(builder, monkeypatch):
    b, started = builder
    monkeypatch.setattr(sys, "version", "0.0.0 (of no interpreter)")
    assert b._start_marshal(False) is not None and len(started) == 1
