"""The C library is built where torch is not installed (its callers may be C programs)."""
import importlib.util
import os

from paper_2607_29591_gb300 import build as B


def test_the_library_needs_no_torch(monkeypatch):
    B.build()
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    ran = []
    monkeypatch.setattr(B.subprocess, "run", lambda cmd, **k: ran.append(cmd))
    assert B.build() == B.LIB and os.path.exists(B.LIB)
    B._bind(force=True)
    assert not ran                                     # nothing is compiled against headers that are not there
