"""The library builds where torch is not installed: the engine and the C boundary need none."""
import importlib.util

from paper_2509_06980_amd import build


def test_no_binding_to_torch_without_torch(monkeypatch):
    find = importlib.util.find_spec
    monkeypatch.setattr(importlib.util, "find_spec", lambda name, *a: None if name == "torch" else find(name, *a))
    calls = []
    monkeypatch.setattr(build.subprocess, "run", lambda *a, **k: calls.append(a))
    assert build.build_torch_binding() is None and not calls
