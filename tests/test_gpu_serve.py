"""The store and the paged cache's operators together, as the example runs them (MI355X)."""
from __future__ import annotations

import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "fp16", "mxfp4"])
def test_serve_step(kind):
    spec = importlib.util.spec_from_file_location("serve_step", os.path.join(ROOT, "examples", "serve_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    assert mod.main(kind, requests=5, passage=160, steps=3) >= 5 * 160
