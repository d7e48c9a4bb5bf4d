"""GPU: the example of a session on a windowed cache runs, and its own checks hold."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_window_session(ctx):
    spec = importlib.util.spec_from_file_location("window_session", os.path.join(ROOT, "examples", "window_session.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert m.main() == 3 * 20 * 22 + 4 + 3
