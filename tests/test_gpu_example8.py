"""GPU: the example of a session runs over pages of 8-bit codes, its own checks with it."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("codes", [torch.float8_e4m3fn, torch.int8])
def test_window_session_in_8_bits(ctx, codes):
    spec = importlib.util.spec_from_file_location("window_session", os.path.join(ROOT, "examples", "window_session.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert m.main(codes) == 3 * 20 * 22 + 4 + 3
