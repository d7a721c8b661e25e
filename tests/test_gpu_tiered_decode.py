"""The example: decoding over a pool whose programs move out and back in."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_outputs_do_not_depend_on_moves():
    spec = importlib.util.spec_from_file_location("tiered_decode", os.path.join(ROOT, "examples", "tiered_decode.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    moved = example.main()
    assert moved["out"] > 0 and moved["in"] > 0 and moved["tokens"] > 1000
