"""The example that runs projections, cache and attention together."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_attention_block():
    spec = importlib.util.spec_from_file_location("attention_block", os.path.join(ROOT, "examples", "attention_block.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    assert example.main() < 2.0 ** -8
