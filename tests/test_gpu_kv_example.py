"""The serving example: q/k/v group, tables, cache, attention and o_proj together, in steps and as one prompt."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_steps_and_one_prompt_agree():
    spec = importlib.util.spec_from_file_location("serve_block", os.path.join(ROOT, "examples", "serve_block.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    # Both ways round q, k and v alike up to the order of sums in fp32, so that a rounding to bfloat16 (2^-9) or to the cache's
    # E4M3 grid (2^-4 of the number) falls the other way now and then; the weights' rounding (2^-9) is of either side.  A
    # part in fifty of the values one grid step off would be 2^-4 / sqrt(50) of the norm; wrong rows would be of order one
    assert example.main(prompts=(150, 20, 70), tokens=12) < 1e-2
