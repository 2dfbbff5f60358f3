"""The decoder operators and the contractions together, as the example uses them."""
import importlib.util
import os

import pytest

import helpers

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_decode_example():
    helpers.api()
    spec = importlib.util.spec_from_file_location("decode_example", os.path.join(ROOT, "examples", "decode.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    # fp32 throughout: products to 2^-21, contractions over 256 and 512 terms, softmax over at most 60 tokens: some 1e-6
    # of the largest output; 1e-5 is the bound that fp32 contractions are held to
    assert example.main(60) < 1e-5
