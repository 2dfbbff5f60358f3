"""The layer of examples/verify.py: residual norms in 8 bits, 4-bit products, rotary append and tree attention together, in one captured
graph, against its plain recomputation."""
import importlib.util
import os

import pytest

from conftest import ROOT


@pytest.mark.gpu
def test_verify_example():
    # Both sides round at the same places, so they differ where a value lies next to a border: a bf16 value moves by 2^-7 of itself, an
    # 8-bit code by 2^-3.  A code is one of 256 terms of a sum of size sqrt(256): 2^-3 / 16 of a usual output; allowed are six of them.
    spec = importlib.util.spec_from_file_location("verify_example", os.path.join(ROOT, "examples", "verify.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    assert example.main(10) < 6 * 2.0 ** -3 / 16
