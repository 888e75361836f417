"""The example that runs the operators together: an MLP block forwards and one fine-tuning step, against unquantised weights in 64 bits."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "fp8_mlp_block.py")


def test_block_and_its_step():
    """A value in 8 bits is within 2^-4 of itself, 2^-4 / sqrt(12) * 2 in the mean square at the most (3.6 %), and an inner product of two such
    operands within sqrt(2) of that. The block adds s, which has no such error, to two products in a row (each with both operands in 8 bits): below
    10 %; its gradients pass through two products and silu's slope with the same errors."""
    spec = importlib.util.spec_from_file_location("fp8_mlp_block", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    for hidden, width, tokens in ((640, 1300, 77), (256, 512, 1), (512, 384, 300)):
        errors = module.check(hidden, width, tokens)
        assert all(e < 0.1 for e in errors.values()), errors
