"""The example that trains adapters and LayerNorms through the operators and serves several collections in one call."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "adapt_block.py")


def test_adapters_learn_and_serve():
    spec = importlib.util.spec_from_file_location("adapt_block", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, difference = example.main(steps=60)
    # Half of the outputs' variance is the teacher's change at the start; dropout of p = 0.05 keeps about p of the branch's variance as noise.
    assert losses[-1] < 0.25 * losses[0], losses
    # Outputs are of order 1 (up to 5 or so): two roundings to bf16 of either path and what the second sublayer makes of the first one's
    assert difference < 4 * 2.0 ** -8 * 5
