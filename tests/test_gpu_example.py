"""examples/attention_block.py: base product, apply, cache and attention together, against float64 on unquantised
values.  Bound: x and the weights each lose up to 2^-4 of a value to e4m3 (an rms of 2.6 % each for values
spread over a binade), k and v again; such errors on the way to y measure 8.3 % together, less where
attention averages them out.  A missing adapter, prompt or head would show as 20 % or more."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def test_attention_block():
    print("\n[gpu case] example", flush=True)
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_block.py")
    spec = importlib.util.spec_from_file_location("attention_block", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert m.main(4) < 0.1
