"""The example of the attention half of a layer, which checks every output of its own."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_layer.py")


@pytest.mark.parametrize("window,sinks,hidden,heads,kv_heads", [(0, 0, 1024, 8, 2), (64, 4, 1024, 8, 2), (40, 0, 640, 10, 10)])
def test_attention_layer(window, sinks, hidden, heads, kv_heads):
    print("case: example", window, sinks, hidden, flush=True)
    spec = importlib.util.spec_from_file_location("attention_layer", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    example.main(window, sinks, hidden, heads, kv_heads, prompt=90, steps=45)
