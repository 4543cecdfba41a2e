"""The example layer: all operators together, as a training step and as a server runs them."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# Between an input and a result stand at most eight results rounded to bfloat16, each within 2^-8 of its value.
ROUNDED = 8 * 2.0 ** -8
# 4 bits: 64 normal numbers span 4.7 deviations on average, so a step is 0.31 and a number 0.09 of a deviation off (root mean square), in keys and in values.  A score of normed
# heads is then off by head_dim ** -0.5 * |q| * 0.09 = 0.09, a weight by a factor of as much, and an average of values by 0.09 of itself for either: 0.13 together.  Twice that.
CACHED = 0.26


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_layer.py")
    spec = importlib.util.spec_from_file_location("attention_layer_example", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("lens,q_heads,k_heads,head_dim", [((300, 1, 133), 8, 2, 128), ((129, 64), 6, 6, 64)])
def test_training_step(example, lens, q_heads, k_heads, head_dim):
    errors = example.train(lens, 256, q_heads, k_heads, head_dim)
    assert all(e <= ROUNDED for e in errors.values()), errors


@pytest.mark.parametrize("lens,q_heads,k_heads,head_dim", [((200, 3, 131), 8, 2, 128), ((77, 64), 6, 6, 64)])
def test_serving(example, lens, q_heads, k_heads, head_dim):
    errors = example.serve(lens, 4, 256, q_heads, k_heads, head_dim)
    assert errors.pop("first piece") <= ROUNDED and all(e <= CACHED for e in errors.values()), errors
