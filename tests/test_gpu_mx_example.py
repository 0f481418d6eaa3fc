"""The offloaded layer of examples/, whose weights and checkpoints cross the encrypted link as MX tensors."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "offloaded_layer.py")


@pytest.fixture(scope="module")
def layer():
    spec = importlib.util.spec_from_file_location("offloaded_layer", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("tokens,width,hidden", [(1, 64, 96), (37, 200, 333), (512, 512, 1024)])
def test_a_step_is_the_layers_in_float32(layer, tokens, width, hidden):
    """y and dx: bf16 rounding of three products in a row, 2^-8 each at most. Gradients from the 8-bit checkpoints: an
    element is off by at most 2^-7 of its block's largest, so by less than 3 parts in 100 of a normal tensor's norm."""
    errors, crossed = layer.run(tokens, width, hidden)
    assert errors[0] < 3 * 2.0 ** -8
    assert all(e < 0.03 + 3 * 2.0 ** -8 for e in errors[1:])
    weights = 2 * (2 * hidden * -(-width // 32) + width * -(-hidden // 32)) * 17
    kept = 2 * tokens * (-(-width // 32) + 3 * -(-hidden // 32)) * 33
    assert crossed == weights + kept


def test_a_tampered_message_is_refused(layer):
    link = layer.Link(bytes(range(32)))
    iv, ct, tags = layer.quantised_message(link, torch.randn(100, 200, device="cuda"))
    ct[777] ^= 1
    with pytest.raises(RuntimeError, match="1 chains"):
        link.fetch((iv, ct, tags))
