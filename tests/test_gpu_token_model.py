"""The example that trains two modules with delayed gradients on the operators of token models."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "token_model.py")


def test_token_model_learns():
    """The loss starts at that of equal chances and falls most of the way to the data's entropy; 8-bit activations leave it where it is."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    spec = importlib.util.spec_from_file_location("token_model", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses, entropy, (plain, eight) = m.train(300, lambda s: print(s, flush=True))
    start, end = losses[0], sum(losses[-20:]) / 20
    assert abs(start - torch.tensor(float(m.VOCAB)).log().item()) < 0.2
    assert end - entropy < 0.3 * (start - entropy), (start, end, entropy)
    assert plain < end + 0.1 and abs(eight - plain) < 0.02 * plain
