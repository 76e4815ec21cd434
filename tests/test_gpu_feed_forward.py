"""The example that takes a feed-forward layer from training to serving, and the layer in its served forms."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_the_example_trains_and_serves():
    """Gradient descent from weights 0.3 off lowers the loss.  A value in 4 bits is a third of its scale's step off at most (relative to
    a block's largest between 1/8 and 1/4 of the value's own binade), near 0.1 of a weight's size over all, so three weights in
    4 bits leave the layer within 0.4; half of a normal weight's entries, the largest, hold 0.96 of its square."""
    import feed_forward
    out = feed_forward.main(["--d", "192", "--f", "500", "--tokens", "96", "--steps", "12"])
    assert out["last_loss"] < 0.9 * out["first_loss"]
    assert out["prompt_4bit"] < 0.4 and out["token_4bit"] < 0.4 and out["prompt_4bit_activations"] < 0.5
    assert out["prompt_pruned_down"] < 0.4


def test_a_layer_refuses_other_tokens_than_its_plan_is_for():
    import torch
    from feed_forward import prune
    from paper_2603_08734_amd import ffn
    w = torch.randn((48, 64), device="cuda").half()
    layer = ffn.FeedForward(torch.randn((64, 48), device="cuda").half(), torch.randn((64, 48), device="cuda").half(), prune(w, 0.5, 8))
    assert layer(torch.randn((8, 48), device="cuda").half()).shape == (8, 48)
    with pytest.raises(ValueError):
        layer(torch.randn((9, 48), device="cuda").half())
    layer.W_down.destroy()
