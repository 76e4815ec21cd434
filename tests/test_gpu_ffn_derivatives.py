"""Derivatives that the feed-forward operators do not have are refused: nothing returns a value whose derivative was dropped."""
import pytest

pytestmark = pytest.mark.gpu


def _weights(kind="float16", f=24, d=64):
    import torch
    return [torch.randn((f, d), device="cuda").to(getattr(torch, kind)) for _ in range(2)]


@pytest.mark.parametrize("t", [1, 20])
def test_forward_mode_is_refused(t):
    """Tensors with a tangent do not say that they require a gradient, and torch.no_grad() does not stop forward mode."""
    import torch
    from torch.autograd import forward_ad
    from paper_2603_08734_amd import ffn, mx4
    wg, wu = _weights()
    W = mx4.quantize(wg)
    x = torch.randn((t, 64), device="cuda").half()
    want = ffn.gated(x, wg, wu)
    with forward_ad.dual_level():
        dual, dual_w = forward_ad.make_dual(x, torch.ones_like(x)), forward_ad.make_dual(wg, torch.ones_like(wg))
        calls = [lambda: ffn.gated(dual, wg, wu), lambda: ffn.gated(x, dual_w, wu), lambda: ffn.gated(x, wu, dual_w), lambda: ffn.gated(dual.view(1, t, 64), wg, wu),
                 lambda: ffn.gated(dual, W, W), lambda: mx4.quantize(dual), lambda: mx4.product(dual, W),
                 lambda: ffn.gated(dual, wg.clone().requires_grad_(), wu)]
        for call in calls:
            with pytest.raises(ValueError, match="forward-mode"):
                call()
            with torch.no_grad(), pytest.raises(ValueError, match="forward-mode"):
                call()
        assert torch.equal(ffn.gated(dual.detach(), wg, wu), want)
        assert torch.equal(ffn.gated(x, wg, wu), want)


def test_a_tangent_of_the_incoming_gradient_is_refused():
    import torch
    from torch.autograd import forward_ad
    from paper_2603_08734_amd import ffn
    wg, wu = _weights()
    x = torch.randn((6, 64), device="cuda").half().requires_grad_()
    with forward_ad.dual_level():
        H = ffn.gated(x, wg, wu)
        dual = forward_ad.make_dual(torch.ones_like(H), torch.ones_like(H))
        with pytest.raises(ValueError, match="forward-mode"):
            torch.autograd.grad(H, x, dual)


@pytest.mark.parametrize("back", ["codes", "plan"])
def test_a_served_layer_refuses_operands_that_want_a_gradient(back):
    import os
    import sys
    import torch
    from torch.autograd import forward_ad
    from paper_2603_08734_amd import ffn, mx4
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    from feed_forward import prune
    wg, wu = _weights(f=64, d=48)
    wd = torch.randn((48, 64), device="cuda").half()
    down = mx4.quantize(wd) if back == "codes" else prune(wd, 0.5, 8)
    x = torch.randn((8, 48), device="cuda").half()
    want = ffn.FeedForward(wg, wu, down)(x)
    for operands in ((x.clone().requires_grad_(), wg, wu), (x, wg.clone().requires_grad_(), wu), (x, wg, wu.clone().requires_grad_())):
        layer = ffn.FeedForward(*operands[1:], down)
        with pytest.raises(ValueError, match="gradient"):
            layer(operands[0])
        with torch.no_grad():
            assert torch.equal(layer(operands[0]), want)
    with forward_ad.dual_level(), pytest.raises(ValueError, match="forward-mode"):
        ffn.FeedForward(wg, wu, down)(forward_ad.make_dual(x, torch.ones_like(x)))
    if back == "plan":
        down.destroy()
