"""Rows that lie far apart in memory: the last token of every sequence, a slice of a large buffer.  The library's products take rows up to
RSH_FFN_MAX_WIDTH = 2^21 elements apart; beyond, rows are copied, and results are those of the copied rows bit for bit."""
import pytest

pytestmark = pytest.mark.gpu
FAR = (1 << 21) + 8


def _far(m, ld=FAR):
    """The same matrix with rows ld elements apart."""
    import torch
    wide = torch.empty((m.shape[0], ld), dtype=m.dtype, device=m.device)
    wide[:, 3:3 + m.shape[1]] = m
    out = wide[:, 3:3 + m.shape[1]]
    assert out.stride(0) == ld
    return out


@pytest.mark.parametrize("t", [2, 5, 40])
@pytest.mark.parametrize("ld", [1 << 21, FAR])
def test_activations_with_rows_far_apart(t, ld):
    import torch
    from paper_2603_08734_amd import ffn, mx4
    x = torch.randn((t, 72), device="cuda").half()
    wg, wu = (torch.randn((24, 72), device="cuda").half() for _ in range(2))
    W = mx4.quantize(wg)
    far = _far(x, ld)
    for call in (lambda m: mx4.product(m, W), lambda m: ffn.gated(m, wg, wu), lambda m: ffn.gated(m, W, W), lambda m: mx4.quantize(m).dequantize()):
        assert torch.equal(call(far), call(x))


@pytest.mark.parametrize("t", [3, 40])
def test_weights_and_gradients_with_rows_far_apart(t):
    import torch
    from paper_2603_08734_amd import ffn
    x = torch.randn((t, 40), device="cuda").half()
    wg, wu = (torch.randn((24, 40), device="cuda").half() for _ in range(2))
    dh = torch.randn((t, 24), device="cuda").half()

    def gradients(x, wg, wu, dh):
        leaves = [m.detach().requires_grad_() for m in (x, wg, wu)]
        H = ffn.gated(*leaves)
        return (H.detach(), *torch.autograd.grad(H, leaves, dh))
    want = gradients(x, wg, wu, dh)
    for operands in ((_far(x), wg, wu, dh), (x, _far(wg), wu, dh), (x, _far(wg), _far(wu), dh), (x, wg, wu, _far(dh))):
        for a, b in zip(gradients(*operands), want):
            assert torch.equal(a, b)
