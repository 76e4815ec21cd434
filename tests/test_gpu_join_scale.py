"""Joins whose scale and dropout together are at the end of fp32's range."""
import pytest
import torch

from oracle import edges

pytestmark = pytest.mark.gpu


def test_scales_that_leave_the_range_with_dropout():
    """The factor of what is kept is scale / (1 - p), a number of fp32: refused where it is not one.  With everything dropped there is no factor."""
    from paper_2603_08734_amd import dropout, residual
    x = torch.ones(3, 64, device="cuda")
    gate = torch.ones(64, device="cuda", requires_grad=True)
    large = 2.0 ** 126
    for p in (0.9, 1 - 2.0 ** -16):
        with pytest.raises(ValueError, match="scale"):
            residual.join(x, x, scale=large, drop=dropout.Drop(p, 1))
    tiny = torch.full_like(x, 2.0 ** -120)
    s = residual.join(torch.zeros_like(x), tiny, scale=large, drop=dropout.Drop(0.5, 1))
    assert torch.equal(s.cpu(), torch.where(edges.kept(3, 64, 0.5, 1, 0)[0], 128.0, 0.0))
    s = residual.join(x, x, gate=gate, scale=large, drop=dropout.Drop(1.0, 1))
    assert torch.equal(s, x) and not torch.autograd.grad(s, gate, torch.ones_like(s))[0].any()
