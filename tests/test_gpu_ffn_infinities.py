"""relu of minus infinity is zero, in every kernel that ends a gated block, and so is what it brings into the gradients."""
import pytest

pytestmark = pytest.mark.gpu


# few rows; a tile; parts of k that are joined
@pytest.mark.parametrize("t,d", [(1, 64), (16, 64), (40, 64), (130, 1056)])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_relu_of_minus_infinity(dtype, t, d):
    import torch
    from paper_2603_08734_amd import ffn
    f = 24
    x = torch.ones((t, d), device="cuda", dtype=getattr(torch, dtype))
    wg, wu = torch.ones((f, d), device="cuda", dtype=x.dtype), torch.full((f, d), 2.0 ** -10, device="cuda", dtype=x.dtype)
    wg[5, 3] = -float("inf")
    wg[6, 3] = float("nan")
    wg[7, 3] = float("inf")
    wg[8] = -1
    leaves = [m.clone().requires_grad_() for m in (x, wg, wu)]
    H = ffn.gated(*leaves, "relu")
    want = torch.full((f,), 2.0 ** -10 * d * d, device="cuda")       # exact, then rounded once
    want[5], want[6], want[7], want[8] = 0, float("nan"), float("inf"), 0
    want = want.to(x.dtype)
    assert torch.equal(torch.nan_to_num(H.detach(), nan=77.0), torch.nan_to_num(want.expand(t, f), nan=77.0))
    _, dwg, dwu = torch.autograd.grad(H, leaves, torch.ones_like(H))
    rows = torch.tensor([5, 8], device="cuda")
    assert not dwg[rows].any() and not dwu[rows].any()
    assert dwu[6].isnan().all() and (dwu[7] == float("inf")).all()


@pytest.mark.parametrize("t", [1, 12, 40])
def test_relu_of_minus_infinity_on_weights_in_4_bits(t):
    import torch
    from paper_2603_08734_amd import ffn, mx4
    w = torch.ones((24, 64), device="cuda")
    w[5] = -1
    W = mx4.quantize(w)
    x = torch.ones((t, 64), device="cuda").bfloat16()
    x[:, 2] = float("inf")
    H = ffn.gated(x, W, mx4.quantize(torch.ones_like(w)), "relu")
    # 0 * infinity: of the formula itself
    assert H[:, 5].isnan().all() and (torch.cat([H[:, :5], H[:, 6:]], dim=1) == float("inf")).all()
    x[:, 2] = 1
    W.scales[5] = 254                     # -4 * 2^127 is below fp32's range
    assert not ffn.gated(x, W, mx4.quantize(torch.ones_like(w)), "relu")[:, 5].any()
