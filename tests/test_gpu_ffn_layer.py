"""The served layer against 64 bits, exactly: operands of small integers, so that the block's results are integers up to 256, which both types have, and
sums of the projection back are exact in fp32; what is left is one rounding."""
import pytest

from test_gpu_ffn_tiles import _equal, _sparse

pytestmark = pytest.mark.gpu


def _operands(t, d, f, kind):
    """X, gate, up and down: 16 entries of -1 and 1 in a weight's row, on average, and half of X not zero."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(t + d + f)
    x, wg, wu = _sparse(g, t, d, 0.5, kind), _sparse(g, f, d, min(1.0, 16 / d), kind), _sparse(g, f, d, min(1.0, 16 / d), kind)
    wd = _sparse(g, d, f, 0.25, kind)
    h = torch.relu(x.double() @ wg.double().t()) * (x.double() @ wu.double().t())
    assert h.abs().max() <= 256
    return x, wg, wu, wd, h @ wd.double().t()


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("t,d,f", [(1, 64, 100), (7, 100, 90), (16, 512, 1000), (40, 96, 257), (300, 264, 520)])
def test_a_projection_back_in_4_bits(t, d, f, four, dtype):
    import torch
    from paper_2603_08734_amd import ffn, mx4
    x, wg, wu, wd, want = _operands(t, d, f, getattr(torch, dtype))
    if four:
        wg, wu = mx4.quantize(wg), mx4.quantize(wu)
    Y = ffn.FeedForward(wg, wu, mx4.quantize(wd), "relu")(x)
    assert Y.shape == (t, d) and Y.dtype == x.dtype
    _equal(Y, want, "Y")


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("t,d,f", [(1, 64, 100), (8, 100, 90), (40, 96, 257), (256, 264, 520)])
def test_a_pruned_projection_back(t, d, f, four):
    import torch
    from paper_2603_08734_amd import Plan, ffn, mx4
    x, wg, wu, wd, want = _operands(t, d, f, torch.float16)
    csr = wd.cpu()
    rows, cols = torch.nonzero(csr, as_tuple=True)
    row_ptr = torch.zeros(d + 1, dtype=torch.int64)
    row_ptr[1:] = torch.bincount(rows, minlength=d).cumsum(0)
    plan = Plan(row_ptr.numpy(), cols.int().numpy(), csr[rows, cols].numpy(), f, t)
    if four:
        wg, wu = mx4.quantize(wg), mx4.quantize(wu)
    Y = ffn.FeedForward(wg, wu, plan, "relu")(x)
    assert Y.shape == (t, d) and Y.dtype == torch.float16
    _equal(Y, want, "Y")
    plan.destroy()
