"""Low-rank adapters: scales of adapters whose sums over tokens are empty, wholly or in some of their parts."""
import pytest
import torch

from test_gpu_adapters_infinities import INF, TYPES, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", [3, 290, 5000])
@pytest.mark.parametrize("value", [INF, float("nan")])
def test_scales_of_adapters_that_no_token_has(t, value):
    """A slot that nothing has filled yet: its gradients are sums over no tokens."""
    for dtype in TYPES:
        check(dtype, t, 2, lambda v: None, n=4, scale=torch.tensor([1.0, 2.0, value, -value]), k=8 if t > 1000 else 24, m=8 if t > 1000 else 136)


def test_infinite_scale_of_an_adapter_with_few_tokens():
    """Its tokens are fewer than the parts that the sum over tokens has."""
    from paper_2603_08734_amd import adapters
    t = 4096
    x = torch.ones(t, 64, device="cuda").bfloat16()
    y = torch.zeros(t, 64, device="cuda").bfloat16()
    index = torch.zeros(t, dtype=torch.int64, device="cuda")
    index[77] = 1
    a, b = (torch.ones(2, 4, 64, device="cuda").bfloat16().requires_grad_() for _ in range(2))
    out = adapters.add(y, x, a, b, index, torch.tensor([1.0, INF], device="cuda"))
    for g in torch.autograd.grad(out, (a, b), torch.ones_like(out)):
        assert torch.equal(g[1], torch.full_like(g[1], INF)) and g[0].isfinite().all()
