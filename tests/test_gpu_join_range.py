"""Norms and joins at the ends of fp32's range."""
import pytest
import torch

from oracle import edges

pytestmark = pytest.mark.gpu

E, EPS = 2.0 ** -24, 1e-5
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("d", [40, 500, 4100, 8192, 9000, 20000, 40001])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_rows_of_the_largest_numbers(d, dtype, kind):
    """Sums of squares of numbers next to the type's largest.  r is about 2^-128, a subnormal number of fp32 with 2^-149 from one to the next: half a
    step of that is 2^-22 of it.  Half of the signs are either, so differences from the mean stay in range."""
    from paper_2603_08734_amd import residual
    T = TYPES[dtype]
    g = torch.Generator().manual_seed(d)
    sign = 1.0 - 2.0 * (torch.arange(d) % 2)
    x = (sign * (2.0 ** 127 + 2.0 ** 126 * torch.rand(3, d, generator=g))).to(T)
    u = torch.finfo(T).eps / 2
    want = edges.norm(x.double(), kind, None, None, EPS)[0]
    v = x.cuda().requires_grad_()
    y = residual.norm(v, residual.Norm(kind, None, None, EPS))
    s, before = residual.join(torch.zeros_like(v), v, before=residual.Norm(kind, None, None, EPS))
    after = residual.join(torch.zeros_like(v), v, after=residual.Norm(kind, None, None, EPS))
    assert torch.equal(s, v)
    for n in (y, before, after):
        assert ((n.detach().double().cpu() - want).abs() <= (u + 2.0 ** -22 + 200 * E) * (want.abs() + 1)).all()
