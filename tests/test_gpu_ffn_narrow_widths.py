"""Gradients of the gated block where the model's width is one, two or three: operands with k across memory have lines of as many elements
there, and a load of eight elements runs through several of them.  Bounds as in test_gpu_ffn."""
import pytest

from test_gpu_ffn import _inputs, _within, backward_64, forward_64

pytestmark = pytest.mark.gpu
LINES = (33, 34, 38, 65, 70, 97)      # of 32 to a slice: the last slice has 1 to 6


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("d", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("t,f", [(a, b) for a in LINES for b in (LINES[0], a, 300)])
def test_gradients_of_narrow_models(t, d, f, dtype):
    import torch
    from paper_2603_08734_amd import ffn
    for stride in (False, True):
        print(f"case narrow {dtype} t={t} d={d} f={f} stride={stride}", flush=True)
        x, wg, wu, dh = _inputs(t, d, f, dtype, t + d + f, stride)
        x64, wg64, wu64, dh64 = (m.double() for m in (x, wg, wu, dh))
        saved = forward_64(x64, wg64, wu64, "silu", dtype)[2]
        leaves = [m.detach().requires_grad_() for m in (x, wg, wu)]
        grads = torch.autograd.grad(ffn.gated(*leaves, "silu"), leaves, dh)
        for got, (ref, bound), name in zip(grads, backward_64(x64, wg64, wu64, dh64, "silu", dtype, saved), ("dX", "dWg", "dWu")):
            _within(got, ref, bound, name)
