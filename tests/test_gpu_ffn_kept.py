"""What the gated block keeps between its passes: gradients of hidden features beside much larger ones, and of projections outside
binary16's range.

Bounds.  G and U are sums of d exact products in fp32, off by e_G and e_U, at most d * 2^-23 of the sums of absolute values, and the
backward pass has them as they were summed.  |act'| <= 1.13 and |act''| <= 0.8 (silu, gelu); the functions are evaluated to within
2^-20 (1 + |G|) of |G|.  dG and dU are rounded once to the inputs' type (u relative, and half a unit of its smallest number) before a
chain of t additions.  Every term is of the hidden feature itself: nothing of a neighbour's size enters a feature's bound.
"""
import pytest

from test_gpu_ffn import ROUNDING, TINY, _within, act_64

pytestmark = pytest.mark.gpu


def weight_gradients_64(x, wg, wu, dh, act, dtype):
    """(dWg, dWu) and their bounds, in 64 bits."""
    u, (t, d) = ROUNDING[dtype], x.shape
    g, up = x @ wg.T, x @ wu.T
    eg, eu = (d * 2.0 ** -23 * (x.abs() @ w.abs().T) for w in (wg, wu))
    a, da = act_64(act, g)
    ev = 2.0 ** -20 * (1 + g.abs()) ** 2
    slope = 0.8 * eg + ev if act != "relu" else (g.abs() <= eg).double()
    out = []
    for v, e in ((dh * up * da, dh.abs() * (eu * (da.abs() + slope) + up.abs() * slope)), (dh * a, dh.abs() * (1.13 * eg + ev * g.abs()))):
        e = e + u * (v.abs() + e) + TINY[dtype]
        ref, before = v.T @ x, e.T @ x.abs() + t * 2.0 ** -23 * ((v.abs() + e).T @ x.abs())
        out.append((ref, u * ref.abs() + (1 + u) * before + TINY[dtype]))
    return out


def _gradients(x, wg, wu, dh, act):
    import torch
    from paper_2603_08734_amd import ffn
    leaves = [m.clone().requires_grad_() for m in (x, wg, wu)]
    return torch.autograd.grad(ffn.gated(*leaves, act), leaves, dh)


# few rows; tiles; tiles whose sums over k come in parts
@pytest.mark.parametrize("t,d,f", [(5, 64, 70), (60, 72, 130), (130, 1056, 60)])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_features_beside_larger_ones(dtype, act, t, d, f):
    """Of four neighbouring hidden features one is 16, 1000 or 2^15 times as large as another in G, and two others so in U."""
    import torch
    for times in (16.0, 1000.0, 2.0 ** 15):
        print(f"case kept {dtype} {act} t={t} d={d} f={f} times={times}", flush=True)
        rng = torch.Generator(device="cuda").manual_seed(t + d + f)
        kind = getattr(torch, dtype)
        x, wg, wu, dh = (torch.randn(s, generator=rng, device="cuda") for s in ((t, d), (f, d), (f, d), (t, f)))
        wg, wu = wg * d ** -0.5, wu * d ** -0.5
        wg[1::4] *= times ** 0.5
        wg[0::4] *= times ** -0.5
        wu[2::4] *= times ** 0.5
        wu[3::4] *= times ** -0.5
        x, wg, wu, dh = (m.to(kind) for m in (x, wg, wu, dh))
        want = weight_gradients_64(*(m.double() for m in (x, wg, wu, dh)), act, dtype)
        for got, (ref, bound), name in zip(_gradients(x, wg, wu, dh, act)[1:], want, ("dWg", "dWu")):
            _within(got, ref, bound, name)


@pytest.mark.parametrize("t", [3, 40])
def test_projections_outside_the_type(t):
    """binary16: G of 1.3e6 and of 2^-33 with gradients that the type has, beside each other."""
    import torch
    d, f = 64, 24
    x = torch.full((t, d), 200.0, device="cuda")
    x[:, ::2] = 2.0 ** -12
    wg = torch.zeros((f, d), device="cuda")
    wg[0::4, 1::2] = 200.0                   # G = 32 * 200 * 200
    wg[1::4, 0::2] = 2.0 ** -24              # G = 32 * 2^-12 * 2^-24 (binary16's smallest number)
    wu = torch.zeros((f, d), device="cuda")
    wu[:, 0] = 0.5
    dh = torch.full((t, f), 2.0 ** -12, device="cuda")
    dh[:, 1::4] = 2.0 ** 12
    x, wg, wu, dh = (m.half() for m in (x, wg, wu, dh))
    for act in ("silu", "relu"):
        want = weight_gradients_64(*(m.double() for m in (x, wg, wu, dh)), act, "float16")
        for got, (ref, bound), name in zip(_gradients(x, wg, wu, dh, act)[1:], want, ("dWg", "dWu")):
            # finite but for what the formula's own result does not fit into the type
            fits = ref.abs() < 60000
            assert fits.sum() > f * d // 2 and torch.isfinite(got[fits]).all()
            _within(torch.where(fits, got, 0), torch.where(fits, ref, 0), bound, name)
        slope = _gradients(x, wg, wu, dh, "relu")[1]
        assert (slope[1::4, 0] > 0).all()         # a positive G of 2^-31 is positive
