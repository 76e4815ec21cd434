"""The gated feed-forward block on the GPU against 64 bits.

Bounds.  u is the type's unit roundoff (2^-8 for bfloat16, 2^-11 for binary16).  G and U are sums of d exact products in fp32:
off by at most d * 2^-23 of the sums of absolute values, called e_G and e_U.  |act'| <= 1.13 and |act''| <= 0.8 for silu and gelu
(relu has act'' = 0 but for a step at 0, so where |G| <= e_G its slope may be either).  The functions themselves are evaluated in
fp32 to within 2^-20 (1 + |G|) of their result's scale |G|.  So H is off by 1.13 |U| e_G + |act(G)| e_U, that evaluation, and one
rounding.  The gradients see G and U rounded (u |G| + e_G, u |U| + e_U off) and dG, dU are rounded once more before a chain of
f (dX: 2 f) or t (dW) additions.
"""
import numpy as np
import pytest

from test_gpu_mx4 import _device, _weight, decode_64

pytestmark = pytest.mark.gpu
ROUNDING = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float16": 2.0 ** -25, "bfloat16": 2.0 ** -133}


def act_64(name, g):
    """act(g), act'(g) in 64 bits."""
    import torch
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu":
        c = 0.5 * (1 + torch.erf(g / 2 ** 0.5))
        return g * c, c + g * torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5
    return g * (g > 0), (g > 0).double()


def forward_64(x, wg, wu, act, dtype):
    """H, its bound, and what the gradients need."""
    u, d = ROUNDING[dtype], x.shape[1]
    g, up = x @ wg.T, x @ wu.T
    eg, eu = (d * 2.0 ** -23 * (x.abs() @ w.abs().T) for w in (wg, wu))
    a, da = act_64(act, g)
    h = a * up
    ev = 2.0 ** -20 * (1 + g.abs()) * g.abs()
    before = up.abs() * (1.13 * eg + ev) + a.abs() * eu + 1.13 * eg * eu + ev * eu
    return h, u * h.abs() + (1 + u) * before + TINY[dtype], (g, up, eg, eu, a, da)


def backward_64(x, wg, wu, dh, act, dtype, saved):
    """(dX, dWg, dWu) and their bounds."""
    u, (t, d), f = ROUNDING[dtype], x.shape, wg.shape[0]
    g, up, eg, eu, a, da = saved
    dg, du = dh * up * da, dh * a
    rg, ru = u * g.abs() + 2 * eg + TINY[dtype], u * up.abs() + 2 * eu + TINY[dtype]       # how far the kept G and U are off
    ev = 2.0 ** -20 * (1 + g.abs()) ** 2
    slope = rg * 0.8 + ev if act != "relu" else (g.abs() <= rg).double()
    e_dg = dh.abs() * (ru * (da.abs() + slope) + up.abs() * slope)
    e_du = dh.abs() * (1.13 * rg + ev * g.abs())
    e_dg, e_du = (e + u * (v.abs() + e) + TINY[dtype] for e, v in ((e_dg, dg), (e_du, du)))
    out = []
    for ref, err, total, chain in (
            (dg @ wg + du @ wu, e_dg @ wg.abs() + e_du @ wu.abs(), dg.abs() @ wg.abs() + du.abs() @ wu.abs(), 2 * f),
            (dg.T @ x, e_dg.T @ x.abs(), dg.abs().T @ x.abs(), t), (du.T @ x, e_du.T @ x.abs(), du.abs().T @ x.abs(), t)):
        before = err + chain * 2.0 ** -23 * (total + err)
        out.append((ref, u * ref.abs() + (1 + u) * before + TINY[dtype]))
    return out


def _inputs(t, d, f, dtype, seed, stride=False):
    import torch
    rng = np.random.default_rng(seed)
    kind = getattr(torch, dtype)

    def matrix(rows, cols, scale):
        m = _device(rng.normal(size=(rows, cols)) * scale).to(kind)
        if not stride:
            return m
        wide = torch.full((rows, cols + 5), float("nan"), dtype=kind, device="cuda")
        wide[:, 3:cols + 3] = m
        return wide[:, 3:cols + 3]
    return matrix(t, d, 1.0), matrix(f, d, d ** -0.5), matrix(f, d, d ** -0.5), matrix(t, f, 0.3)


def _within(got, ref, bound, what):
    err = (got.double() - ref).abs()
    assert (err <= bound).all(), f"{what}: {err.max().item()} is {((err - bound).max()).item()} over"


SIZES = [(1, 1, 1), (1, 64, 100), (3, 7, 5), (16, 32, 33), (17, 100, 64), (33, 65, 31), (5, 520, 16), (130, 129, 257), (64, 256, 512), (300, 40, 140),
         (1, 1500, 70), (12, 2056, 48)]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("t,d,f", SIZES)
def test_block_and_gradients(t, d, f, act, dtype):
    import torch
    from paper_2603_08734_amd import ffn
    for stride in (False, True):
        print(f"case gated {dtype} {act} t={t} d={d} f={f} stride={stride}", flush=True)
        x, wg, wu, dh = _inputs(t, d, f, dtype, t + d + f, stride)
        x64, wg64, wu64, dh64 = (m.double() for m in (x, wg, wu, dh))
        h, bound, saved = forward_64(x64, wg64, wu64, act, dtype)
        H = ffn.gated(x, wg, wu, act)
        _within(H, h, bound, "H")
        leaves = [m.detach().requires_grad_() for m in (x, wg, wu)]
        H2 = ffn.gated(*leaves, act)
        assert torch.equal(H2.detach(), H)           # keeping G and U changes nothing
        grads = torch.autograd.grad(H2, leaves, dh)
        for got, (ref, bound), name in zip(grads, backward_64(x64, wg64, wu64, dh64, act, dtype, saved), ("dX", "dWg", "dWu")):
            assert got.shape == ref.shape and got.dtype == x.dtype
            _within(got, ref, bound, name)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("t,d,f", [(1, 64, 100), (1, 4096, 96), (7, 100, 33), (8, 31, 64), (16, 512, 130), (17, 1056, 20), (40, 200, 129), (300, 100, 260)])
def test_block_on_weights_in_4_bits(t, d, f, dtype):
    import torch
    from paper_2603_08734_amd import ffn, mx4
    rng = np.random.default_rng(t + d + f)
    # scales near 1 / (4 sqrt(d))
    wg, wu = ((codes, (scales.astype(int) + 5 - d.bit_length() // 2).astype(np.uint8)) for codes, scales in (_weight(rng, f, d) for _ in range(2)))
    Wg, Wu = (mx4.Mx4(*(_device(a) for a in w), d) for w in (wg, wu))
    w64 = [torch.from_numpy(decode_64(*w, d)).cuda() for w in (wg, wu)]
    for stride in (False, True):
        x = _inputs(t, d, f, dtype, d, stride)[0]
        for act in ("silu", "gelu", "relu"):
            print(f"case gated 4 bits {dtype} {act} t={t} d={d} f={f} stride={stride}", flush=True)
            h, bound, _ = forward_64(x.double(), *w64, act, dtype)
            _within(ffn.gated(x, Wg, Wu, act), h, bound, act)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradients_against_differences(act):
    """Central differences of the block in 64 bits along random directions, at a point the type holds exactly: the gradient's
    projection differs by the gradients' own bounds and by the differences' third-order term, below 1e-6 of the terms at a
    step of 1e-4."""
    import torch
    from paper_2603_08734_amd import ffn
    t, d, f = 9, 48, 40
    x, wg, wu, dh = _inputs(t, d, f, "float16", 3)
    leaves = [m.detach().requires_grad_() for m in (x, wg, wu)]
    grads = torch.autograd.grad(ffn.gated(*leaves, act), leaves, dh)
    p = [m.double() for m in (x, wg, wu)]
    bounds = [b for _, b in backward_64(*p, dh.double(), act, "float16", forward_64(*p, act, "float16")[2])]
    g = torch.Generator(device="cuda").manual_seed(1)
    for i in range(3):
        v = torch.randn(p[i].shape, generator=g, device="cuda", dtype=torch.float64)
        step, ends = 1e-4, []
        for s in (step, -step):
            q = list(p)
            q[i] = p[i] + s * v
            a, _ = act_64(act, q[0] @ q[1].T)
            ends.append((a * (q[0] @ q[2].T) * dh.double()).sum())
        want = (ends[0] - ends[1]) / (2 * step)
        got = (grads[i].double() * v).sum()
        assert (got - want).abs() <= (bounds[i] * v.abs()).sum() + 1e-6 * (grads[i].double() * v).abs().sum()


@pytest.mark.parametrize("t", [3, 40, 300])
def test_small_numbers_beside_large_ones(t):
    """The forward pass keeps four numbers with one exponent.  A positive one stays positive however large its neighbours are (relu's
    slope), an infinity leaves its neighbours finite, and what is kept is off by 2^-13 of the largest of the four at most."""
    import torch
    from paper_2603_08734_amd import ffn
    d, f = 64, 24
    x = torch.full((t, d), 0.125, device="cuda").bfloat16()
    wg = torch.full((f, d), 100.0, device="cuda").bfloat16()
    wg[1::4], wg[2::4] = 2.0 ** -30, -(2.0 ** -30)
    wu = torch.full((f, d), 0.5, device="cuda").bfloat16()
    dh = torch.ones((t, f), device="cuda").bfloat16()
    leaves = [m.clone().requires_grad_() for m in (x, wg, wu)]
    _, dwg, dwu = torch.autograd.grad(ffn.gated(*leaves, "relu"), leaves, dh)
    want = torch.full((f,), t * 4.0 * 0.125, device="cuda")      # sum over t of dH U x, U = 64 * 0.125 * 0.5
    want[2::4] = 0
    assert ((dwg[:, 0].float() - want).abs() <= 2.0 ** -8 * want).all()
    small = t * 0.125 * 64 * 0.125 * 2.0 ** -30                  # sum over t of dH G x
    assert ((dwu[1::4].float() - small).abs() <= 2.0 ** -8 * small + t * 0.125 * 800 * 2.0 ** -13).all() and not dwu[2::4].any()
    wg[0, 0] = float("inf")                                      # G of column 0
    leaves = [m.clone().requires_grad_() for m in (x, wg, wu)]
    dx, dwg, dwu = torch.autograd.grad(ffn.gated(*leaves, "silu"), leaves, dh)
    assert torch.isfinite(dwg[1:]).all() and torch.isfinite(dwu[1:]).all() and not torch.isfinite(dwu[0]).any()


def test_some_gradients_only():
    import torch
    from paper_2603_08734_amd import ffn
    x, wg, wu, dh = _inputs(70, 50, 60, "bfloat16", 1)
    leaves = [m.detach().requires_grad_() for m in (x, wg, wu)]
    whole = torch.autograd.grad(ffn.gated(*leaves), leaves, dh)
    for pick in ((0,), (1,), (2,), (0, 2), (1, 2)):
        part = [m.detach().requires_grad_(i in pick) for i, m in enumerate((x, wg, wu))]
        got = torch.autograd.grad(ffn.gated(*part), [part[i] for i in pick], dh)
        for i, a in zip(pick, got):
            assert torch.equal(a, whole[i])


def test_shapes_and_views():
    import torch
    from paper_2603_08734_amd import ffn
    x, wg, wu, dh = _inputs(24, 40, 56, "float16", 2)
    want = ffn.gated(x, wg, wu)
    assert torch.equal(ffn.gated(x.view(2, 3, 4, 40), wg, wu), want.view(2, 3, 4, 56))
    assert torch.equal(ffn.gated(x[5], wg, wu).view(1, -1), ffn.gated(x[5:6], wg, wu))
    assert torch.equal(ffn.gated(x, wg.t().contiguous().t(), wu), want)              # a transposed weight
    assert torch.equal(ffn.gated(x[:, None].expand(24, 3, 40), wg, wu)[:, 1], want)  # repeated rows
    leaf = wg[0].clone().requires_grad_()                                            # a broadcast weight: its gradient adds up
    broad = leaf.expand(56, 40)
    (got,) = torch.autograd.grad(ffn.gated(x, broad, wu), leaf, dh)
    full = broad.detach().clone().requires_grad_()
    (rows,) = torch.autograd.grad(ffn.gated(x, full, wu), full, dh)
    assert torch.equal(got, rows.sum(0)) or (got - rows.float().sum(0)).abs().max() <= 2.0 ** -10 * rows.float().abs().sum(0).max()


def test_empty_sizes():
    import torch
    from paper_2603_08734_amd import ffn, mx4
    for t, d, f in ((0, 16, 8), (4, 0, 8), (4, 16, 0)):
        leaves = [torch.randn(s, device="cuda").half().requires_grad_() for s in ((t, d), (f, d), (f, d))]
        H = ffn.gated(*leaves)
        assert H.shape == (t, f) and not H.any()
        for g, leaf in zip(torch.autograd.grad(H, leaves, torch.ones_like(H)), leaves):
            assert g.shape == leaf.shape and not g.any()
    W = mx4.quantize(torch.randn((8, 40), device="cuda"))
    assert ffn.gated(torch.empty((2, 0, 40), dtype=torch.float16, device="cuda"), W, W).shape == (2, 0, 8)


@pytest.mark.parametrize("t", [1, 20, 150])
def test_a_nan_or_infinity_stays_in_its_rows(t):
    import torch
    from paper_2603_08734_amd import ffn
    x, wg, wu, _ = _inputs(t, 72, 90, "bfloat16", 4)
    x[t - 1, 70] = float("nan")
    wu[33, 71] = float("inf")
    H = ffn.gated(x, wg, wu)
    want = torch.ones(H.shape, dtype=torch.bool, device="cuda")
    want[t - 1] = False
    want[:, 33] = False
    assert torch.equal(torch.isfinite(H), want)


def test_the_same_twice_and_on_another_stream():
    import torch
    from paper_2603_08734_amd import ffn
    for t, d, f in ((1, 4096, 64), (200, 300, 400), (700, 64, 72)):
        x, wg, wu, dh = _inputs(t, d, f, "bfloat16", 7)
        leaves = [m.detach().requires_grad_() for m in (x, wg, wu)]

        def step():
            H = ffn.gated(*leaves)
            return (H.detach(), *torch.autograd.grad(H, leaves, dh))
        first = step()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            second = step()
        torch.cuda.current_stream().wait_stream(side)
        for a, b in zip(first, second):
            assert torch.equal(a, b)


def test_second_derivatives_are_refused():
    import torch
    from paper_2603_08734_amd import ffn
    leaves = [m.detach().requires_grad_() for m in _inputs(4, 16, 8, "float16", 1)[:3]]
    (g,) = torch.autograd.grad(ffn.gated(*leaves).float().sum(), leaves[0], create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


def test_calls_refuse():
    import torch
    from paper_2603_08734_amd import ffn, mx4
    x, wg, wu, _ = _inputs(4, 64, 8, "float16", 1)
    W = mx4.quantize(wg)
    for args in ((x.float(), wg, wu), (x, wg.bfloat16(), wu), (x, wg, wu[:7]), (x[:, :63], wg, wu), (x, wg, W), (x, wg.cpu(), wu), (x, wg, wu, "tanh"),
                 (x.clone().requires_grad_(), W, W), (3.0, wg, wu)):
        with pytest.raises((TypeError, ValueError)):
            ffn.gated(*args)
