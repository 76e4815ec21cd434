"""Low-rank adapters: infinities come out where the formula has them, in both 16-bit types and all passes, and NaN only where it has none.

Expected values are the formula's in 64 bits.  The numbers are small integers, so every sum is exact in fp32 and finite results are rounded once.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = [torch.float16, torch.bfloat16]
INF = float("inf")


def integers(g, *shape):
    v = torch.randint(1, 4, shape, generator=g) * (2 * torch.randint(0, 2, shape, generator=g) - 1)
    return v.double()


def formula(y, x, a, b, dout, index, scale):
    """out, dX, dA, dB; every product by itself, so that zeros times infinities are NaN where the formula has them."""
    n = a.shape[0]
    out, dx, da, db = y.clone(), torch.zeros_like(x), torch.zeros_like(a), torch.zeros_like(b)
    for i in range(n):
        rows = torch.nonzero(index == i).squeeze(1)
        if not len(rows):
            continue
        xi, gi = x[rows], dout[rows]
        h = (xi[:, None, :] * a[i][None]).sum(2)
        dh = (gi[:, None, :] * b[i][None]).sum(2)
        out[rows] += scale[i] * (h[:, :, None] * b[i][None]).sum(1)
        dx[rows] = scale[i] * (dh[:, :, None] * a[i][None]).sum(1)
        da[i] = scale[i] * (dh[:, :, None] * xi[:, None, :]).sum(0)
        db[i] = scale[i] * (h[:, :, None] * gi[:, None, :]).sum(0)
    return out, dx, da, db


def same(got, want):
    want = want.to(got.dtype).double()
    got = got.detach().double().cpu()
    ok = (got == want) | (got.isnan() & want.isnan())
    assert got.shape == want.shape and bool(ok.all()), f"{int((~ok).sum())} of {ok.numel()} differ, first at {torch.nonzero(~ok)[0].tolist()}: {got[~ok][0]} for {want[~ok][0]}"


def check(dtype, t, r, where, n=2, scale=None, k=24, m=136):
    from paper_2603_08734_amd import adapters
    g = torch.Generator().manual_seed(t + r)
    v = dict(y=integers(g, t, m), x=integers(g, t, k), a=integers(g, n, r, k), b=integers(g, n, r, m), dout=integers(g, t, m))
    index = torch.arange(t) % 2
    scale = torch.ones(n) if scale is None else scale
    where(v)
    want = formula(*v.values(), index, scale.double())
    cuda = {name: c.to(dtype).cuda().requires_grad_(name != "dout") for name, c in v.items()}
    args = [cuda[name] for name in ("y", "x", "a", "b")]
    out = adapters.add(*args, index.cuda(), scale.cuda())
    same(out, want[0])
    with torch.no_grad():
        same(adapters.add(*args, index.cuda(), scale.cuda()), want[0])
    for got, value in zip(torch.autograd.grad(out, args[1:], cuda["dout"]), want[1:]):
        same(got, value)


def put(name, *at, value=INF):
    def where(v):
        v[name][at] = value
    return where


PLACES = {"x": put("x", 2, 3), "x_minus": put("x", 1, 0, value=-INF), "a": put("a", 0, 0, 5), "b": put("b", 1, 0, 100), "b_minus": put("b", 0, 0, 7, value=-INF),
          "dout": put("dout", 2, 90), "dout_minus": put("dout", 0, 3, value=-INF), "nan": put("x", 1, 1, value=float("nan"))}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t", [3, 290])
@pytest.mark.parametrize("r", [1, 2, 17, 40])
@pytest.mark.parametrize("place", list(PLACES))
def test_infinities_where_the_formula_has_them(dtype, t, r, place):
    check(dtype, t, r, PLACES[place])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("t", [3, 290])
def test_zeros_times_infinities_and_infinities_of_both_signs(dtype, t):
    def where(v):
        v["x"][0, 2], v["x"][2, 2], v["x"][2, 4] = INF, INF, -INF
        v["a"][0, 0, 2], v["a"][0, 1, 2], v["a"][0, :, 4] = 1, 0, -1
        v["b"][0, :, 5] = 0
        v["b"][0, 0, 9] = -INF
        v["dout"][1, 3] = INF
    check(dtype, t, 3, where)
