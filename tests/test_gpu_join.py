"""Norms, joins and their gradients against the formulas in 64 bits.

Bounds.  E = 2^-24 is half a step of fp32, u half a step of the result's type.  A sum over a row of d terms is made of at most
DEPTH(d) = 8 (d / 8192 + 1) + 26 additions one after the other (a lane's, those across lanes, those across waves), so a mean is off by at most
DEPTH E times the mean of the terms' magnitudes, r by half of that relative, and 16 more roundings cover what a single element goes through.
With K = DEPTH + 16 and e(.) for the error of .:
  N(x)   e <= E K (|xh w| + r |w| mean|x| + |b|) + e(x) part: r |w| (e(x) + mean e(x) + |xh| mean(|xh| e(x)))
  S      e <= E 8 (|X| + |scale gate D|) + |scale gate| e(D)
  both once more rounded: + u |value|.
Gradients use xh of the sum formed again in fp32: e(xh) = r 2 E K (|S| + mean|S|) + E K |xh| + what e(S) brings.
  N'(g)  e <= r [E K (|gw| + mean|gw| + |xh| mean|gw xh|) + e(xh) mean|gw xh| + (|xh| + e(xh)) mean(|gw| e(xh)) + w-weighted errors of g]:
           (xh + a) (m + b) - xh m = a m + xh b + a b, and the last counts where a row is so even that the sums' rounding is all of its spread
  vectors  e <= sum over rows of (|g| e(xh) + |xh| e(g)) + E (T + 64) sum |terms|, T rows one after the other: at most t.
Results in binary16 may be subnormal: + 2^-25.  The tests evaluate these with the reference's own 64-bit magnitudes.
"""
import pytest
import torch

from oracle import edges

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
EPS = 1e-5
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def least(dtype):
    return 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134


def close(got, want, bound, dtype, what):
    """bound: of the error before the last rounding."""
    got = got.detach().double().cpu()
    u = half_step(dtype)
    off = (got - want).abs() - (bound + u * (want.abs() + bound) + least(dtype))
    assert got.shape == want.shape and bool((off <= 0).all()), f"{what}: {(off.max()).item()} beyond the bound at {off.argmax().item()}, sizes {tuple(want.shape)}"


def mean(v):
    return v.mean(dim=-1, keepdim=True)


def build(t, d, kind, dtype, params, after, before, gate, p, seed=0, bias=True, weight=True):
    g = torch.Generator().manual_seed(seed * 7919 + t * 31 + d)

    def normal(*shape, scale=1.0, to=dtype):
        return (torch.randn(shape, generator=g) * scale).to(to)
    m = {"x": normal(t, d) + 0.25, "b": normal(t, d, scale=2.0), "ds": normal(t, d, scale=0.1), "dy": normal(t, d, scale=0.1)}
    for name, there in (("after", after), ("before", before)):
        if there and weight:
            m["w_" + name] = normal(d, scale=0.3, to=params) + 1
        if there and bias:
            m["b_" + name] = normal(d, scale=0.3, to=params)
    if gate != "none":
        m["gate"] = normal(*((d,) if gate == "vector" else (t, d)), to=params)
    return m


LEAVES = ["x", "b", "gate", "w_after", "b_after", "w_before", "b_before"]


def library(m, kind, after, before, scale, drop, device="cuda", alone=False, grads=True, leaves=None):
    from paper_2603_08734_amd import residual
    v = {n: x.to(device) for n, x in m.items()}
    names = [n for n in (leaves or LEAVES) if n in v and not (alone and n in ("b", "gate", "w_after", "b_after"))]
    if grads:
        for n in names:
            v[n] = v[n].requires_grad_()
    n1 = residual.Norm(kind, v.get("w_after"), v.get("b_after"), EPS) if after else None
    n2 = residual.Norm(kind, v.get("w_before"), v.get("b_before"), EPS) if before else None
    out = {}
    if alone:
        out["Y"] = residual.norm(v["x"], n2)
    else:
        r = residual.join(v["x"], v["b"], after=n1, gate=v.get("gate"), scale=scale, drop=drop, before=n2)
        out["S"] = r[0] if before else r
        if before:
            out["Y"] = r[1]
    if grads:
        seeds = {"S": v["ds"], "Y": v["dy"]}
        for n, g in zip(names, torch.autograd.grad(list(out.values()), [v[n] for n in names], [seeds[o] for o in out])):
            out["d" + n] = g
    return out


def reference(m, kind, after, before, scale, drop, dtype, alone=False, grads=True, t_chain=None):
    """{name: (value, bound)}"""
    v = {n: x.double() for n, x in m.items()}
    t, d = v["x"].shape
    K = 8 * (d / 8192 + 1) + 26 + 16
    names = [n for n in LEAVES if n in v and not (alone and n in ("b", "gate", "w_after", "b_after"))]
    for n in names:
        v[n].requires_grad_()
    w1, c1, w2, c2 = v.get("w_after"), v.get("b_after"), v.get("w_before"), v.get("b_before")
    gate = v.get("gate")
    zero = torch.zeros((), dtype=torch.float64)
    if alone:
        y, sh, sr = edges.norm(v["x"], kind, w2, c2, EPS)
        r = {"S": v["x"], "Y": y, "Sh": sh, "Sr": sr}
    else:
        r = edges.join(v["x"], v["b"], (kind, w1, c1, EPS) if after else None, gate, scale, drop, (kind, w2, c2, EPS) if before else None)
    found = {}
    if grads:
        outs = [r[o] for o in ("S", "Y") if o in r and not (alone and o == "S")]
        seeds = [{"S": v["ds"], "Y": v["dy"]}[o] for o in ("S", "Y") if o in r and not (alone and o == "S")]
        found = dict(zip(names, torch.autograd.grad(outs, [v[n] for n in names], seeds)))
    with torch.no_grad():
        a = lambda q: zero if q is None else q.abs()        # noqa: E731
        one = torch.ones((), dtype=torch.float64)
        W1, W2 = one if w1 is None else w1.abs(), one if w2 is None else w2.abs()
        out, eS = {}, torch.zeros_like(v["x"])
        if not alone:
            eD = zero
            if after:
                eD = E * K * (r["bh"].abs() * W1 + r["br"] * W1 * mean(v["b"].abs()) + a(c1))
            factor = abs(scale) * (one if gate is None else gate.abs())
            keep = one if drop is None else torch.where(drop[0], drop[1], 0.0)
            eS = 8 * E * (v["x"].abs() + factor * r["D"].abs()) + factor * keep * eD
            out["S"] = (r["S"], eS)
        if before:
            Sh, Sr = r["Sh"].abs(), r["Sr"]
            eY = E * K * (Sh * W2 + Sr * W2 * mean(r["S"].abs()) + a(c2)) + Sr * W2 * (eS + mean(eS) + Sh * mean(Sh * eS))
            out["Y"] = (r["Y"], eY)
        if grads:
            chain = E * (t + 64)
            eds = zero
            ds = v["ds"].abs() if not alone else zero
            if before:
                g = v["dy"].abs() * W2
                S = r["S"].abs()
                exh = Sr * 2 * E * K * (S + mean(S)) + E * K * Sh + Sr * (eS + mean(eS) + Sh * mean(Sh * eS))
                back = g + mean(g) + Sh * mean(g * Sh)
                eds = Sr * (E * K * back + exh * mean(g * Sh) + (Sh + exh) * mean(g * exh)) + E * K * Sr * back + Sr * back * mean(Sh * eS) * Sr
                ds = ds + Sr * back
                if w2 is not None:
                    out["dw_before"] = (found["w_before"], (v["dy"].abs() * exh).sum(0) + chain * (v["dy"].abs() * Sh).sum(0))
                if c2 is not None:
                    out["db_before"] = (found["b_before"], chain * v["dy"].abs().sum(0))
            eds = eds + 4 * E * ds
            out["dx"] = (found["x"], eds)
            if not alone:
                f = abs(scale) * keep * (1 + 4 * E)
                if gate is not None:
                    n = r["n"].abs()
                    each = f * (eds * n + ds * (eD + 8 * E * n))
                    if gate.dim() == 1:
                        each = each.sum(0) + chain * (f * ds * n).sum(0)
                    out["dgate"] = (found["gate"], each)
                    f = f * gate.abs()
                gb, egb = f * ds, f * (eds + 8 * E * ds)
                if after:
                    bh, br = r["bh"].abs(), r["br"]
                    B = v["b"].abs()
                    ebh = br * 2 * E * K * (B + mean(B)) + E * K * bh
                    if w1 is not None:
                        out["dw_after"] = (found["w_after"], (gb * ebh + egb * bh).sum(0) + chain * (gb * bh).sum(0))
                    if c1 is not None:
                        out["db_after"] = (found["b_after"], egb.sum(0) + chain * gb.sum(0))
                    g, eg = gb * W1, (egb + 4 * E * gb) * W1
                    back = g + mean(g) + bh * mean(g * bh)
                    egb = br * (2 * E * K * back + eg + mean(eg) + bh * mean(eg * bh) + ebh * mean(g * bh) + (bh + ebh) * mean(g * ebh))
                out["db"] = (found["b"], egb)
    return {n: (x.detach(), torch.as_tensor(b).expand_as(x)) for n, (x, b) in out.items()}


def check(t, d, kind, dtype, params="fp32", after=True, before=True, gate="vector", p=0.0, alone=False, grads=True, bias=True, weight=True, m=None):
    from paper_2603_08734_amd import dropout
    T, P = TYPES[dtype], TYPES[params]
    m = m or build(t, d, kind, T, P, after, before, gate, p, bias=bias, weight=weight)
    seed, offset = 0x0123456789ABCDEF + d, 77
    drop = dropout.Drop(p, seed, offset) if p else None
    got = library(m, kind, after, before, 0.75, drop, alone=alone, grads=grads)
    want = reference(m, kind, after, before, 0.75, edges.kept(t, d, p, seed, offset) if p else None, T, alone=alone, grads=grads)
    assert set(got) == set(want)
    for name, (value, bound) in want.items():
        of = name[1:] if name[0] == "d" else name
        close(got[name], value, bound, m[of].dtype if of in m and of not in ("x", "b") else T, f"{name} {kind} {dtype}")


# every team and the lengths around its end, rows of odd lengths, rows beyond registers
WIDTHS = [1, 2, 7, 8, 9, 63, 64, 65, 100, 128, 129, 255, 257, 500, 513, 1000, 1025, 2049, 4100, 8191, 8192, 8193, 16384, 16391, 40001]


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype", list(TYPES))
def test_whole_join_of_every_width(d, dtype):
    check(5, d, "layer" if d % 2 else "rms", dtype, p=0.1)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("after", [False, True])
@pytest.mark.parametrize("before", [False, True])
@pytest.mark.parametrize("gate", ["none", "vector", "full"])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_every_form(kind, after, before, gate, p):
    check(7, 77, kind, "fp32", after=after, before=before, gate=gate, p=p)
    check(3, 1032, kind, "bf16", params="bf16", after=after, before=before, gate=gate, p=p)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("d", [1, 40, 64, 300, 4096, 9000])
@pytest.mark.parametrize("dtype,params", [("fp32", "fp32"), ("fp16", "fp32"), ("bf16", "bf16"), ("fp16", "fp16")])
def test_norms_alone(kind, d, dtype, params):
    check(6, d, kind, dtype, params=params, alone=True, after=False, gate="none")


@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("d", [61, 2048, 10000])
def test_parameters_that_are_not_there(weight, bias, d):
    for kind in ("rms", "layer"):
        check(4, d, kind, "fp32", weight=weight, bias=bias, gate="none")
        check(4, d, kind, "fp32", weight=weight, bias=bias, gate="none", alone=True, after=False)


@pytest.mark.parametrize("t", [1, 2, 31, 32, 33, 257, 3000])
@pytest.mark.parametrize("d", [24, 200, 1000])
def test_numbers_of_rows(t, d):
    """More rows than workgroups, and teams without a row."""
    check(t, d, "layer", "fp16", p=0.2)


def test_many_rows_of_every_kind():
    check(70001, 8, "rms", "fp32", gate="none")
    check(1300, 8192, "rms", "bf16", p=0.1)
    check(300, 8200, "layer", "bf16", p=0.1)


def test_results_do_not_change_from_call_to_call():
    m = build(900, 1000, "layer", torch.bfloat16, torch.float32, True, True, "vector", 0.1)
    from paper_2603_08734_amd import dropout
    one = library(m, "layer", True, True, 0.5, dropout.Drop(0.1, 3))
    for _ in range(3):
        two = library(m, "layer", True, True, 0.5, dropout.Drop(0.1, 3))
        assert all(torch.equal(one[n], two[n]) for n in one)


def test_rows_with_strides_and_any_alignment():
    """Rows cut out of wider ones, at every offset, transposed and broadcast operands."""
    from paper_2603_08734_amd import residual
    for dtype in TYPES.values():
        big = torch.randn(9, 700, device="cuda").to(dtype)
        other = torch.randn(9, 700, device="cuda").to(dtype)
        w = torch.rand(700, device="cuda") + 0.5
        for at, d in ((0, 64), (1, 64), (3, 131), (5, 520)):
            x, b = big[:, at:at + d], other[:, at + 2:at + 2 + d]
            n = residual.Norm("layer", w[at:at + d], None, EPS)
            plain = residual.join(x.contiguous(), b.contiguous(), after=n, before=n)
            for got, want in zip(residual.join(x, b, after=n, before=n), plain):
                assert torch.equal(got, want)
            assert torch.equal(residual.norm(x[::2], n), residual.norm(x[::2].contiguous(), n))
        x = torch.randn(40, 9, device="cuda").to(dtype).t()
        n = residual.Norm("rms", None, None, EPS)
        assert torch.equal(residual.norm(x, n), residual.norm(x.contiguous(), n))
        row = torch.randn(1, 40, device="cuda").to(dtype).requires_grad_()
        s = residual.join(x, row.expand(9, 40))
        assert torch.equal(s, residual.join(x, row.detach().expand(9, 40).contiguous()))
        (g,) = torch.autograd.grad(s, row, torch.ones_like(s))
        assert torch.equal(g, torch.full_like(row, 9.0))


def test_gradients_that_are_strided_or_missing():
    from paper_2603_08734_amd import residual
    torch.manual_seed(3)
    x, b = (torch.randn(6, 50, device="cuda", requires_grad=True) for _ in range(2))
    w = torch.rand(50, device="cuda", requires_grad=True)
    n = residual.Norm("rms", w, None, EPS)
    S, Y = residual.join(x, b, after=n, before=n)
    wide = torch.randn(6, 100, device="cuda")
    one = torch.autograd.grad([S, Y], [x, b, w], [wide[:, ::2], wide[:, 50:]], retain_graph=True)
    two = torch.autograd.grad([S, Y], [x, b, w], [wide[:, ::2].contiguous(), wide[:, 50:].contiguous()], retain_graph=True)
    assert all(torch.equal(p, q) for p, q in zip(one, two))
    only_s = torch.autograd.grad(S, [x, b, w], wide[:, ::2], retain_graph=True)
    only_y = torch.autograd.grad(Y, [x, b, w], wide[:, 50:], retain_graph=True)
    for p, q, r in zip(only_s, only_y, one):
        # one more rounding of each half
        assert torch.allclose(p + q, r, rtol=0, atol=64 * E * (p.abs().max() + q.abs().max()).item())
    assert torch.equal(only_s[0], wide[:, ::2])
    (g,) = torch.autograd.grad(Y, [w], wide[:, 50:], retain_graph=True)
    assert torch.equal(g, only_y[2])


def test_gradients_by_differences():
    """fp32: central differences of the library's own forward pass in the direction of its gradient."""
    from paper_2603_08734_amd import dropout, residual
    torch.manual_seed(4)
    x, b = (torch.randn(4, 24, device="cuda") for _ in range(2))
    gate, w1, w2, c = (torch.randn(24, device="cuda") for _ in range(4))
    cs, cy = torch.randn(4, 24, device="cuda"), torch.randn(4, 24, device="cuda")
    leaves = [v.requires_grad_() for v in (x, b, gate, w1, w2, c)]
    drop = dropout.Drop(0.25, 9)

    def f(x, b, gate, w1, w2, c):
        S, Y = residual.join(x, b, after=residual.Norm("layer", w1, c, 1e-2), gate=gate, scale=1.5, drop=drop, before=residual.Norm("rms", w2, c, 1e-2))
        return (S.double() * cs).sum() + (Y.double() * cy).sum()
    grads = torch.autograd.grad(f(*leaves), leaves)
    for i, g in enumerate(grads):
        step = 2.0 ** -7 / g.norm()
        with torch.no_grad():
            up, down = (f(*(v + s * step * g if j == i else v for j, v in enumerate(leaves))) for s in (1, -1))
        # values are off by a few 2^-24 of their sum of magnitudes (about 200), the difference's own error is of third order in 2^-7
        slope, want = ((up - down) / (2 * step)).item(), g.double().square().sum().item()
        assert abs(slope - want) < 0.01 * want + 400 * 8 * E / (2 * step).item()


def test_values_whose_squares_leave_the_range():
    from paper_2603_08734_amd import residual
    for dtype in (torch.float32, torch.bfloat16):
        for d in (40, 1000, 9000):
            x = (torch.randn(3, d) * 2.0 ** 90).to(dtype)
            for kind in ("rms", "layer"):
                y = residual.norm(x.cuda(), residual.Norm(kind, None, None, EPS)).double().cpu()
                want = edges.norm(x.double(), kind, None, None, EPS)[0]
                assert ((y - want).abs() <= (half_step(dtype) + 200 * E) * (want.abs() + 1)).all()


@pytest.mark.parametrize("d", [20, 700, 9000])
def test_infinities_and_nan_stay_in_their_rows(d):
    from paper_2603_08734_amd import dropout, residual
    x = torch.randn(4, d, device="cuda")
    b = torch.randn(4, d, device="cuda")
    clean = residual.join(x, b, before=residual.Norm("layer", None, None, EPS))
    x[1, d // 2] = float("nan")
    b[2, 3] = float("inf")
    S, Y = residual.join(x, b, before=residual.Norm("layer", None, None, EPS))
    for got, want in ((S, clean[0]), (Y, clean[1])):
        assert torch.equal(got[[0, 3]], want[[0, 3]])
    assert Y[1].isnan().all() and S[2, 3].isinf() and Y[2].isnan().all()
    y = residual.norm(b, residual.Norm("rms", None, None, EPS))
    assert y[2, 3].isnan() and (y[2].isnan().sum() == 1) and not y[2, 4:].any()
    # what is dropped is gone, whatever it was
    drop = dropout.Drop(1.0, 1)
    assert torch.equal(residual.join(clean[0], torch.full_like(b, float("nan")), drop=drop), clean[0])


def test_rows_of_zeros():
    from paper_2603_08734_amd import residual
    x = torch.zeros(3, 100, device="cuda", dtype=torch.float16, requires_grad=True)
    for kind in ("rms", "layer"):
        y = residual.norm(x, residual.Norm(kind, None, None, 2.0 ** -10))
        (g,) = torch.autograd.grad(y, x, torch.ones_like(y))
        assert not y.any() and torch.equal(g, torch.full_like(g, 32.0 if kind == "rms" else 0.0))


def test_shapes():
    from paper_2603_08734_amd import residual
    n = residual.Norm("rms", None, None, EPS)
    x = torch.randn(2, 3, 5, 48, device="cuda")
    gate = torch.randn(2, 3, 5, 48, device="cuda", requires_grad=True)
    S, Y = residual.join(x, x, gate=gate, before=n)
    flat = [v.reshape(30, 48) for v in (x, gate.detach())]
    for got, want in zip((S, Y), residual.join(flat[0], flat[0], gate=flat[1], before=n)):
        assert got.shape == x.shape and torch.equal(got.reshape(30, 48), want)
    assert torch.autograd.grad(Y, gate, torch.ones_like(Y))[0].shape == gate.shape
    assert torch.equal(residual.norm(x[0, 0, 0], n), residual.norm(flat[0][:1], n)[0])
    for shape in ((0, 16), (4, 0), (2, 0, 8)):
        e = torch.zeros(shape, device="cuda", requires_grad=True)
        w = torch.ones(shape[-1], device="cuda", requires_grad=True)
        S, Y = residual.join(e, e, gate=w, before=residual.Norm("rms", w, None, EPS))
        assert S.shape == Y.shape == e.shape
        grads = torch.autograd.grad([S, Y], [e, w], [torch.ones_like(S), torch.ones_like(Y)])
        assert grads[0].shape == e.shape and not grads[1].any()
        assert residual.norm(e, residual.Norm("layer", w, None, EPS)).shape == e.shape


def test_same_tensor_on_both_sides_and_twice_as_parameter():
    from paper_2603_08734_amd import residual
    x = torch.randn(5, 96, device="cuda", requires_grad=True)
    w = torch.rand(96, device="cuda", requires_grad=True)
    n = residual.Norm("rms", w, None, EPS)
    S, Y = residual.join(x, x, after=n, gate=w, before=n)
    got = torch.autograd.grad([S, Y], [x, w], [torch.ones_like(S), torch.ones_like(Y)])
    x64, w64 = x.detach().double().cpu().requires_grad_(), w.detach().double().cpu().requires_grad_()
    r = edges.join(x64, x64, ("rms", w64, None, EPS), w64, 1.0, None, ("rms", w64, None, EPS))
    want = torch.autograd.grad([r["S"], r["Y"]], [x64, w64], [torch.ones_like(r["S"]), torch.ones_like(r["Y"])])
    for g, v in zip(got, want):
        # sums of up to a dozen terms of order one to ten, each off by less than K E of them
        assert ((g.double().cpu() - v).abs() <= 60 * 16 * E * (1 + v.abs().max())).all()


def test_captured_and_replayed():
    """A training step of join and dropout in a graph; the seed moves between replays and every replay draws its own numbers."""
    from paper_2603_08734_amd import dropout, residual
    torch.manual_seed(5)
    x, b, c = (torch.randn(33, 320, device="cuda") for _ in range(3))
    w = torch.rand(320, device="cuda")
    seed = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step(x, b, w, seed):
        with torch.enable_grad():
            leaves = [v.detach().requires_grad_() for v in (x, b, w)]
            n = residual.Norm("layer", leaves[2], None, EPS)
            S, Y = residual.join(leaves[0], leaves[1], after=n, gate=leaves[2], drop=dropout.Drop(0.2, seed, 3), before=n)
            return [S.detach(), Y.detach(), *torch.autograd.grad([S, Y], leaves, [c, c])]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x, b, w, seed)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(x, b, w, seed)
    seen = []
    for i in range(4):
        seed.fill_(1000 + i)
        x.copy_(torch.randn_like(x))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in out]
        want = step(x, b, w, torch.tensor([1000 + i], device="cuda"))
        whole = step(x, b, w, seed)
        assert all(torch.equal(p, q) and torch.equal(p, r) for p, q, r in zip(got, want, whole))
        seen.append(got[0] == x)
    assert not torch.equal(seen[0], seen[1])


def test_two_streams_at_once():
    from paper_2603_08734_amd import residual
    n = residual.Norm("rms", None, None, EPS)
    xs = [torch.randn(2000, 1024, device="cuda", requires_grad=True) for _ in range(2)]
    want = []
    for x in xs:
        y = residual.norm(x, n)
        want.append((y.detach(), torch.autograd.grad(y, x, x.detach())[0]))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [None, None]
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            y = residual.norm(xs[i], n)
            got[i] = (y.detach(), torch.autograd.grad(y, xs[i], xs[i].detach())[0])
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(g, w))


def test_refusals_on_the_gpu():
    from torch.autograd import forward_ad

    from paper_2603_08734_amd import dropout, residual
    x = torch.randn(4, 32, device="cuda")
    w = torch.ones(32, device="cuda")
    n = residual.Norm("rms", w)
    for call, kind in ((lambda: residual.join(x, x.half()), ValueError), (lambda: residual.join(x, x[:3]), ValueError),
                       (lambda: residual.join(x, None), TypeError), (lambda: residual.join(x, x, gate=w[:31]), ValueError),
                       (lambda: residual.join(x, x, gate=w.cpu()), ValueError), (lambda: residual.join(x, x, gate=w.double()), ValueError), (lambda: residual.norm(x.half(), residual.Norm("rms", w.bfloat16())), ValueError),
                       (lambda: residual.join(x, x, gate=w.half()), ValueError),
                       (lambda: residual.join(x, x, scale=float("nan")), ValueError), (lambda: residual.join(x, x, drop=0.1), TypeError),
                       (lambda: residual.join(x, x, before="rms"), TypeError), (lambda: residual.norm(x, None), TypeError),
                       (lambda: residual.norm(x.double(), n), TypeError), (lambda: residual.norm(x[:, :31], n), ValueError),
                       (lambda: residual.norm(x.long(), n), TypeError), (lambda: residual.norm(torch.tensor(1.0, device="cuda"), n), TypeError),
                       (lambda: dropout.Drop(0.1, torch.zeros(2, dtype=torch.int64, device="cuda")), ValueError)):
        with pytest.raises(kind):
            call()
    v = x.clone().requires_grad_()
    y = residual.norm(v, n)
    (g,) = torch.autograd.grad(y, v, torch.ones_like(y), create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), v)
    with forward_ad.dual_level(), pytest.raises(ValueError, match="forward-mode"):
        residual.norm(forward_ad.make_dual(x, x), n)
    seed = torch.zeros(1, dtype=torch.int64, device="cuda")
    s = residual.join(v, v, drop=dropout.Drop(0.5, seed))
    seed.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(s, v, torch.ones_like(s))
    S, Y = residual.join(v, v * 1, before=n)
    S.detach().add_(1)      # the gradients do not read it
    torch.autograd.grad(Y, v, torch.ones_like(Y), retain_graph=True)
    v.detach().add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(Y, v, torch.ones_like(Y))


def test_offsets_beyond_32_bits():
    """Rows whose elements lie more than 2^31 from the first, by their number or by their distance: the same results as by themselves."""
    from paper_2603_08734_amd import dropout, residual
    n = residual.Norm("layer", torch.rand(32768, device="cuda") + 0.5, None, EPS)
    t = 70000
    x = torch.empty(t, 32768, dtype=torch.float16, device="cuda")
    x[:] = torch.randn(1, 32768, device="cuda").half()
    x[-5:] = torch.randn(5, 32768, device="cuda").half()
    drop = dropout.Drop(0.5, 1)
    y = residual.norm(x, n)
    assert torch.equal(y[-5:], residual.norm(x[-5:], n)) and torch.equal(y[:2], residual.norm(x[:2], n))
    del y
    z = dropout.dropout(x, drop)
    kept, factor = edges.kept(1, 8, 0.5, 1, 0)
    assert torch.equal(z[0, :8].cpu() != 0, kept[0] & (x[0, :8].cpu() != 0)) and torch.equal(z[-1][z[-1] != 0], 2 * x[-1][z[-1] != 0])
    del z, x
    for d, ld in ((40, 1 << 28), (40, (1 << 28) + 3), (600, 1 << 28)):
        base = torch.empty(9 * ld, dtype=torch.float16, device="cuda")
        far = base.as_strided((9, d), (ld, 1))
        far[:] = torch.randn(9, d, device="cuda").half()
        near = far.contiguous()
        n = residual.Norm("rms", None, None, EPS)
        leaves = [v.detach().requires_grad_() for v in (far, near)]
        outs = [residual.join(v, near, before=n) for v in leaves]
        grads = [torch.autograd.grad(list(o), v, [near, near])[0] for o, v in zip(outs, leaves)]
        assert all(torch.equal(p, q) for p, q in zip(*outs)) and torch.equal(*grads)
        assert torch.equal(dropout.dropout(far, drop), dropout.dropout(near, drop))
        del base, far, leaves
