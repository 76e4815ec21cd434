"""Low-rank adapters and their gradients against the formulas in 64 bits.

Bounds.  E = 2^-24 is half a step of fp32, u half a step of the result's type.  H = X A^T: products of 16-bit numbers are exact in fp32, and a
sum of k of them is at most k / 8 + 40 additions one after the other (eight waves of a workgroup, then the waves, then the parts):
e(H) <= E (k / 8 + 40) |X| |A|^T.  The second product takes H as two numbers of bfloat16, P = 2^-17 of it off, and numbers of binary16 as two
exact ones: at most 4 r terms, e <= (P + E (4 r + 40)) s |H| |B| + s e(H) |B|, Y is added (E of the sum), and the result rounded once: + u |value|.
A factor's gradient is a sum over the tokens of an adapter in the same form, at most 4 t terms one after the other:
e <= s e(dH)^T |X| + (P + E (4 t + 64)) s |dH|^T |X|.  Results in binary16 may be subnormal: + 2^-25.
"""
import pytest
import torch

from oracle import edges

pytestmark = pytest.mark.gpu

E, P = 2.0 ** -24, 2.0 ** -17
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def make(t, k, m, n, r, dtype, index="random", scaled=True, seed=0):
    g = torch.Generator().manual_seed(seed + 13 * t + k + 7 * m + n + r)
    T = TYPES[dtype]

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g) * scale).to(T)
    i = {"random": lambda: torch.randint(-1, n, (t,), generator=g),
         "runs": lambda: torch.randint(-1, n, (t,), generator=g).sort().values.roll(t // 3),
         "one": lambda: torch.full((t,), n - 1), "none": lambda: torch.full((t,), -1),
         "outside": lambda: torch.randint(-3, 2 * n + 2, (t,), generator=g) * torch.randint(0, 2, (t,), generator=g) * 2 ** 20}[index]()
    return dict(y=normal(t, m), x=normal(t, k), a=normal(n, r, k, scale=k ** -0.5), b=normal(n, r, m, scale=0.5), dout=normal(t, m, scale=0.25),
                index=i.to(torch.int32 if seed % 2 else torch.int64), scales=(torch.rand(n, generator=g) * 2 - 0.5) if scaled else None)


def library(c, grads=True):
    from paper_2603_08734_amd import adapters
    v = {name: x if x is None else x.cuda() for name, x in c.items()}
    leaves = [v[n].requires_grad_(grads) for n in ("y", "x", "a", "b")]
    out = adapters.add(*leaves, v["index"], v["scales"])
    if not grads:
        return [out]
    return [out.detach(), *torch.autograd.grad(out, leaves, v["dout"])]


def reference(c, device):
    """[(value, bound before the last rounding)] of out, dY, dX, dA, dB."""
    y, x, a, b, dout = (c[n].double().to(device) for n in ("y", "x", "a", "b", "dout"))
    (t, k), (n, r, m) = x.shape, b.shape
    out, eout, dx, edx = y.clone(), y.abs() * E, torch.zeros_like(x), torch.zeros_like(x)
    da, eda, db, edb = torch.zeros_like(a), torch.zeros_like(a), torch.zeros_like(b), torch.zeros_like(b)
    for i in range(n):
        rows = torch.nonzero(c["index"] == i).squeeze(1).to(device)
        s = 1.0 if c["scales"] is None else c["scales"][i].item()
        xi, gi, S = x[rows], dout[rows], abs(s)
        h, dh = xi @ a[i].t(), gi @ b[i].t()
        eh, edh = E * (k / 8 + 40) * (xi.abs() @ a[i].abs().t()), E * (m / 8 + 40) * (gi.abs() @ b[i].abs().t())
        out[rows] += s * (h @ b[i])
        eout[rows] += S * (eh @ b[i].abs()) + (P + E * (4 * r + 40)) * S * (h.abs() @ b[i].abs()) + 2 * E * out[rows].abs()
        dx[rows] = s * (dh @ a[i])
        edx[rows] = S * (edh @ a[i].abs()) + (P + E * (4 * r + 40)) * S * (dh.abs() @ a[i].abs())
        da[i], db[i] = s * (dh.t() @ xi), s * (h.t() @ gi)
        chain = P + E * (4 * len(rows) + 64)
        eda[i] = S * (edh.t() @ xi.abs()) + chain * S * (dh.abs().t() @ xi.abs())
        edb[i] = S * (eh.t() @ gi.abs()) + chain * S * (h.abs().t() @ gi.abs())
    return [(out, eout), (dout, torch.zeros_like(dout)), (dx, edx), (da, eda), (db, edb)]


def check(c, grads=True):
    """With gradients, and without: few tokens then go in one launch."""
    if grads:
        check(c, False)
    got, want = library(c, grads), reference(c, "cuda" if c["x"].numel() > 1 << 18 else "cpu")
    dtype = c["x"].dtype
    u, least = torch.finfo(dtype).eps / 2, 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134
    for name, g, (value, bound) in zip(("out", "dY", "dX", "dA", "dB"), got, want):
        assert g.shape == value.shape and g.dtype == dtype
        off = (g.double().to(value.device) - value).abs() - (bound + u * (value.abs() + bound) + least)
        assert bool((off <= 0).all()), f"{name}: {off.max().item()} beyond the bound, {int((off > 0).sum())} of {off.numel()}"
    return got


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("t", [1, 2, 15, 16, 17, 33, 64, 65, 255, 256, 257, 300, 1000])
@pytest.mark.parametrize("index", ["random", "runs", "one"])
def test_tokens(dtype, t, index):
    check(make(t, 96, 136, 5, 8, dtype, index))


@pytest.mark.parametrize("r", [1, 3, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 128, 130, 512])
@pytest.mark.parametrize("t", [9, 290])
def test_ranks(r, t):
    check(make(t, 200, 152, 3, r, "bf16", seed=1))


@pytest.mark.parametrize("k,m", [(1, 1), (1, 64), (64, 1), (7, 9), (8, 8), (63, 65), (64, 127), (65, 128), (129, 511), (1000, 513), (4100, 1003), (30, 1025)])
@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("t", [5, 270])
def test_widths(k, m, dtype, t):
    check(make(t, k, m, 4, 12, dtype, seed=t))


@pytest.mark.parametrize("n,t", [(1, 40), (1, 3000), (61, 77), (200, 2000), (500, 300), (2047, 900), (2048, 900), (4096, 700)])
def test_numbers_of_adapters(n, t):
    check(make(t, 40, 48, n, 4, "fp16"))
    check(make(t, 40, 48, n, 4, "fp16", "runs", seed=1))


@pytest.mark.parametrize("t", [6, 256, 400])
@pytest.mark.parametrize("index", ["none", "outside"])
def test_tokens_without_an_adapter(t, index):
    for seed in (0, 1):
        c = make(t, 72, 88, 3, 16, "bf16", index, seed=seed)
        got = check(c)
        plain = ~((c["index"] >= 0) & (c["index"] < 3))
        assert torch.equal(got[0].cpu()[plain], c["y"][plain]) and not got[2].cpu()[plain].any()
        if index == "none":
            assert not got[3].any() and not got[4].any()


def test_indexes_of_64_bits_that_look_small():
    """2^32 + 1 is no adapter."""
    c = make(20, 32, 32, 3, 4, "fp16")
    c["index"] = torch.where(torch.arange(20) % 2 == 0, (1 << 32) + 1, 1)
    got = check(c)
    assert torch.equal(got[0].cpu()[::2], c["y"][::2])


@pytest.mark.parametrize("k,m,r", [(8192, 2100, 16), (8200, 1024, 20), (16384, 64, 16), (16400, 64, 16), (1024, 3000, 32), (1000, 5000, 33)])
def test_few_tokens_around_what_one_launch_takes(k, m, r):
    for t in (1, 3, 40):
        check(make(t, k, m, 5, r, "bf16", "random" if t > 1 else "one"))


@pytest.mark.parametrize("scaled", [False, True])
def test_long_widths(scaled):
    check(make(3, 20000, 9000, 4, 16, "bf16", scaled=scaled))
    check(make(700, 8192, 4096, 4, 64, "bf16", "runs", scaled=scaled))
    check(make(2500, 1024, 2000, 2, 24, "fp16", "runs", scaled=scaled))


def test_many_tokens():
    check(make(70000, 32, 24, 6, 4, "bf16", "random"))
    check(make(40000, 16, 16, 1, 4, "fp16", "one"))


def test_results_do_not_change_from_call_to_call():
    for t in (50, 1500):
        c = make(t, 520, 260, 7, 20, "bf16")
        one = library(c)
        for _ in range(3):
            assert all(torch.equal(p, q) for p, q in zip(one, library(c)))


def test_order_of_the_tokens_does_not_matter_to_a_token():
    from paper_2603_08734_amd import adapters
    for t in (100, 900):
        c = {n: x.cuda() for n, x in make(t, 300, 520, 9, 16, "fp16").items()}
        p = torch.randperm(t, device="cuda")
        out = adapters.add(c["y"], c["x"], c["a"], c["b"], c["index"], c["scales"])
        assert torch.equal(adapters.add(c["y"][p], c["x"][p], c["a"], c["b"], c["index"][p], c["scales"]), out[p])


def test_strides_alignment_and_shapes():
    from paper_2603_08734_amd import adapters
    for t in (30, 300):
        c = {n: x.cuda() for n, x in make(t, 200, 136, 3, 8, "bf16").items()}
        args = c["a"], c["b"], c["index"], c["scales"]
        want = adapters.add(c["y"], c["x"], *args)
        wide = torch.randn(t, 411, device="cuda").bfloat16()
        for at in (0, 1, 5):
            wide[:, at:at + 200], wide[:, 203 + at:339 + at] = c["x"], c["y"]
            assert torch.equal(adapters.add(wide[:, 203 + at:339 + at], wide[:, at:at + 200], *args), want)
        assert torch.equal(adapters.add(c["y"].t().contiguous().t(), c["x"].t().contiguous().t(), *args), want)
        two = torch.stack([c["index"], c["index"] + 1], dim=1)[:, 0]
        transposed = [f.transpose(1, 2).contiguous().transpose(1, 2) for f in args[:2]]
        assert torch.equal(adapters.add(c["y"], c["x"], *transposed, two, c["scales"]), want)
        shaped = adapters.add(c["y"].view(2, t // 2, 136), c["x"].view(2, t // 2, 200), args[0], args[1], c["index"].view(2, -1), args[3])
        assert torch.equal(shaped.view(t, 136), want)
        assert torch.equal(adapters.add(c["y"][7], c["x"][7], args[0], args[1], c["index"][7], args[3]), want[7])
        # a prefix of a longer buffer: rows behind the batch are not read for it
        assert torch.equal(adapters.add(c["y"][:20], c["x"][:20], args[0], args[1], args[2][:20], args[3]), want[:20])
        leaf = c["x"].clone().requires_grad_()
        out = adapters.add(c["y"], leaf, *args)
        grad = torch.randn(136, t, device="cuda").bfloat16().t()
        assert torch.equal(torch.autograd.grad(out, leaf, grad, retain_graph=True)[0], torch.autograd.grad(out, leaf, grad.contiguous())[0])


def test_empty_sizes():
    from paper_2603_08734_amd import adapters
    for t, k, m, n, r in ((0, 8, 8, 2, 4), (3, 0, 8, 2, 4), (3, 8, 0, 2, 4), (3, 8, 8, 0, 4), (3, 8, 8, 2, 0)):
        y, x, a, b = (torch.ones(s, device="cuda", dtype=torch.float16, requires_grad=True) for s in ((t, m), (t, k), (n, r, k), (n, r, m)))
        out = adapters.add(y, x, a, b, torch.zeros(t, dtype=torch.int64, device="cuda"))
        assert torch.equal(out, y)
        grads = torch.autograd.grad(out, (y, x, a, b), torch.ones_like(out))
        assert not any(g.any() for g in grads[1:]) and torch.equal(grads[0], torch.ones_like(y))
        with torch.no_grad():
            out = adapters.add(y, x, a, b, torch.zeros(t, dtype=torch.int32, device="cuda"))
            assert torch.equal(out, y) and (out.numel() == 0 or out.data_ptr() != y.data_ptr())


@pytest.mark.parametrize("value", [60000.0, float("inf"), float("nan")])
def test_empty_sizes_leave_out_what_the_operands_hold(value):
    """Nothing is multiplied, so nothing of X (whose sum overflows, or is no number), A, B or dout reaches the others."""
    from paper_2603_08734_amd import adapters
    for t, k, m, n, r in ((3, 0, 8, 2, 4), (3, 8, 8, 0, 4), (3, 8, 8, 2, 0)):
        y = torch.ones((t, m), device="cuda", dtype=torch.float16, requires_grad=True)
        x, a, b = (torch.full(s, value, device="cuda", dtype=torch.float16, requires_grad=True) for s in ((t, k), (n, r, k), (n, r, m)))
        out = adapters.add(y, x, a, b, torch.zeros(t, dtype=torch.int64, device="cuda"))
        assert torch.equal(out, y)
        grads = torch.autograd.grad(out, (y, x, a, b), torch.full_like(out, value))
        assert all(torch.equal(g, torch.zeros_like(v)) for g, v in zip(grads[1:], (x, a, b)))


@pytest.mark.parametrize("want", [(0,), (1,), (2,), (3,), (0, 2), (1, 3)])
def test_some_gradients(want):
    from paper_2603_08734_amd import adapters
    c = make(280, 100, 72, 4, 8, "bf16")
    whole = library(c)[1:]
    v = {n: x.cuda() for n, x in c.items()}
    leaves = [v[n] for n in ("y", "x", "a", "b")]
    for i in want:
        leaves[i].requires_grad_()
    out = adapters.add(*leaves, v["index"], v["scales"])
    for i, g in zip(want, torch.autograd.grad(out, [leaves[i] for i in want], v["dout"])):
        assert torch.equal(g, whole[i])


def test_large_and_infinite_values_stay_with_their_tokens():
    from paper_2603_08734_amd import adapters
    for t in (40, 400):
        c = {n: x.cuda() for n, x in make(t, 64, 64, 2, 16, "fp16", "random").items()}
        c["index"] = torch.arange(t, device="cuda") % 2
        args = c["a"], c["b"], c["index"], c["scales"]
        clean = adapters.add(c["y"], c["x"], *args)
        x = c["x"].clone()
        x[4], x[5, 3], x[6, 0] = 60000, float("nan"), float("inf")
        out = adapters.add(c["y"], x, *args)
        rest = [i for i in range(t) if i not in (4, 5, 6)]
        assert torch.equal(out[rest], clean[rest]) and out[5].isnan().all() and not out[6].isfinite().any()
        # sums beyond binary16 between the two products: they are fp32
        big = torch.full_like(c["a"], 16.0)
        small = torch.full_like(c["b"], 2.0 ** -16)
        got = adapters.add(torch.zeros_like(c["y"]), torch.full_like(c["x"], 1024.0), big, small, c["index"])
        assert torch.equal(got, torch.full_like(got, 16 * 64 * 16 * 1024 * 2.0 ** -16))


def test_subnormal_numbers():
    """Products of numbers of binary16 below its normal range: exact in fp32, H = 64 2^-24 2^-2 and so on."""
    from paper_2603_08734_amd import adapters
    for t in (20, 300):
        x, a, b = torch.full((t, 64), 2.0 ** -24), torch.full((1, 4, 64), 0.25), torch.full((1, 4, 48), 2.0 ** -20 * 3)
        x, a, b = (v.half().cuda().requires_grad_() for v in (x, a, b))
        y = torch.zeros(t, 48, device="cuda").half()
        i = torch.zeros(t, dtype=torch.int32, device="cuda")
        scales = torch.tensor([2.0 ** 24], device="cuda")
        out = adapters.add(y, x, a, b, i, scales)
        assert torch.equal(out, torch.full_like(out, 4 * 64 * 2.0 ** -24 * 0.25 * 3 * 2.0 ** -20 * 2 ** 24))
        dx, da, db = torch.autograd.grad(out, (x, a, b), torch.full_like(out, 2.0 ** -10))
        assert torch.equal(dx, torch.full_like(dx, 4 * 48 * 3 * 2.0 ** -20 * 2.0 ** -10 * 0.25 * 2 ** 24))
        assert torch.equal(da, torch.full_like(da, t * 48 * 3 * 2.0 ** -20 * 2.0 ** -10 * 2.0 ** -24 * 2 ** 24))
        assert torch.equal(db, torch.full_like(db, t * 64 * 2.0 ** -24 * 0.25 * 2.0 ** -10 * 2 ** 24))


def test_captured_and_replayed():
    """A decoding step and a training step in graphs; other tokens and other adapters at every replay."""
    from paper_2603_08734_amd import adapters
    for t, train in ((12, False), (300, False), (12, True), (300, True)):
        cs = [{n: x.cuda() for n, x in make(t, 200, 136, 5, 16, "bf16", seed=2 * s).items()} for s in range(4)]
        v = {n: x.clone() for n, x in cs[0].items()}

        def step(c):
            with torch.enable_grad():
                leaves = [c[n].detach().requires_grad_(train) for n in ("y", "x", "a", "b")]
                out = adapters.add(*leaves, c["index"], c["scales"])
                return [out.detach(), *(torch.autograd.grad(out, leaves, c["dout"]) if train else ())]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(v)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(v)
        for c in cs[1:] + cs[:2]:
            for n in v:
                v[n].copy_(c[n])
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(out, step(c)))


def test_two_streams_at_once():
    cs = [make(1200, 512, 640, 6, 32, "bf16", seed=2 * s) for s in range(2)]
    want = [library(c) for c in cs]
    torch.cuda.synchronize()
    got = [None, None]
    for i in range(2):
        with torch.cuda.stream(torch.cuda.Stream()):
            got[i] = library(cs[i])
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(g, w))


def test_gradients_by_differences():
    """The gradient's size along itself: the formula is linear in each factor, so a central difference of fp16 values that are exact has no
    error of its own; what is left is the rounding of the outputs, u of each, against a change of step |g|^2."""
    from paper_2603_08734_amd import adapters
    c = {n: x if x is None else x.cuda() for n, x in make(260, 48, 40, 3, 8, "fp16").items()}
    leaves = [c[n].requires_grad_() for n in ("x", "a", "b")]
    grads = torch.autograd.grad(adapters.add(c["y"], *leaves, c["index"], c["scales"]), leaves, c["dout"])
    for i, g in enumerate(grads):
        values = []
        for sign in (1, -1):
            moved = [(v.detach().float() + sign * g.float()).half() if j == i else v.detach() for j, v in enumerate(leaves)]
            step = moved[i].double() - leaves[i].detach().double()
            values.append(((adapters.add(c["y"], *moved, c["index"], c["scales"]).double() * c["dout"].double()).sum().item(),
                           (step * g.double()).sum().item()))
        slope, want = values[0][0] - values[1][0], values[0][1] - values[1][1]
        rounding = 2 * 2.0 ** -11 * (c["dout"].double().abs() * 64).sum().item()
        assert abs(slope - want) <= rounding + 0.01 * abs(want)


def test_refusals_on_the_gpu():
    from torch.autograd import forward_ad

    from paper_2603_08734_amd import adapters, binding
    c = {n: x.cuda() for n, x in make(6, 32, 40, 3, 8, "fp16").items()}
    y, x, a, b, i, s = (c[n] for n in ("y", "x", "a", "b", "index", "scales"))
    for args, kind in (((y.float(), x, a, b, i, s), TypeError), ((y.float(), x.float(), a.float(), b.float(), i, s), TypeError),
                       ((y, x, a.bfloat16(), b, i, s), TypeError), ((y, x, a, b, i.float(), s), TypeError), ((y, x, a, b, i.short(), s), TypeError),
                       ((y, x, a, b, [0] * 6, s), TypeError), ((y[:5], x, a, b, i, s), ValueError), ((y, x[:, :31], a, b, i, s), ValueError),
                       ((y, x, a[:2], b, i, s), ValueError), ((y, x, a, b[:, :7], i, s), ValueError), ((y, x, a[0], b[0], i, s), ValueError),
                       ((y, x, a, b, i[:5], s), ValueError), ((y, x, a, b, i, s[:2]), ValueError), ((y, x, a, b, i, s.double()), ValueError),
                       ((y, x, a, b, i, 2.0), ValueError), ((y, x, a, b, i.cpu(), s), ValueError), ((y, x, a, b.cpu(), i, s), ValueError),
                       ((y, x, a, b, i, s.clone().requires_grad_()), ValueError),
                       ((y, x, torch.zeros(4097, 1, 32, device="cuda").half(), torch.zeros(4097, 1, 40, device="cuda").half(), i), binding.RshError),
                       ((y, x, torch.zeros(1, 513, 32, device="cuda").half(), torch.zeros(1, 513, 40, device="cuda").half(), i), binding.RshError)):
        with pytest.raises(kind):
            adapters.add(*args)
    v = x.clone().requires_grad_()
    (g,) = torch.autograd.grad(adapters.add(y, v, a, b, i, s), v, torch.ones_like(y), create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.float().sum(), v)
    with forward_ad.dual_level(), pytest.raises(ValueError, match="forward-mode"):
        adapters.add(forward_ad.make_dual(y, y), x, a, b, i, s)


def test_offsets_beyond_32_bits():
    """Adapters whose factors lie more than 2^31 elements from the first, and tokens far apart."""
    from paper_2603_08734_amd import adapters
    n, r, k, m = 4096, 16, 33000, 64
    a = torch.empty(n, r, k, dtype=torch.bfloat16, device="cuda")
    b = torch.empty(n, r, m, dtype=torch.bfloat16, device="cuda")
    a[4090:], b[4090:] = torch.randn(6, r, k, device="cuda").bfloat16(), torch.randn(6, r, m, device="cuda").bfloat16()
    for t in (7, 300):
        x, y = torch.randn(t, k, device="cuda").bfloat16(), torch.randn(t, m, device="cuda").bfloat16()
        i = torch.randint(4090, 4096, (t,), device="cuda")
        # the parts of k go by how many adapters there may be, so by the bounds
        value, bound = reference(dict(y=y, x=x, a=a[4090:], b=b[4090:], dout=y, index=i - 4090, scales=None), "cuda")[0]
        off = (adapters.add(y, x, a, b, i).double() - value).abs() - (bound + 2.0 ** -8 * (value.abs() + bound))
        assert bool((off <= 0).all())
    base = torch.empty(6 << 28, dtype=torch.bfloat16, device="cuda")
    far = base.as_strided((6, 200), (1 << 28, 1))
    far[:] = torch.randn(6, 200, device="cuda").bfloat16()
    i = torch.arange(6, device="cuda") % 3
    a, b, y = torch.randn(3, 8, 200, device="cuda").bfloat16(), torch.randn(3, 8, 72, device="cuda").bfloat16(), torch.randn(6, 72, device="cuda").bfloat16()
    assert torch.equal(adapters.add(y, far, a, b, i), adapters.add(y, far.contiguous(), a, b, i))
