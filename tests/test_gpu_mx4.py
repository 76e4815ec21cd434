"""Matrices in microscaled 4-bit floating point on the GPU: conversions bit for bit against the definition in 64 bits, products
against a product of the decoded values in 64 bits.

Bounds of the products.  Values of two 4-bit operands and their products are exact, as are bfloat16 or binary16 times a value in
4 bits (beside binary16 a value enters relative to its row, exactly over 33 powers of two; the tests of wider rows say what they
allow).  A chain of k fp32 additions is off by at most k * 2^-23 of the sum of absolute values (the matrix units need not round
to nearest), and the result is rounded once: 2^-8 relative for bfloat16, 2^-11 for binary16 and 2^-25 where it is subnormal.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
ROUNDING = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}


def quantize_64(x):
    """(codes [rows, 32 B] one per cell, scale bytes [rows, B]) of a float64 matrix, from the definition."""
    rows, k = x.shape
    blocks = -(-k // 32)
    v = np.zeros((rows, blocks * 32))
    v[:, :k] = x
    v = v.reshape(rows, blocks, 32)
    bad = ~np.isfinite(v).all(axis=2)
    v = np.where(bad[..., None], 0.0, v)
    top = np.abs(v).max(axis=2)
    e = np.where(top > 0, np.frexp(top)[1] - 1 - 2, -127).clip(-127, 127)
    m = np.ldexp(np.abs(v), -e[..., None])
    d = np.abs(m[..., None] - GRID)
    code = np.argmin(d, axis=3)
    # the other neighbour at the same distance, where that has the even code
    other = np.minimum(code + 1, 7)
    tie = (np.take_along_axis(d, code[..., None], 3)[..., 0] == np.take_along_axis(d, other[..., None], 3)[..., 0]) & (other != code)
    code = np.where(tie & (code % 2 == 1), other, code)
    code = code | (np.signbit(v) * 8)
    return code.reshape(rows, -1), np.where(bad, 255, e + 127)


def decode_64(codes, scales, k):
    """Values (float64) of packed codes and scale bytes."""
    c = np.stack([codes & 15, codes >> 4], axis=2).reshape(codes.shape[0], -1)
    v = GRID[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (v.reshape(codes.shape[0], -1, 32) * s[..., None]).reshape(codes.shape[0], -1)[:, :k]


def _pack(c):
    return (c[:, 0::2] | c[:, 1::2] << 4).astype(np.uint8)


def _special_values(dtype, rows, k, seed):
    """Blocks of every size that the type has, ties, zeros of both signs, subnormals, the largest number, infinities and NaN."""
    import torch
    g = torch.Generator().manual_seed(seed)
    lo, hi = {torch.float32: (-149, 127), torch.bfloat16: (-133, 127), torch.float16: (-24, 15)}[dtype]
    x = torch.randn((rows, k), generator=g, dtype=torch.float64)
    e = torch.randint(lo, hi, (rows, -(-k // 32)), generator=g).repeat_interleave(32, dim=1)[:, :k]
    x = torch.ldexp(x.clamp(-1.99, 1.99), e).to(dtype)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 4.0, -0.25, -2.5, -5.0, 6.5, 7.99, 0.0, -0.0]).repeat(2)
    n = min(k, 32)
    x[0, :n] = ties[:n].to(dtype)
    if rows > 4:
        x[1] = 0
        x[2, ::3] = -0.0
        x[3, k - 1] = float("inf")
        x[4, 0] = float("nan")
        x[rows - 1, :n] = torch.finfo(dtype).max
    return x


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rows,k", [(1, 1), (1, 32), (3, 31), (5, 33), (7, 8), (64, 64), (33, 100), (2, 4096 + 5), (1, 8192), (1030, 96), (129, 1000)])
def test_conversions_bit_for_bit(dtype, rows, k):
    import torch
    from paper_2603_08734_amd import mx4
    print(f"case mx4 convert {dtype} {rows} x {k}", flush=True)
    x = _special_values(getattr(torch, dtype), rows, k, rows + k)
    wide = torch.full((rows, k + 3), float("nan"), dtype=x.dtype, device="cuda")      # the same rows with a stride, off alignment
    wide[:, 1:k + 1] = x.cuda()
    want_c, want_s = quantize_64(x.double().numpy())
    for X in (x.cuda(), wide[:, 1:k + 1]):
        Q = mx4.quantize(X)
        c, s = Q.codes.cpu().numpy(), Q.scales.cpu().numpy()
        assert np.array_equal(s, want_s)
        got = np.stack([c & 15, c >> 4], axis=2).reshape(rows, -1)
        # a zero may carry either sign; cells past the end are zero
        assert np.array_equal(np.where(got & 7, got, 0), np.where(want_c & 7, want_c, 0)) and not got[:, k:].any()
    values = decode_64(Q.codes.cpu().numpy(), want_s, k)
    for out in (torch.float32, torch.bfloat16, torch.float16):
        Y = mx4.dequantize(Q, out)
        assert Y.dtype == out and Y.shape == (rows, k)
        want = torch.from_numpy(values).to(out)      # 64 bits to the type: one rounding
        assert torch.equal(torch.nan_to_num(Y.cpu(), nan=77.0), torch.nan_to_num(want, nan=77.0))
    for t in (torch.float32, torch.bfloat16):        # what 4 bits hold comes back the same
        again = mx4.quantize(mx4.dequantize(Q, t).nan_to_num(0.0))
        finite = torch.from_numpy((want_s != 255).all(axis=1))
        assert torch.equal(mx4.dequantize(again)[finite.cuda()], mx4.dequantize(Q)[finite.cuda()])


def test_every_code_and_scale():
    import torch
    from paper_2603_08734_amd import mx4
    codes = torch.arange(256, dtype=torch.uint8).view(16, 16).repeat(256, 1)
    scales = torch.arange(256, dtype=torch.uint8).repeat_interleave(16).view(-1, 1)
    Q = mx4.Mx4(codes.cuda(), scales.cuda(), 32)
    want = torch.from_numpy(decode_64(codes.numpy(), scales.numpy(), 32))
    for out in (torch.float32, torch.bfloat16, torch.float16):
        assert torch.equal(torch.nan_to_num(mx4.dequantize(Q, out).cpu(), nan=77.0), torch.nan_to_num(want.to(out), nan=77.0))


def _weight(rng, n, k, spread=4):
    """Packed codes and scales of an n x k matrix whose blocks differ by `spread` powers of two."""
    blocks = -(-k // 32)
    c = rng.integers(0, 16, (n, blocks * 32))
    c[:, k:] = 0
    return _pack(c), rng.integers(118, 118 + spread, (n, blocks)).astype(np.uint8)


def _device(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _check(got, ref, total, k, dtype, extra=0.0):
    """got against ref in 64 bits; total: sums of absolute values."""
    u = ROUNDING[dtype]
    err = np.abs(got.double().cpu().numpy() - ref)
    bound = u * np.abs(ref) + (2.0 ** -25 if dtype == "float16" else 0.0) + (1 + u) * (k * 2.0 ** -23 + extra) * total
    assert (err <= bound).all(), f"{err.max()} over {(err - bound).max()}"


# one token, edges of the groups of 8, 16 and 32 that kernels for few tokens take, and of tiles
TOKENS = (1, 2, 7, 9, 16, 17, 33, 64, 65, 130, 257)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("t", TOKENS)
@pytest.mark.parametrize("n,k", [(1, 1), (16, 32), (33, 31), (100, 129), (256, 512), (130, 4100), (515, 1056)])
def test_products(t, n, k, dtype):
    import torch
    from paper_2603_08734_amd import mx4
    print(f"case mx4 product {dtype} t={t} n={n} k={k}", flush=True)
    rng = np.random.default_rng(1000 * t + n + k)
    W = mx4.Mx4(*(_device(a) for a in _weight(rng, n, k)), k)
    w = decode_64(W.codes.cpu().numpy(), W.scales.cpu().numpy(), k)
    x = _device(rng.normal(size=(t, k + 5))).to(getattr(torch, dtype))
    for X in (x[:, :k].contiguous(), x[:, 3:k + 3]):       # without gaps; rows with a stride, off alignment
        x64 = X.double().cpu().numpy()
        Y = mx4.product(X, W)
        assert Y.dtype == X.dtype
        _check(Y, x64 @ w.T, np.abs(x64) @ np.abs(w).T, k, dtype)
    Q = mx4.quantize(X)
    q = decode_64(Q.codes.cpu().numpy(), Q.scales.cpu().numpy(), k)
    _check(mx4.product(Q, W, getattr(torch, dtype)), q @ w.T, np.abs(q) @ np.abs(w).T, k, dtype)


@pytest.mark.parametrize("t", [1, 5, 16, 40, 200])
def test_scales_far_apart(t):
    """Blocks of one row whose scales differ by up to 60 powers of two, and rows whose scales are at the ends of the range.
    Beside binary16 a value below 2^-24 of 2^kSpan = 2^10 of its row's largest scale is rounded: 2^-25 / 2^10 of that scale,
    and the row's largest block has at least one value of half its scale."""
    import torch
    from paper_2603_08734_amd import mx4
    rng = np.random.default_rng(t)
    n, k = 70, 640
    codes, scales = _weight(rng, n, k)
    scales = rng.integers(90, 150, scales.shape).astype(np.uint8)
    codes = np.where(codes & 7, codes, 1 | codes).astype(np.uint8)
    w = decode_64(codes, scales, k)
    W = mx4.Mx4(_device(codes), _device(scales), k)
    x = _device(rng.normal(size=(t, k)))
    x16 = x.half()
    x64 = x16.double().cpu().numpy()
    lost = 2.0 ** -35 * np.abs(x64).sum(1)[:, None] * np.ldexp(1.0, scales.max(1).astype(int) - 127)[None, :]
    ref, total = x64 @ w.T, np.abs(x64) @ np.abs(w).T
    u = 2.0 ** -11
    got = mx4.product(x16, W).double().cpu().numpy()
    big = np.abs(ref) > 65000
    assert (np.abs(got - ref) <= u * np.abs(ref) + 2.0 ** -25 + (1 + u) * (k * 2.0 ** -23 * total + lost))[~big].all()
    xb = x.bfloat16()
    x64 = xb.double().cpu().numpy()
    _check(mx4.product(xb, W), x64 @ w.T, np.abs(x64) @ np.abs(w).T, k, "bfloat16")
    Q = mx4.quantize(xb)
    q = decode_64(Q.codes.cpu().numpy(), Q.scales.cpu().numpy(), k)
    _check(mx4.product(Q, W, torch.bfloat16), q @ w.T, np.abs(q) @ np.abs(w).T, k, "bfloat16")


@pytest.mark.parametrize("t", [1, 8, 20, 140])
def test_a_nan_or_infinity_stays_in_its_rows(t):
    import torch
    from paper_2603_08734_amd import mx4
    rng = np.random.default_rng(t)
    n, k = 100, 200
    codes, scales = _weight(rng, n, k)
    codes = np.where(codes & 7, codes, 1 | codes).astype(np.uint8)
    scales[40, 3] = 255
    W = mx4.Mx4(_device(codes), _device(scales), k)
    for dtype in (torch.float16, torch.bfloat16):
        X = _device(rng.normal(size=(t, k))).to(dtype)
        X[t - 1, 190] = float("inf")
        Y = mx4.product(X, W)
        want = torch.ones((t, n), dtype=torch.bool, device="cuda")
        want[t - 1] = False
        want[:, 40] = False
        assert torch.equal(torch.isfinite(Y), want) and Y[:, 40].isnan().all()
        Q = mx4.quantize(X)
        assert Q.scales[t - 1, 5] == 255
        Y = mx4.product(Q, W, dtype)
        assert torch.equal(torch.isfinite(Y), want)


def test_results_do_not_depend_on_the_run_or_the_stream():
    import torch
    from paper_2603_08734_amd import mx4
    rng = np.random.default_rng(0)
    for t, n, k in ((1, 300, 4096), (12, 64, 8192), (64, 512, 6000), (300, 520, 1000)):
        W = mx4.Mx4(*(_device(a) for a in _weight(rng, n, k)), k)
        X = _device(rng.normal(size=(t, k))).bfloat16()
        first = mx4.product(X, W), mx4.product(mx4.quantize(X), W, torch.float16)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            second = mx4.product(X, W), mx4.product(mx4.quantize(X), W, torch.float16)
        torch.cuda.current_stream().wait_stream(side)
        for a, b in zip(first, second):
            assert torch.equal(a, b)


def test_products_in_a_graph():
    """A captured product, replayed on new activations between eager work, gives what the eager one does."""
    import torch
    from paper_2603_08734_amd import mx4
    rng = np.random.default_rng(5)
    for t, n, k in ((1, 300, 4096), (70, 200, 3000)):
        W = mx4.Mx4(*(_device(a) for a in _weight(rng, n, k)), k)
        X = _device(rng.normal(size=(t, k))).bfloat16()
        mx4.product(mx4.quantize(X), W, torch.bfloat16)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = mx4.product(X, W), mx4.product(mx4.quantize(X), W, torch.bfloat16)
        for _ in range(3):
            X.copy_(_device(rng.normal(size=(t, k))))
            want = mx4.product(X, W), mx4.product(mx4.quantize(X), W, torch.bfloat16)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(out, want):
                assert torch.equal(a, b)


def test_empty_sizes():
    import torch
    from paper_2603_08734_amd import mx4
    W = mx4.quantize(torch.randn((5, 40), device="cuda"))
    assert mx4.product(torch.empty((0, 40), dtype=torch.float16, device="cuda"), W).shape == (0, 5)
    none = mx4.quantize(torch.empty((0, 40), device="cuda"))
    assert none.dequantize().shape == (0, 40)
    assert mx4.product(torch.ones((3, 40), dtype=torch.float16, device="cuda"), none).shape == (3, 0)
    thin = mx4.quantize(torch.empty((5, 0), device="cuda"))
    assert torch.equal(mx4.product(torch.empty((3, 0), dtype=torch.float16, device="cuda"), thin),
                       torch.zeros((3, 5), dtype=torch.float16, device="cuda"))


def test_calls_refuse():
    import torch
    from paper_2603_08734_amd import mx4
    X = torch.randn((4, 64), device="cuda")
    W = mx4.quantize(X)
    for bad in (X, X.half()[:, :32], X.half()[0], X.half().cpu()):
        with pytest.raises((TypeError, ValueError)):
            mx4.product(bad, W)
    with pytest.raises(TypeError):
        mx4.product(W, W)                         # no type for the result
    with pytest.raises(TypeError):
        mx4.product(X.half(), W, torch.bfloat16)  # another type than the activations'
    with pytest.raises(TypeError):
        mx4.product(X.half(), X.half())
    with pytest.raises(TypeError):
        mx4.quantize(X.double())
    with pytest.raises(TypeError):
        mx4.dequantize(W, torch.float64)
    with pytest.raises(ValueError):
        mx4.product(X.half().requires_grad_(), W)
    with pytest.raises(ValueError):
        mx4.Mx4(W.codes, W.scales, 65)
    with pytest.raises(ValueError):
        mx4.Mx4(W.codes[:3], W.scales, 64)
    with torch.no_grad():
        mx4.product(X.half().requires_grad_(), W)
