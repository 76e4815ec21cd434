"""Products whose scales lie at the ends of the byte's range, with activations that bring the results back to numbers of ordinary size.

Bounds as in test_gpu_mx4: values and products of values are exact in fp32 wherever they are numbers that fp32 has, subnormal ones among them (a
value in 4 bits has two bits, and its smallest, 2^-128, is a subnormal number of bfloat16 and fp32).  quantize gives scales up to 252; beyond, the largest
values are infinite in fp32 and bfloat16."""
import numpy as np
import pytest

from test_gpu_mx4 import _check, _device, _weight, decode_64

pytestmark = pytest.mark.gpu


def _matrix(rng, n, k, lo, hi):
    """A matrix in 4 bits whose scales are bytes lo .. hi - 1, every one of them somewhere, and its values in 64 bits."""
    from paper_2603_08734_amd import mx4
    codes, scales = _weight(rng, n, k)
    scales = rng.integers(lo, hi, scales.shape).astype(np.uint8)
    scales.flat[:hi - lo] = np.arange(lo, hi)
    return mx4.Mx4(_device(codes), _device(scales), k), decode_64(codes, scales, k)


@pytest.mark.parametrize("t", [1, 5, 12, 40, 200])
@pytest.mark.parametrize("lo,hi,x_scale", [(0, 6, 110), (240, 253, -112), (0, 1, 120)])
def test_bfloat16_beside_the_ends(lo, hi, x_scale, t):
    import torch
    from paper_2603_08734_amd import mx4
    rng = np.random.default_rng(t + lo)
    n, k = 70, 640
    W, w = _matrix(rng, n, k, lo, hi)
    X = _device(rng.normal(size=(t, k)) * 2.0 ** x_scale).bfloat16()
    x = X.double().cpu().numpy()
    _check(mx4.product(X, W), x @ w.T, np.abs(x) @ np.abs(w).T, k, "bfloat16")
    Q = mx4.quantize(X)
    q = decode_64(Q.codes.cpu().numpy(), Q.scales.cpu().numpy(), k)
    _check(mx4.product(Q, W, torch.bfloat16), q @ w.T, np.abs(q) @ np.abs(w).T, k, "bfloat16")
    if lo < 200 and x_scale < 120:        # results near 2^-12 and below
        _check(mx4.product(Q, W, torch.float16), q @ w.T, np.abs(q) @ np.abs(w).T, k, "float16")


@pytest.mark.parametrize("t", [1, 5, 12, 40, 200])
def test_binary16_beside_the_ends(t):
    """binary16 activations have no size that brings such scales back: results are zero below 2^-25, infinite of the sum's sign above the type."""
    import torch
    from paper_2603_08734_amd import mx4
    rng = np.random.default_rng(t)
    n, k = 70, 640
    X = _device(rng.normal(size=(t, k)) * 100).half()
    x = X.double().cpu().numpy()
    W, _ = _matrix(rng, n, k, 0, 20)
    assert not mx4.product(X, W).any()
    W, w = _matrix(rng, n, k, 215, 226)
    ref, total = x @ w.T, np.abs(x) @ np.abs(w).T
    sure = np.abs(ref) > 1e5 + k * 2.0 ** -23 * total
    got = mx4.product(X, W).cpu().numpy()
    assert sure.mean() > 0.99 and (got[sure] == np.copysign(np.inf, ref[sure])).all() and not np.isnan(got).any()


@pytest.mark.parametrize("t", [1, 12, 40])
def test_rows_of_both_ends_beside_each_other(t):
    """A row of small scales is as exact between rows of large ones as by itself."""
    import torch
    from paper_2603_08734_amd import mx4
    rng = np.random.default_rng(t)
    n, k = 40, 384
    W, _ = _matrix(rng, n, k, 100, 110)
    W.scales[1::2] += 60
    both = _device(rng.normal(size=(t, k)) * 2.0 ** -8)
    for X in (both.half(), both.bfloat16()):
        Y = mx4.product(X, W)
        for rows in (slice(0, None, 2), slice(1, None, 2)):
            part = mx4.Mx4(W.codes[rows].contiguous(), W.scales[rows].contiguous(), k)
            one = mx4.product(X, part)
            w = decode_64(part.codes.cpu().numpy(), part.scales.cpu().numpy(), k)
            x = X.double().cpu().numpy()
            ref, total = x @ w.T, np.abs(x) @ np.abs(w).T
            if X.dtype == torch.float16 and np.abs(ref).max() > 60000:
                assert torch.equal(Y[:, rows], one)       # infinite alike
            else:
                name = str(X.dtype).split(".")[1]
                _check(Y[:, rows], ref, total, k, name)
                _check(one, ref, total, k, name)
