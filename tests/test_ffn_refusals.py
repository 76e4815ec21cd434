"""Argument checks of the feed-forward entry points at the C boundary.  Every call here is refused before anything is launched, so
the addresses are never followed and no GPU is needed."""
import ctypes

import pytest

from paper_2603_08734_amd import binding as b

P = 1 << 20      # an address that is aligned to anything asked for


def test_conversions_refuse():
    L = b.lib()
    for f, (x, codes, scales) in ((lambda x, c, s, t, r, k, ld: L.rsh_mx4_quantize(x, t, r, k, ld, c, s, None), (P, P, P)),
                                  (lambda x, c, s, t, r, k, ld: L.rsh_mx4_dequantize(c, s, r, k, x, t, ld, None), (P, P, P))):
        for i in range(3):
            ptrs = [x, codes, scales]
            ptrs[i] = None
            assert f(*ptrs, b.RSH_F32, 4, 64, 64) == b.RSH_ERR_NULL
        for kind, rows, k, ld in ((b.RSH_MX4, 4, 64, 64), (-1, 4, 64, 64), (b.RSH_F32, 0, 64, 64), (b.RSH_F32, 4, 0, 64), (b.RSH_F32, 4, 64, 63)):
            assert f(x, codes, scales, kind, rows, k, ld) == b.RSH_ERR_BAD_OPTION
        assert f(x + 2, codes, scales, b.RSH_F32, 4, 64, 64) == b.RSH_ERR_BAD_OPTION
        assert f(x + 1, codes, scales, b.RSH_F16, 4, 64, 64) == b.RSH_ERR_BAD_OPTION
        assert f(x, codes + 8, scales, b.RSH_F16, 4, 64, 64) == b.RSH_ERR_BAD_OPTION
        assert f(x, codes, scales, b.RSH_F16, 1 << 31, 64, 64) == b.RSH_ERR_TOO_LARGE


def _product(x=P, xs=None, xt=b.RSH_F16, ld=64, w=P, ws=P, y=P, yt=b.RSH_F16, t=4, n=8, k=64, work=P):
    return b.lib().rsh_mx4_product(x, xs, xt, ld, w, ws, y, yt, t, n, k, work, None)


@pytest.mark.parametrize("status,change", [
    (b.RSH_ERR_NULL, dict(x=None)), (b.RSH_ERR_NULL, dict(w=None)), (b.RSH_ERR_NULL, dict(ws=None)), (b.RSH_ERR_NULL, dict(y=None)),
    (b.RSH_ERR_NULL, dict(xt=b.RSH_MX4)), (b.RSH_ERR_BAD_OPTION, dict(xs=P)), (b.RSH_ERR_BAD_OPTION, dict(xt=b.RSH_F32)),
    (b.RSH_ERR_BAD_OPTION, dict(yt=b.RSH_BF16)), (b.RSH_ERR_BAD_OPTION, dict(yt=b.RSH_F32, xt=b.RSH_MX4, xs=P)), (b.RSH_ERR_BAD_OPTION, dict(ld=63)),
    (b.RSH_ERR_BAD_OPTION, dict(t=0)), (b.RSH_ERR_BAD_OPTION, dict(n=-1)), (b.RSH_ERR_BAD_OPTION, dict(k=0)), (b.RSH_ERR_BAD_OPTION, dict(w=P + 8)),
    (b.RSH_ERR_BAD_OPTION, dict(y=P + 1)), (b.RSH_ERR_BAD_OPTION, dict(x=P + 8, xt=b.RSH_MX4, xs=P)), (b.RSH_ERR_BAD_OPTION, dict(k=1 << 31)),
    (b.RSH_ERR_TOO_LARGE, dict(t=(1 << 31) - 1, n=(1 << 31) - 1))])
def test_products_refuse(status, change):
    assert _product(**change) == status


def _forward(x=P, kind=b.RSH_F16, ld_x=64, wg=P, wu=P, ld_w=64, gs=None, us=None, act=0, h=P, g=None, u=None, t=4, d=64, f=8, work=P):
    return b.lib().rsh_gated_forward(x, kind, ld_x, wg, wu, ld_w, gs, us, act, h, g, u, t, d, f, work, None)


@pytest.mark.parametrize("status,change", [
    (b.RSH_ERR_NULL, dict(x=None)), (b.RSH_ERR_NULL, dict(wg=None)), (b.RSH_ERR_NULL, dict(wu=None)), (b.RSH_ERR_NULL, dict(h=None)),
    (b.RSH_ERR_NULL, dict(gs=P)), (b.RSH_ERR_NULL, dict(g=P)), (b.RSH_ERR_BAD_OPTION, dict(kind=b.RSH_F32)), (b.RSH_ERR_BAD_OPTION, dict(act=3)),
    (b.RSH_ERR_BAD_OPTION, dict(act=-1)), (b.RSH_ERR_BAD_OPTION, dict(ld_x=63)), (b.RSH_ERR_BAD_OPTION, dict(ld_w=63)), (b.RSH_ERR_BAD_OPTION, dict(t=0)),
    (b.RSH_ERR_BAD_OPTION, dict(d=0)), (b.RSH_ERR_BAD_OPTION, dict(f=0)), (b.RSH_ERR_BAD_OPTION, dict(wg=P + 8, gs=P, us=P)),
    (b.RSH_ERR_BAD_OPTION, dict(wg=P + 1)), (b.RSH_ERR_BAD_OPTION, dict(g=P + 2, u=P))])
def test_blocks_refuse(status, change):
    assert _forward(**change) == status


def _backward(x=P, kind=b.RSH_F16, ld_x=64, wg=P, wu=P, ld_w=64, g=P, u=P, dh=P, ld_h=8, act=0, dx=P, dwg=P, dwu=P, t=4, d=64, f=8, work=P):
    return b.lib().rsh_gated_backward(x, kind, ld_x, wg, wu, ld_w, g, u, dh, ld_h, act, dx, dwg, dwu, t, d, f, work, None)


@pytest.mark.parametrize("status,change", [
    (b.RSH_ERR_NULL, dict(x=None)), (b.RSH_ERR_NULL, dict(wg=None)), (b.RSH_ERR_NULL, dict(g=None)), (b.RSH_ERR_NULL, dict(u=None)),
    (b.RSH_ERR_NULL, dict(dh=None)), (b.RSH_ERR_NULL, dict(work=None)), (b.RSH_ERR_NULL, dict(dx=None, dwg=None, dwu=None)),
    (b.RSH_ERR_BAD_OPTION, dict(kind=b.RSH_MX4)), (b.RSH_ERR_BAD_OPTION, dict(ld_h=7)), (b.RSH_ERR_BAD_OPTION, dict(ld_w=63)),
    (b.RSH_ERR_BAD_OPTION, dict(t=0)), (b.RSH_ERR_BAD_OPTION, dict(work=P + 2)), (b.RSH_ERR_BAD_OPTION, dict(dx=P + 1))])
def test_gradients_refuse(status, change):
    assert _backward(**change) == status


def test_work_sizes():
    L, n = b.lib(), ctypes.c_int64(-1)
    assert L.rsh_gated_backward_work(4, 64, 9, ctypes.byref(n)) == 0 and n.value >= 2 * 2 * 4 * 16
    for f, args in ((L.rsh_mx4_product_work, (b.RSH_F16, 4, 8, 64)), (L.rsh_gated_forward_work, (b.RSH_MX4, 4, 64, 8))):
        assert f(*args, ctypes.byref(n)) == 0 and n.value >= 0
        assert f(*args, None) == b.RSH_ERR_NULL
        assert f(b.RSH_F32, *args[1:], ctypes.byref(n)) == b.RSH_ERR_BAD_OPTION
        assert f(args[0], 0, *args[2:], ctypes.byref(n)) == b.RSH_ERR_BAD_OPTION
    assert L.rsh_gated_backward_work(4, 64, -1, ctypes.byref(n)) == b.RSH_ERR_BAD_OPTION and L.rsh_gated_backward_work(4, 64, 9, None) == b.RSH_ERR_NULL


def test_calls_without_a_gpu_refuse():
    """Nothing falls back to another device: operands in host memory are refused by name."""
    import torch
    from paper_2603_08734_amd import ffn, mx4
    x, w = torch.zeros((2, 32), dtype=torch.float16), torch.zeros((4, 32), dtype=torch.float16)
    with pytest.raises(ValueError, match="X"):
        mx4.quantize(x)
    with pytest.raises(ValueError, match="X"):
        ffn.gated(x, w, w)
    with pytest.raises(ValueError, match="codes"):
        mx4.Mx4(torch.zeros((4, 16), dtype=torch.uint8), torch.zeros((4, 1), dtype=torch.uint8), 32)
