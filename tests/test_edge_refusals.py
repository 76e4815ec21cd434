"""Argument checks of dropout, joins and adapters at the C boundary.  Every call here is refused before anything is launched, so the addresses
are never followed and no GPU is needed."""
import ctypes

import pytest

from paper_2603_08734_amd import binding as b

P = 1 << 20      # an address that is aligned to anything asked for
INF = float("inf")


def _drop(share=1000, seed_dev=None):
    return b.rsh_drop_t(1, 2, seed_dev, share)


@pytest.mark.parametrize("status,change", [
    (b.RSH_ERR_NULL, dict(x=None)), (b.RSH_ERR_NULL, dict(y=None)), (b.RSH_ERR_NULL, dict(drop=None)), (b.RSH_ERR_BAD_OPTION, dict(kind=b.RSH_MX4)),
    (b.RSH_ERR_BAD_OPTION, dict(t=0)), (b.RSH_ERR_BAD_OPTION, dict(d=0)), (b.RSH_ERR_BAD_OPTION, dict(t=1 << 31)), (b.RSH_ERR_BAD_OPTION, dict(ld=63)),
    (b.RSH_ERR_TOO_LARGE, dict(d=(1 << 21) + 1, ld=1 << 22)), (b.RSH_ERR_BAD_OPTION, dict(drop=_drop(65537))), (b.RSH_ERR_BAD_OPTION, dict(drop=_drop(1, P + 4))),
    (b.RSH_ERR_BAD_OPTION, dict(x=P + 1)), (b.RSH_ERR_BAD_OPTION, dict(x=P + 2, kind=b.RSH_F32)), (b.RSH_ERR_BAD_OPTION, dict(y=P, ld=65))])
def test_dropout_refuses(status, change):
    a = dict(x=P, kind=b.RSH_F16, t=4, d=64, ld=64, drop=_drop(), y=P)
    a.update(change)
    drop = a["drop"]
    assert b.lib().rsh_dropout(a["x"], a["kind"], a["t"], a["d"], a["ld"], drop if drop is None else ctypes.byref(drop), a["y"], None) == status


def _norm(kind=b.RSH_NORM_RMS, weight=P, bias=None, stats=P, weight_type=b.RSH_F32, bias_type=b.RSH_F32, eps=1e-5):
    return b.rsh_norm_t(weight, bias, stats, weight_type, bias_type, kind, eps)


def _join(**change):
    a = dict(X=P, B=2 * P, gate=P, S=3 * P, Y=4 * P, t=4, d=64, ld_x=64, ld_b=64, ld_gate=0, after=_norm(), before=_norm(), drop=_drop(), type=b.RSH_F16,
             gate_type=b.RSH_F16, scale=1.0)
    a.update(change)
    return b.rsh_join_t(**a)


JOINS = [
    (b.RSH_ERR_BAD_OPTION, dict(type=b.RSH_MX4)), (b.RSH_ERR_BAD_OPTION, dict(t=0)), (b.RSH_ERR_BAD_OPTION, dict(d=-1)),
    (b.RSH_ERR_TOO_LARGE, dict(d=(1 << 21) + 1)), (b.RSH_ERR_BAD_OPTION, dict(ld_b=63)), (b.RSH_ERR_BAD_OPTION, dict(ld_b=(1 << 29) + 1)),
    (b.RSH_ERR_BAD_OPTION, dict(ld_gate=63)), (b.RSH_ERR_BAD_OPTION, dict(gate_type=b.RSH_MX4)), (b.RSH_ERR_BAD_OPTION, dict(gate_type=b.RSH_BF16)),
    (b.RSH_ERR_BAD_OPTION, dict(gate=None, ld_gate=64)), (b.RSH_ERR_BAD_OPTION, dict(after=_norm(weight_type=b.RSH_BF16))), (b.RSH_ERR_BAD_OPTION, dict(gate=P + 1)),
    (b.RSH_ERR_BAD_OPTION, dict(scale=INF)), (b.RSH_ERR_BAD_OPTION, dict(scale=float("nan"))), (b.RSH_ERR_BAD_OPTION, dict(drop=_drop(1 << 17))),
    (b.RSH_ERR_BAD_OPTION, dict(after=_norm(kind=3))), (b.RSH_ERR_BAD_OPTION, dict(before=_norm(eps=0))), (b.RSH_ERR_BAD_OPTION, dict(before=_norm(eps=INF))),
    (b.RSH_ERR_BAD_OPTION, dict(after=_norm(eps=float("nan")))), (b.RSH_ERR_BAD_OPTION, dict(after=_norm(weight_type=b.RSH_MX4))),
    (b.RSH_ERR_BAD_OPTION, dict(after=_norm(weight=P + 2))), (b.RSH_ERR_BAD_OPTION, dict(before=_norm(bias=P + 2))),
    (b.RSH_ERR_BAD_OPTION, dict(before=_norm(stats=P + 4))), (b.RSH_ERR_BAD_OPTION, dict(B=P + 1)), (b.RSH_ERR_BAD_OPTION, dict(S=3 * P + 1))]


@pytest.mark.parametrize("status,change", JOINS + [
    (b.RSH_ERR_NULL, dict(X=None)), (b.RSH_ERR_NULL, dict(B=None)), (b.RSH_ERR_NULL, dict(S=None)), (b.RSH_ERR_NULL, dict(Y=None)),
    (b.RSH_ERR_NULL, dict(before=_norm(kind=b.RSH_NORM_NONE))), (b.RSH_ERR_NULL, dict(B=None, S=None, Y=None, before=_norm(kind=b.RSH_NORM_NONE))),
    (b.RSH_ERR_BAD_OPTION, dict(ld_x=63)), (b.RSH_ERR_BAD_OPTION, dict(S=P)), (b.RSH_ERR_BAD_OPTION, dict(S=2 * P)),
    (b.RSH_ERR_BAD_OPTION, dict(Y=P)), (b.RSH_ERR_BAD_OPTION, dict(Y=2 * P)), (b.RSH_ERR_BAD_OPTION, dict(Y=3 * P)),
    (b.RSH_ERR_BAD_OPTION, dict(B=None, S=None, Y=P)), (b.RSH_ERR_BAD_OPTION, dict(before=_norm(eps=1e-45)))])
def test_joins_refuse(status, change):
    assert b.lib().rsh_join_forward(ctypes.byref(_join(**change)), None) == status


def test_nothing_to_join():
    assert b.lib().rsh_join_forward(None, None) == b.RSH_ERR_NULL
    assert b.lib().rsh_join_backward(None, None, None) == b.RSH_ERR_NULL
    assert b.lib().rsh_join_backward(ctypes.byref(_join()), None, None) == b.RSH_ERR_NULL


def _gradients(**change):
    a = {n: P for n, _ in b.rsh_join_gradients_t._fields_}
    a.update(after_bias=None, before_bias=None, ld_ds=64, ld_dy=64)
    a.update(change)
    return b.rsh_join_gradients_t(**a)


@pytest.mark.parametrize("status,join,gradients", [(s, c, {}) for s, c in JOINS] + [
    (b.RSH_ERR_NULL, {}, dict(dS=None, dY=None)), (b.RSH_ERR_NULL, {}, dict(work=None)), (b.RSH_ERR_NULL, dict(X=None), {}),
    (b.RSH_ERR_NULL, dict(before=_norm(stats=None)), {}), (b.RSH_ERR_NULL, dict(after=_norm(stats=None)), {}),
    (b.RSH_ERR_NULL, {}, dict(dX=None, dB=None, dgate=None, after_weight=None, before_weight=None)),
    (b.RSH_ERR_BAD_OPTION, dict(B=None), {}), (b.RSH_ERR_BAD_OPTION, dict(gate=None), {}), (b.RSH_ERR_BAD_OPTION, {}, dict(after_bias=P)),
    (b.RSH_ERR_BAD_OPTION, {}, dict(before_bias=P)), (b.RSH_ERR_BAD_OPTION, dict(after=_norm(weight=None)), {}),
    (b.RSH_ERR_BAD_OPTION, dict(before=_norm(kind=b.RSH_NORM_NONE)), {}), (b.RSH_ERR_BAD_OPTION, {}, dict(dY=None)),
    (b.RSH_ERR_BAD_OPTION, {}, dict(ld_ds=63)), (b.RSH_ERR_BAD_OPTION, {}, dict(ld_dy=63)), (b.RSH_ERR_BAD_OPTION, {}, dict(work=P + 4)),
    (b.RSH_ERR_BAD_OPTION, {}, dict(dX=P + 1)), (b.RSH_ERR_BAD_OPTION, {}, dict(after_weight=P + 2))])
def test_gradients_of_joins_refuse(status, join, gradients):
    assert b.lib().rsh_join_backward(ctypes.byref(_join(**join)), ctypes.byref(_gradients(**gradients)), None) == status


def _adapters(**change):
    a = dict(X=P, Y=P, A=P, B=P, index=P, scales=P, out=2 * P, kept=P, t=4, k=64, m=32, ld_x=64, ld_y=32, n=3, r=8, type=b.RSH_F16, index_size=4)
    a.update(change)
    return b.rsh_adapters_t(**a)


ADAPTERS = [
    (b.RSH_ERR_NULL, dict(A=None)), (b.RSH_ERR_NULL, dict(B=None)), (b.RSH_ERR_NULL, dict(index=None)), (b.RSH_ERR_BAD_OPTION, dict(t=0)),
    (b.RSH_ERR_BAD_OPTION, dict(k=0)), (b.RSH_ERR_BAD_OPTION, dict(m=-1)), (b.RSH_ERR_BAD_OPTION, dict(n=0)), (b.RSH_ERR_BAD_OPTION, dict(r=0)),
    (b.RSH_ERR_BAD_OPTION, dict(t=1 << 31)), (b.RSH_ERR_TOO_LARGE, dict(n=4097)), (b.RSH_ERR_TOO_LARGE, dict(r=513)),
    (b.RSH_ERR_TOO_LARGE, dict(k=(1 << 21) + 1)), (b.RSH_ERR_TOO_LARGE, dict(m=(1 << 21) + 1)), (b.RSH_ERR_BAD_OPTION, dict(type=b.RSH_F32)),
    (b.RSH_ERR_BAD_OPTION, dict(index_size=2)), (b.RSH_ERR_BAD_OPTION, dict(index=P + 4, index_size=8)), (b.RSH_ERR_BAD_OPTION, dict(scales=P + 2)),
    (b.RSH_ERR_BAD_OPTION, dict(kept=P + 8)), (b.RSH_ERR_BAD_OPTION, dict(A=P + 1)), (b.RSH_ERR_BAD_OPTION, dict(ld_x=63)),
    (b.RSH_ERR_BAD_OPTION, dict(ld_y=31))]


@pytest.mark.parametrize("status,change", ADAPTERS + [(b.RSH_ERR_NULL, dict(X=None)), (b.RSH_ERR_NULL, dict(out=None)),
                                                      (b.RSH_ERR_BAD_OPTION, dict(out=P, ld_y=40))])
def test_adapters_refuse(status, change):
    assert b.lib().rsh_adapters_forward(ctypes.byref(_adapters(**change)), P, None) == status


@pytest.mark.parametrize("status,change,call", [(s, c, {}) for s, c in ADAPTERS] + [
    (b.RSH_ERR_NULL, {}, dict(dout=None)), (b.RSH_ERR_NULL, {}, dict(dX=None, dA=None, dB=None)), (b.RSH_ERR_NULL, dict(X=None), {}),
    (b.RSH_ERR_NULL, dict(kept=None), {}), (b.RSH_ERR_NULL, {}, dict(work=None)), (b.RSH_ERR_BAD_OPTION, {}, dict(work=P + 8)),
    (b.RSH_ERR_BAD_OPTION, {}, dict(ld=31)), (b.RSH_ERR_BAD_OPTION, {}, dict(dA=P + 1))])
def test_gradients_of_adapters_refuse(status, change, call):
    a = dict(dout=P, ld=32, dX=P, dA=P, dB=P, work=P)
    a.update(call)
    assert b.lib().rsh_adapters_backward(ctypes.byref(_adapters(**change)), *a.values(), None) == status


def test_work_sizes():
    L, n = b.lib(), ctypes.c_int64(-1)
    assert L.rsh_adapters_forward(ctypes.byref(_adapters()), None, None) == b.RSH_ERR_NULL      # something is kept
    assert L.rsh_adapters_forward(ctypes.byref(_adapters(t=257, kept=None)), None, None) == b.RSH_ERR_NULL
    assert L.rsh_adapters_forward_work(4, 64, 32, 3, 8, 0, ctypes.byref(n)) == 0 and n.value == 0      # one launch, nothing between
    for f in (lambda *a: L.rsh_adapters_forward_work(*a[:5], 1, a[5]), L.rsh_adapters_backward_work):
        for t in (1, 256, 257, 100000):
            assert f(t, 64, 32, 3, 8, ctypes.byref(n)) == 0 and n.value >= 4 * t * 16
        assert f(4, 64, 32, 3, 8, None) == b.RSH_ERR_NULL and f(4, 64, 32, 0, 8, ctypes.byref(n)) == b.RSH_ERR_BAD_OPTION and n.value == 0
    assert L.rsh_adapters_kept(300, 3, 20, ctypes.byref(n)) == 0 and n.value >= 4 * 300 * 32 and L.rsh_adapters_kept(300, 3, 20, None) == b.RSH_ERR_NULL
    assert L.rsh_adapters_kept(300, 4097, 20, ctypes.byref(n)) == b.RSH_ERR_TOO_LARGE and n.value == 0
    for d in (64, 8192, 8193):
        assert L.rsh_join_backward_work(100, d, 3, ctypes.byref(n)) == 0 and n.value >= 4 * 3 * d
        assert L.rsh_join_backward_work(100, d, 0, ctypes.byref(n)) == 0 and n.value == (16 * 100 if d > 8192 else 0)
    assert L.rsh_join_backward_work(100, 64, 6, ctypes.byref(n)) == b.RSH_ERR_BAD_OPTION and L.rsh_join_backward_work(100, 64, 1, None) == b.RSH_ERR_NULL


def test_calls_without_a_gpu_refuse():
    """Nothing falls back to another device: operands in host memory are refused by name."""
    import torch

    from paper_2603_08734_amd import adapters, dropout, residual
    x = torch.zeros((2, 32), dtype=torch.float16)
    for call, match in ((lambda: residual.norm(x, residual.Norm()), "X"), (lambda: residual.join(x, x), "X"),
                        (lambda: dropout.dropout(x, dropout.Drop(0.1, 1)), "X"), (lambda: dropout.Drop(0.1, torch.zeros(1, dtype=torch.int64)), "seed"),
                        (lambda: dropout.Drop(1.5, 1), "p"), (lambda: dropout.Drop(float("nan"), 1), "p"), (lambda: residual.Norm("batch"), "kind"),
                        (lambda: residual.Norm(eps=0.0), "eps"), (lambda: residual.Norm(eps=1e-45), "eps"),
                        (lambda: adapters.add(x, x, x[:, None], x[:, None], torch.zeros(2, dtype=torch.int64)), "one GPU")):
        with pytest.raises(ValueError, match=match):
            call()


def test_a_drop_does_not_change():
    """A backward pass draws the forward pass's numbers from it again."""
    import copy
    import pickle
    from paper_2603_08734_amd.dropout import Drop
    drop = Drop(0.3, -5, 7)
    for name in ("share", "seed", "offset"):
        with pytest.raises(AttributeError):
            setattr(drop, name, 1)
    for other in (drop, copy.deepcopy(drop), pickle.loads(pickle.dumps(drop))):
        assert (other.share, other.seed, other.offset) == (round(0.3 * 65536), (1 << 64) - 5, 7)
