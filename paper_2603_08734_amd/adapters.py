"""Low-rank adapters of many requests at once beside a projection that they share.

    Y = mx4.product(X, W4)                              # or any other projection [t, m] of X [t, k], shared by all requests
    Y = adapters.add(Y, X, A, B, index, scales)         # row j: Y_j + scales[i] (X_j A[i]^T) B[i] with i = index[j]

A [n, r, k] and B [n, r, m]: n adapters of rank r, both factors rank first (products along their rows serve the forward and the backward
pass alike).  Tokens may come in any order; one whose index is not 0 .. n - 1 has no adapter and keeps its row of Y.  Binary16 or bfloat16;
X A[i]^T stays in fp32 between the two products and enters the second with all of its bits, and results are rounded once.  Up to 4096 adapters of
rank up to 512 and 2^28 tokens.  Autograd-aware (reverse mode, first derivatives) in Y, X, A
and B; scales are constants.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding
from .dropout import MOST
from .mx4 import HALVES, _on, _rows, _tangent

_FORWARD_MODE = "adapters have no forward-mode derivative: call them on detached operands"


def _struct(X, ld_x, Y, ld_y, A, B, index, scales, out, kept, t, k, m):
    a = binding._address
    return binding.rsh_adapters_t(a(X), a(Y), A.data_ptr(), B.data_ptr(), index.data_ptr(), a(scales), a(out), a(kept), t, k, m, ld_x, ld_y, A.shape[0],
                                  A.shape[1], HALVES[A.dtype], index.element_size())


def _forward(Y, X, A, B, index, scales, keep):
    (t, k), m = X.shape, Y.shape[1]
    x, ld_x = _rows(X, MOST)
    y, ld_y = _rows(Y, MOST)
    out = Y.new_empty((t, m))
    kept = binding.adapters_kept(X, t, A.shape[0], A.shape[1]) if keep else None
    with _on(x.get_device()):
        binding.adapters_forward(_struct(x, ld_x, y, ld_y, A, B, index, scales, out, kept, t, k, m), x)
    return out, kept


def _backward(ctx, dout):
    if _tangent(dout):
        raise ValueError(_FORWARD_MODE)
    X, A, B, index, scales, kept = ctx.saved_tensors
    t, m, k = dout.shape[0], B.shape[2], A.shape[2]
    want_y, want_x, want_a, want_b = ctx.needs_input_grad[:4]
    dX = dout.new_empty((t, k)) if want_x else None
    dA = torch.empty_like(A) if want_a else None
    dB = torch.empty_like(B) if want_b else None
    if want_x or want_a or want_b:
        g, ld_g = _rows(dout, MOST)
        x, ld_x = _rows(X, MOST) if want_a else (None, 0)
        with _on(g.get_device()):
            binding.adapters_backward(_struct(x, ld_x, None, 0, A, B, index, scales, None, kept, t, k, m), g, ld_g, dX, dA, dB)
    return dout if want_y else None, dX, dA, dB, None, None


_backward_once = once_differentiable(_backward)


class _Adapt(torch.autograd.Function):
    @staticmethod
    def forward(ctx, Y, X, A, B, index, scales):
        out, kept = _forward(Y, X, A, B, index, scales, any(ctx.needs_input_grad[1:4]))
        ctx.save_for_backward(X if ctx.needs_input_grad[2] else None, A, B, index, scales, kept)
        return out

    @staticmethod
    def backward(ctx, dout):
        # where the gradients' own graph is wanted, it ends here with an error
        return _backward_once(ctx, dout) if torch.is_grad_enabled() else _backward(ctx, dout)


def _refuse(Y, X, A, B, index, scales):
    """Say what does not fit."""
    for name, v in (("Y", Y), ("X", X), ("A", A), ("B", B), ("index", index)):
        if not isinstance(v, torch.Tensor):
            raise TypeError(f"{name}: expected a tensor, got {type(v)}")
    if X.dtype not in HALVES or any(v.dtype != X.dtype for v in (Y, A, B)):
        raise TypeError(f"expected one type for Y, X, A and B, one of {list(HALVES)}; got {Y.dtype}, {X.dtype}, {A.dtype} and {B.dtype}")
    if index.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"index: expected int32 or int64, got {index.dtype}")
    if (X.dim() < 1 or Y.dim() < 1 or A.dim() != 3 or B.dim() != 3 or A.shape[:2] != B.shape[:2] or A.shape[2] != X.shape[-1] or B.shape[2] != Y.shape[-1] or
            X.shape[:-1] != Y.shape[:-1] or index.shape != X.shape[:-1]):
        raise ValueError(f"Y {tuple(Y.shape)}, X {tuple(X.shape)}, A {tuple(A.shape)}, B {tuple(B.shape)} and index {tuple(index.shape)} do not fit: "
                         "expected [..., m], [..., k], [n, r, k], [n, r, m] and [...]")
    if scales is not None and (not isinstance(scales, torch.Tensor) or scales.dtype != torch.float32 or tuple(scales.shape) != (A.shape[0],)):
        raise ValueError(f"scales: expected fp32 ({A.shape[0]},) or None, got {getattr(scales, 'dtype', type(scales))} {tuple(getattr(scales, 'shape', ()))}")
    devices = {str(v.device) for v in (Y, X, A, B, index, scales) if v is not None}
    if len(devices) > 1 or not X.is_cuda:
        raise ValueError(f"operands are on {sorted(devices)}; expected one GPU")
    if scales is not None and scales.requires_grad and torch.is_grad_enabled():
        raise ValueError("scales have no gradient: pass them detached")
    if _tangent(*(v for v in (Y, X, A, B, scales) if v is not None)):
        raise ValueError(_FORWARD_MODE)


def _fits(Y, X, A, B, index, scales) -> bool:
    """The ordinary case of what is refused otherwise: matrices on one GPU."""
    for v in (Y, X, A, B, index):
        if not isinstance(v, torch.Tensor):
            return False
    dtype, device = X.dtype, X.get_device()
    if X.dim() != 2 or Y.dim() != 2 or A.dim() != 3 or B.dim() != 3 or dtype not in HALVES or index.dtype not in (torch.int32, torch.int64) or device < 0:
        return False
    (t, k), (n, r, ka), m = X.shape, A.shape, Y.shape[1]
    if Y.shape[0] != t or ka != k or B.shape != (n, r, m) or index.shape != (t,) or not Y.dtype == A.dtype == B.dtype == dtype:
        return False
    if not Y.get_device() == A.get_device() == B.get_device() == index.get_device() == device:
        return False
    return scales is None or (isinstance(scales, torch.Tensor) and scales.dtype == torch.float32 and scales.shape == (n,) and
                              scales.get_device() == device and not scales.requires_grad and not _tangent(scales))


def add(Y, X, A, B, index, scales=None):
    """Y + scales[i] (X A[i]^T) B[i] for every token, i its index: X [..., k], Y [..., m], index [...] int32 or int64, scales fp32 [n] or None for
    ones."""
    if not _fits(Y, X, A, B, index, scales) or _tangent(Y, X, A, B):
        _refuse(Y, X, A, B, index, scales)
    k, m = X.shape[-1], Y.shape[-1]
    grads = torch.is_grad_enabled() and any(v.requires_grad for v in (Y, X, A, B))
    if 0 in (Y.numel(), X.numel(), A.numel(), B.numel()):
        # no sums: Y, and zeros as the others' gradients, whatever the operands hold
        return Y + sum(v.reshape(-1)[:0].sum() for v in (X, A, B)) if grads else Y.clone()
    flat = X.dim() == 2
    rows = [Y, X, index] if flat else [Y.reshape(-1, m), X.reshape(-1, k), index.reshape(-1)]
    A, B, index = A.contiguous(), B.contiguous(), rows[2].contiguous()
    scales = scales if scales is None else scales.detach().contiguous()
    out = _Adapt.apply(rows[0], rows[1], A, B, index, scales) if grads else _forward(rows[0], rows[1], A, B, index, scales, False)[0]
    return out if flat else out.reshape(Y.shape)
