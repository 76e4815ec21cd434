"""The gated feed-forward block H = act(X Wg^T) * (X Wu^T), forward and backward, in kernels of the library.

    H = ffn.gated(X, W_gate, W_up, "silu")     # binary16 or bfloat16, X [..., d], weights [f, d]; autograd-aware (reverse mode)
    H = ffn.gated(X, Wg4, Wu4, "silu")         # the weights in 4 bits (mx4.quantize), for serving

Both projections, the activation and the product run as one kernel (``rsh_gated_forward``): sums are fp32 until H is rounded.
A forward pass that will be differentiated keeps both projections in fp32; the backward pass
(``rsh_gated_backward``) forms their gradients in one pass over them, rounds those to the inputs' type, and multiplies.  In binary16
that rounding has the type's range: scale the loss, as for any gradients in binary16.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding
from .binding import Plan
from .mx4 import HALVES, Mx4, _no_gradient, _on, _rows, _tangent, product

_FORWARD_MODE = "the gated block and its gradients have no forward-mode derivative: call them on detached operands"
ACTIVATIONS = {"silu": binding.RSH_ACT_SILU, "gelu": binding.RSH_ACT_GELU, "relu": binding.RSH_ACT_RELU}


def _weights(Wg, Wu):
    """Both weights as matrices with one row stride, and that."""
    Wg, ld = _rows(Wg)
    Wu, ld_u = _rows(Wu)
    return (Wg, Wu, ld) if ld == ld_u else (Wg.contiguous(), Wu.contiguous(), Wg.shape[1])


def _forward(X, Wg, Wu, act, keep):
    x, ld_x = _rows(X)
    wg, wu, ld_w = _weights(Wg, Wu)
    with _on(x.get_device()):
        return binding.gated_forward(x, HALVES[x.dtype], ld_x, wg, wu, ld_w, None, None, act, wg.shape[0], keep)


def _backward(ctx, dH):
    if _tangent(dH):
        raise ValueError(_FORWARD_MODE)
    X, Wg, Wu, kept = ctx.saved_tensors
    x, ld_x = _rows(X)
    wg, wu, ld_w = _weights(Wg, Wu)
    dH, ld_h = _rows(dH)
    with _on(x.get_device()):
        return (*binding.gated_backward(x, HALVES[x.dtype], ld_x, wg, wu, ld_w, kept, dH, ld_h, ctx.act, ctx.needs_input_grad), None)


_backward_once = once_differentiable(_backward)


class _Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, X, Wg, Wu, act):
        H, kept = _forward(X, Wg, Wu, act, True)
        ctx.act = act
        ctx.save_for_backward(X, Wg, Wu, kept)
        return H

    @staticmethod
    def backward(ctx, dH):
        # where the gradients' own graph is wanted, it ends here with an error
        return _backward_once(ctx, dH) if torch.is_grad_enabled() else _backward(ctx, dH)


def _refuse(X, W_gate, W_up, activation):
    """Say what does not fit."""
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation: expected one of {list(ACTIVATIONS)}, got {activation!r}")
    if not isinstance(X, torch.Tensor) or X.dim() < 1:
        raise TypeError(f"X: expected a tensor [..., d], got {type(X)}")
    four = isinstance(W_gate, Mx4)
    if four != isinstance(W_up, Mx4):
        raise TypeError("W_gate and W_up: either both in 4 bits or neither")
    if tuple(W_up.shape) != tuple(W_gate.shape) or len(W_gate.shape) != 2 or W_gate.shape[1] != X.shape[-1]:
        raise ValueError(f"X {tuple(X.shape)}, W_gate {tuple(W_gate.shape)} and W_up {tuple(W_up.shape)} do not fit")
    if X.dtype not in HALVES or (not four and (W_gate.dtype != X.dtype or W_up.dtype != X.dtype)):
        raise TypeError(f"expected one type for X and 16-bit weights, one of {list(HALVES)}; X is {X.dtype}")
    raise ValueError(f"X is on {X.device}, W_gate on {W_gate.device}, W_up on {W_up.device}; expected one GPU")


def gated(X, W_gate, W_up, activation: str = "silu"):
    """act(X W_gate^T) * (X W_up^T): X [..., d], weights [f, d] of X's type or in 4 bits, result [..., f]."""
    act, four = ACTIVATIONS.get(activation), isinstance(W_gate, Mx4)
    if act is None or not isinstance(X, torch.Tensor) or X.dim() < 1 or X.dtype not in HALVES or four != isinstance(W_up, Mx4):
        _refuse(X, W_gate, W_up, activation)
    shape, device = W_gate.shape, X.get_device()
    a, b = (W_gate.codes, W_up.codes) if four else (W_gate, W_up)
    if (W_up.shape != shape or len(shape) != 2 or shape[1] != X.shape[-1] or device < 0 or a.get_device() != device or b.get_device() != device or
            not (four or a.dtype == b.dtype == X.dtype)):
        _refuse(X, W_gate, W_up, activation)
    f, d = shape
    flat = X.dim() == 2
    rows = X if flat else X.reshape(-1, d) if d else X.reshape(X.shape[:-1].numel(), 0)
    if four:
        _no_gradient(X)
    elif _tangent(X, W_gate, W_up):
        raise ValueError(_FORWARD_MODE)
    if rows.shape[0] == 0 or f == 0 or d == 0:
        # no sums: zeros, whose gradients are zeros
        H = rows.sum() * 0 + rows.new_zeros((rows.shape[0], f))
        H = H if four else H + (W_gate.sum() + W_up.sum()) * 0
    elif four:
        x, ld_x = _rows(rows)
        with _on(device):
            H = binding.gated_forward(x, HALVES[x.dtype], ld_x, a, b, 0, W_gate.scales, W_up.scales, act, f, False)[0]
    elif (X.requires_grad or W_gate.requires_grad or W_up.requires_grad) and torch.is_grad_enabled():
        H = _Gated.apply(rows, W_gate, W_up, act)
    else:
        H = _forward(rows, W_gate, W_up, act, False)[0]
    return H if flat else H.reshape(*X.shape[:-1], f)


class FeedForward:
    """A gated feed-forward layer as it is served: Y = W_down (act(X W_gate^T) * (X W_up^T)).

    W_gate, W_up: [f, d] of the activations' type, or in 4 bits (``mx4.quantize``).  W_down: [d, f] in 4 bits, or a ``Plan`` of the
    pruned weight for exactly as many tokens as X has (binary16: the sparse product takes the tokens as columns).  Either way the layer
    has no gradient, and operands that want one are refused while gradients are recorded."""

    def __init__(self, W_gate, W_up, W_down, activation: str = "silu"):
        if not isinstance(W_down, (Mx4, Plan)):
            raise TypeError(f"W_down: expected Mx4 or Plan, got {type(W_down)}")
        shape = (W_down.n_rows, W_down.n_cols) if isinstance(W_down, Plan) else W_down.shape
        if len(W_gate.shape) != 2 or shape[1] != W_gate.shape[0]:
            raise ValueError(f"W_gate {tuple(W_gate.shape)} and W_down {shape}: expected [f, d] and [d, f]")
        self.W_gate, self.W_up, self.W_down, self.activation = W_gate, W_up, W_down, activation

    def __call__(self, X):
        """X: [t, d]; result [t, d] of its type, from a ``Plan`` the transposed view of a [d, t] matrix."""
        if not isinstance(X, torch.Tensor) or X.dim() != 2:
            raise ValueError(f"X: expected a matrix, got {tuple(X.shape) if isinstance(X, torch.Tensor) else type(X)}")
        if isinstance(self.W_down, Plan) and (X.dtype != torch.float16 or X.shape[0] != self.W_down.N):
            raise ValueError(f"the plan is for {self.W_down.N} tokens of binary16, got {X.shape[0]} of {X.dtype}")
        _no_gradient(*(m for m in (X, self.W_gate, self.W_up) if isinstance(m, torch.Tensor)))
        H = gated(X, self.W_gate, self.W_up, self.activation)
        if isinstance(self.W_down, Mx4):
            return product(H, self.W_down)
        Y = torch.empty((self.W_down.n_rows, self.W_down.N), dtype=torch.float16, device=H.device)
        with _on(H.get_device()):
            self.W_down.spmm_f16(H.t().contiguous(), Y)
        return Y.t()
